// Softmax attention over windows of any length, forward and backward (bf16 in,
// fp32 accumulation, head dimension 64 or 128), key/value heads shared by
// groups of query heads, keys past a sequence's length and (causal) past the
// query's own position left out.
//
// The scores of 32 keys at a time never leave the registers: the forward keeps
// each query's running maximum m and sum l of exp(S - m) and rescales what it
// has accumulated when m grows.  The backward makes P = exp(S - lse) again from
// the forward's lse instead of reading it.
//
// P, and in the backward dS, are rounded to bf16 for the second products: the matrix
// unit's fp32 products run at an eighth of the rate (154 and 1290 TFLOP/s).  Each adds to
// a result about what the rounding of the result itself does (0.0024 in norm for 0.0017).
// In calls of few scores nothing is left out (ga_rest).
//
// Tiles, fragments and the transposed scores (a lane owns a query, or a key in
// the key/value gradients, and 16 rows of a 32 x 32 tile) are tile64.h's.
// A tile of 128 columns is two of 64.
#include "hcmix_internal.h"
#include "device_common.h"
#include "tile64.h"

#include <algorithm>
#include <type_traits>

namespace hcmix {

namespace {

constexpr int GA_THREADS = 256;
constexpr float GA_LOG2E = 1.4426950408889634f, GA_LN2 = 0.6931471805599453f;
constexpr int GA_STEP = 32;         // rows of a streamed tile
// Rows of a block of four waves (32 to a wave).
constexpr int GA_ROWS = 128;

// A buffer's index known at compile time: its LDS addresses are then offsets in
// the instructions, not a third of a turn's vector work.
template <int I>
using Const = std::integral_constant<int, I>;

// A block's waves meet, each with at most N of its copies on their way and its LDS
// reads done.
template <int N>
__device__ __forceinline__ void ga_meet() {
  static_assert(N < 16, "");
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0070 | N);       // vmcnt N, expcnt any, lgkmcnt 0
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Fragments of a tile of R rows.
template <int R>
__device__ __forceinline__ bf16x8 ga_frag(const bf16* t, int r0, int c0, int lane) {
  return att_frag(t + (c0 >> 6) * R * HD, r0, c0 & 63, lane);
}
template <int R>
__device__ __forceinline__ bf16x8 ga_trfrag(const bf16* t, int k0, int c0, int lane) {
  return att_trfrag(t + (c0 >> 6) * R * HD, k0, c0 & 63, lane);
}

// What att_pack's rounding leaves of those registers, rounded in its turn.  In a call
// of few scores the roundings of P and dS do not average out: of 1024 and fewer, dq
// and dk were up to 1.5 to 2.8 times as far off as their own rounding to bf16 leaves
// them, 1.42 in the mean; from 131072 on 1.45 at most (scores of order 1).  Such a call
// waits for latencies, so that the FINE kernels' second products with what is left, and
// what they take for D, cost it less than they compute (1 x 128, 2 heads of 64 5.2 + 12.7
// us, 5.4 + 14.6; 1 x 16 of 512, 4 heads of 128 9.0 + 18.7, 10.3 + 23.5), and its results
// are as near as their own rounding.
__device__ __forceinline__ bf16x8 ga_rest(const f32x16& s, int m) {
  bf16x8 v;
#pragma unroll
  for (int e = 0; e < 8; e++) v[e] = to_bf16(s[8 * m + e] - (float)to_bf16(s[8 * m + e]));
  return v;
}

// A tile's way straight into LDS: rows row0 .. + R of an array with rows `stride`
// elements apart; rows at `valid` and behind are copies of the last before it
// (finite where the valid ones are: their P is 0).  A wave copies every W-th piece
// of 8 rows by 64 columns, lane l the 16 bytes that the swizzle wants there.
template <int D, int R, int W = 4>
struct TileDma {
  static constexpr int PER = D / 64 * R / 8 / W;     // pieces of a wave
  unsigned off[PER];                                 // source bytes from row row0
  int wave, lane;
  __device__ __forceinline__ unsigned at(int j, int last, unsigned stride) const {
    const int blk = wave + W * j, r = blk % (R / 8) * 8 + (lane >> 3);
    return 2 * ((unsigned)min(r, last) * stride + blk / (R / 8) * HD + 8 * ((lane & 7) ^ att_sw(r)));
  }
  __device__ __forceinline__ TileDma(int w, int l, int64_t stride) : wave(w), lane(l) {
#pragma unroll
    for (int j = 0; j < PER; j++) off[j] = at(j, R, (unsigned)stride);
  }
  __device__ __forceinline__ void load(const bf16* base, int64_t stride, int row0, int valid,
                                       bf16* tile) const {
    const bf16* src = uniform_base(base + (size_t)row0 * stride);
    if (row0 + R <= valid) {
#pragma unroll
      for (int j = 0; j < PER; j++) dma16_at(src, off[j], tile + (wave + W * j) * 512);
    } else {
#pragma unroll
      for (int j = 0; j < PER; j++)
        dma16_at(src, at(j, valid - 1 - row0, (unsigned)stride), tile + (wave + W * j) * 512);
    }
  }
};

// This block's (sequence, head, tile).  Under a causal mask a head's tiles differ
// in work up to its whole length, and a heavy one that starts late is waited for:
// tiles come in order of their work, the heaviest of all heads first (8 x 4096,
// 16 heads over 4: head after head, dK and dV took 870 us, so 630).  The heads are
// dealt to the XCDs (blocks go to the 8 of them in turn), so that an L2 holds the
// keys and values that a group's heads and a head's tiles share, and on an XCD
// taken in chunks of four rounds of 64 blocks (two: 1.5% slower, all at once: the
// same).  A number of heads that is no multiple of 8 is spread over the XCDs as it
// comes.
struct Item {
  int b, h, tile;
};
__device__ __forceinline__ bool ga_item(int batch, int heads, int tiles, bool last_first, Item* it) {
  const unsigned all = (unsigned)batch * heads;
  unsigned bh, t;
  if (blockIdx.x >= all * tiles) return false;
  if (all % 8 == 0) {
    const unsigned per = all / 8, xcd = blockIdx.x % 8, k = blockIdx.x / 8;
    const unsigned size = min(per, (255u + tiles) / tiles);
    const unsigned chunk = k / (size * tiles), r = k - chunk * size * tiles;
    const unsigned n = min(size, per - chunk * size);
    t = r / n;
    bh = xcd * per + chunk * size + (r - t * n);
  } else {
    t = blockIdx.x / all;
    bh = blockIdx.x - t * all;
  }
  it->b = bh / heads;
  it->h = bh - it->b * heads;
  it->tile = last_first ? tiles - 1 - t : t;
  return true;
}

__device__ __forceinline__ int ga_length(const GroupedArgs& a, int b) {
  int n = a.n_k;
  if (a.lengths) {
    n = __builtin_amdgcn_readfirstlane(a.lengths[b]);
    n = n < 0 ? 0 : n > a.n_k ? a.n_k : n;
  }
  return n;
}

// Rows row0 + lane % 32 of an array as MFMA operands: 8 columns per lane and k16
// step; rows at `valid` and behind are zeros.
template <int D>
__device__ __forceinline__ void ga_rows(bf16x8 (&f)[D / 16], const bf16* base, size_t stride,
                                        int row0, int valid, int lane) {
  const int r = row0 + (lane & 31);
#pragma unroll
  for (int ks = 0; ks < D / 16; ks++) {
    u32x4 v = {0, 0, 0, 0};
    if (r < valid) v = *(const u32x4*)(base + (size_t)r * stride + 16 * ks + 8 * (lane >> 5));
    f[ks] = __builtin_bit_cast(bf16x8, v);
  }
}

// ---------------------------------------------------------------------------
// Forward
// ---------------------------------------------------------------------------
// A wave has 32 queries.  m grows only when a tile's largest score passes it
// by more than GA_SLACK (in log2 units; P and l then stay below 2^GA_SLACK and
// that times the number of keys, far from any limit), so that the rescaling of
// what has been accumulated, and the exchange of the maximum between the two
// lanes of a query, is a rare branch.  Tiles of 32 keys leave registers for more waves
// than 64 (64 x 256, 8 heads of 64 over 2 17.4 us with 64, 15.5; 8 x 4096, 8 of 128
// over 2 275, 261; 8 x 4096, 16 of 64 over 4 317, 311; 16 x 500 12.9, 13.6).
//
// A block is W waves of queries by KS sets that share its key tiles in turn and
// join at the end: 4 by 1, and where the blocks are few, so that a wave alone on
// its SIMD waits for itself and the longest block is the call's time, 2 by 4 (head
// dimension 64) or 2 by 2.  us, causal, 8 heads over 2, with 4 by 2, 2 by 4, 2 by
// 2: 1 x 1000 of 64 13.3, 10.8, 11.9; 2 x 2048 of 64 23.8, 21.0, 22.1; 3 x 1000 of
// 128 21.0, 21.4, 17.5; 2 x 2048 of 128 34.8, 32.0, 29.8.
constexpr float GA_SLACK = 8.f;

// Whether the loops of the forward and of dQ carry the next tile's products, which the
// matrix unit makes while the vector unit works on this one's (the last turn makes
// some that nothing takes).  With head dimension 64 the registers that this takes are
// better spent on a fourth wave of a SIMD, which hides the same: us of forward and
// backward with the products ahead, and so, 8 heads over 2: 64 x 256 15.4 + 44.7,
// 14.5 + 41.7; 300 x 64 16.5 + 45.8, 15.2 + 42.0; 8 x 4096, 16 over 4 303 + 936, the
// same.  128: 8 x 4096 252 + 892, 256 + 910 without.
constexpr bool ga_ahead(int D) { return D == 128; }

template <int D, int W, int KS, bool FINE = false>
__global__ __launch_bounds__(64 * W * KS, 2) void ga_fwd_kernel(GroupedArgs a) {
  constexpr int ROWS = 32 * W;
  constexpr bool AHEAD = ga_ahead(D);
  __shared__ __attribute__((aligned(1024))) bf16 sKV[KS][2][2][GA_STEP * D];   // keys, values
  Item it;
  if (!ga_item(a.batch, a.q_heads, (a.n_q + ROWS - 1) / ROWS, a.causal, &it)) return;
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const int wave = wave_index<W * KS>() % W, set = wave_index<W * KS>() / W;
  const int kvh = it.h / a.group, len = ga_length(a, it.b), off = a.n_k - a.n_q;
  const int blk0 = it.tile * ROWS, q0 = blk0 + 32 * wave;
  const bf16* qb = a.q + (size_t)it.b * a.n_q * a.q_stride + (size_t)it.h * D;
  const bf16* kb = a.k + (size_t)it.b * a.n_k * a.k_stride + (size_t)kvh * D;
  const bf16* vb = a.v + (size_t)it.b * a.n_k * a.v_stride + (size_t)kvh * D;
  // keys that the block's last query, and this wave's, sees; keys that all of its do
  const int blk_end = a.causal ? min(len, blk0 + ROWS + off) : len;
  const int wave_end = a.causal ? min(len, q0 + 32 + off) : len;
  const int full_end = a.causal ? min(len, q0 + 1 + off) : len;
  // tiles of the block, of this set (tile t of it is tile t KS + set), that this wave sees
  const int all = blk_end > 0 ? (blk_end + GA_STEP - 1) / GA_STEP : 0;
  const int turns = (all + KS - 1) / KS, tiles = (all - set + KS - 1) / KS;
  const int seen = q0 < a.n_q && wave_end > 0 ? (wave_end + GA_STEP - 1) / GA_STEP : 0;
  const int mine = (seen - set + KS - 1) / KS;
  bf16(*sK)[GA_STEP * D] = sKV[set][0];
  bf16(*sV)[GA_STEP * D] = sKV[set][1];
  bf16x8 qf[D / 16];
  ga_rows<D>(qf, qb, a.q_stride, q0, a.n_q, lane);
  f32x16 o[D / 32] = {};
  const float sc = a.scale * GA_LOG2E;
  float m = -3e38f, l = 0.f, limit = -INFINITY;      // limit: the score from which m grows
  const TileDma<D, GA_STEP, W> dk(wave, lane, a.k_stride), dv(wave, lane, a.v_stride);
  auto load_k = [&](int t, bf16* to) {
    if (t < tiles) dk.load(kb, a.k_stride, (t * KS + set) * GA_STEP, len, to);
  };
  auto load_v = [&](int t, bf16* to) {
    if (t < tiles) dv.load(vb, a.v_stride, (t * KS + set) * GA_STEP, len, to);
  };
  auto scores = [&](const bf16* tk, f32x16& r) {
    r = f32x16{};
#pragma unroll
    for (int ks = 0; ks < D / 16; ks++) r = mfma32(ga_frag<GA_STEP>(tk, 0, 16 * ks, lane), qf[ks], r);
  };
  auto turn = [&](auto buf, int t, f32x16& s, f32x16& next) {   // buf: t % 2
    wait_dma();
    __syncthreads();
    load_k(t + 1 + AHEAD, sK[AHEAD ? buf : buf ^ 1]);
    load_v(t + 1, sV[buf ^ 1]);
    if (t >= mine) return;               // wave-uniform
    if constexpr (!AHEAD) scores(sK[buf], s);
    const int k0 = (t * KS + set) * GA_STEP;
    if (k0 + GA_STEP > full_end) {
      asm volatile("; tile with keys that some query does not see");   // no selects elsewhere
      // register e of a lane: key k0 + 8 (e / 4) + 4 half + e % 4
      const int end = (a.causal ? min(len, q0 + (lane & 31) + 1 + off) : len) - k0 - 4 * half;
#pragma unroll
      for (int e = 0; e < 16; e++)
        if (8 * (e >> 2) + (e & 3) >= end) s[e] = -INFINITY;
    }
    float mx = s[0];
#pragma unroll
    for (int e = 1; e < 16; e++) mx = fmaxf(mx, s[e]);
    if (__any(mx > limit)) {
      // of the rows whose own scores ask for it: a row's result does not depend on others
      const float top = fmaxf(mx, __shfl_xor(mx, 32)), mn = top > limit ? fmaxf(m, top * sc) : m;
      const float alpha = __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      limit = (mn + GA_SLACK) / sc;
      l *= alpha;
#pragma unroll
      for (int d = 0; d < D / 32; d++)
#pragma unroll
        for (int e = 0; e < 16; e++) o[d][e] *= alpha;
    }
    if constexpr (AHEAD) scores(sK[buf ^ 1], next);
    const bf16* tv = sV[buf];
#pragma unroll
    for (int e = 0; e < 16; e++) {
      s[e] = __builtin_amdgcn_exp2f(fmaf(s[e], sc, -m));
      l += s[e];
    }
#pragma unroll
    for (int mm = 0; mm < 2; mm++) {
      const bf16x8 pf = att_pack(s, mm);
#pragma unroll
      for (int d = 0; d < D / 32; d++)
        o[d] = mfma32(ga_trfrag<GA_STEP>(tv, 16 * mm, 32 * d, lane), pf, o[d]);
    }
    if constexpr (FINE) {
#pragma unroll
      for (int mm = 0; mm < 2; mm++) {
        const bf16x8 pf = ga_rest(s, mm);
#pragma unroll
        for (int d = 0; d < D / 32; d++)
          o[d] = mfma32(ga_trfrag<GA_STEP>(tv, 16 * mm, 32 * d, lane), pf, o[d]);
      }
    }
  };
  if (turns) {
    f32x16 s, next;
    load_k(0, sK[0]);
    load_v(0, sV[0]);
    if constexpr (AHEAD) {
      load_k(1, sK[1]);
      wait_dma();
      __syncthreads();
      scores(sK[0], s);
    }
    for (int t = 0; t < turns; t += 2) {
      turn(Const<0>(), t, s, next);
      if (t + 1 < turns) turn(Const<1>(), t + 1, next, s);
    }
  }
  if constexpr (KS > 1) {
    // the other sets' sums to the first, through the tiles' place: [set][wave][register quad][lane]
    constexpr int QUADS = (D / 8 + 1) * 64;
    static_assert(sizeof(sKV) >= (KS - 1) * W * QUADS * sizeof(f32x4), "");
    f32x4* to = (f32x4*)sKV + wave * QUADS + lane;
    __syncthreads();
    if (set) {
      f32x4* mine = to + (set - 1) * W * QUADS;
#pragma unroll
      for (int d = 0; d < D / 32; d++)
#pragma unroll
        for (int g = 0; g < 4; g++)
          mine[(4 * d + g) * 64] = f32x4{o[d][4 * g], o[d][4 * g + 1], o[d][4 * g + 2], o[d][4 * g + 3]};
      mine[D / 8 * 64] = f32x4{m, l, 0.f, 0.f};
    }
    __syncthreads();
    if (set) return;
    for (int other = 1; other < KS; other++, to += W * QUADS) {
      const f32x4 ml = to[D / 8 * 64];
      const float mn = fmaxf(m, ml[0]), x = __builtin_amdgcn_exp2f(m - mn), y = __builtin_amdgcn_exp2f(ml[0] - mn);
      m = mn;
      l = l * x + ml[1] * y;
#pragma unroll
      for (int d = 0; d < D / 32; d++)
#pragma unroll
        for (int g = 0; g < 4; g++) {
          const f32x4 v = to[(4 * d + g) * 64];
#pragma unroll
          for (int r = 0; r < 4; r++) o[d][4 * g + r] = o[d][4 * g + r] * x + v[r] * y;
        }
    }
  }
  if (q0 >= a.n_q) return;
  l += __shfl_xor(l, 32);
  const float inv = l == 0.f ? 0.f : 1.f / l;      // 0: the row sees nothing
  const size_t os = (size_t)a.q_heads * D;
  bf16* ob = a.out + ((size_t)it.b * a.n_q + q0) * os + (size_t)it.h * D;
#pragma unroll
  for (int d = 0; d < D / 32; d++) att_store(ob + 32 * d, os, o[d], inv, lane, a.n_q - q0);
  if (half == 0 && q0 + lane < a.n_q)
    a.lse[((size_t)it.b * a.q_heads + it.h) * a.n_q + q0 + lane] =
        l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * GA_LN2;
}

// ---------------------------------------------------------------------------
// Backward, in two kernels: dQ by query tiles, dK and dV by key tiles, each
// making S and dP again (7 products of the 5 that one would need with atomics on
// dQ, whose order changes results).  Both stream tiles of 32 rows through up to four
// buffers in LDS; dK and dV, and dQ of head dimension 128, carry the next tile's S
// and dP while the vector unit works on this one's.
//
// With lanes and registers as in the forward, P = exp2((S - lse / scale) scale
// log2 e); a row that sees nothing takes -inf for -lse: its P is 0.
//
// D = sum_j P_j dP_j = dout . out.  The second form is one pass over two rows,
// but out is rounded to bf16, and dS = P (dP - D) cancels the more the fewer keys
// share a row: a row that sees one key has dS = 0, and got 2^-9 |dout| |out|
// instead (dq and dk of windows of 10 keys were 0.0046 off in all, 0.0024 so).
// So rows that see no more than 128 keys, which the buffers of all sets hold at once,
// take the first form, over sum_j P_j, which lse's own rounding keeps from being 1.  The
// others take D' = dout . out.  Its rounding adds nothing to see where scores are of order
// 1 (dq of rows of 129 and more keys 0.0024 off, as of fewer), but the more the fewer keys
// share a row's weight (0.0035 where scores are of order 3), so that FINE calls take the
// rest as well: D - D' = sum_j P_j (dP_j - D') / sum_j P_j, known behind the last key, and
// dq = sum_j P_j (dP_j - D') k_j - (D - D') sum_j P_j k_j.  The last sum is a product more
// (1 x 16 x 512, 4 heads 13.8 us for the whole backward without, 15.2; of 128 20.0, 23.4:
// a wave to a SIMD, for its registers).
// ---------------------------------------------------------------------------
constexpr int GA_BUFS = 4;

// What the dQ kernel leaves for the other, for each head and 32 rows: 32 of
// -lse / scale, then 32 of -D.
__device__ __forceinline__ size_t ga_stats(int bh, int n_q, int row0) {
  return ((size_t)bh * ((n_q + 31) / 32) + row0 / 32) * 64;
}

template <int D, int W, int KS, bool FINE = false>
__global__ __launch_bounds__(64 * W * KS, FINE && D == 128 ? 1 : 2) void ga_bwd_q_kernel(GroupedArgs a) {
  constexpr int ROWS = 32 * W;
  // Sets of waves on one SIMD hide what products ahead do: then two buffers are enough,
  // and the LDS of the others is a second block's (8 heads of 128 over 2: 3 x 1000 71.2
  // us for the whole backward with four and products ahead, 67.8 so; 1 x 4096, 8 over 4
  // 204, 197; of 64: 2 x 2048 68.8, 64.4).
  constexpr bool AHEAD = ga_ahead(D) && KS == 1;
  constexpr int BUFS = KS == 1 ? GA_BUFS : 2;
  __shared__ __attribute__((aligned(1024))) bf16 sKV[KS][2][BUFS][GA_STEP * D];   // keys, values
  Item it;
  if (!ga_item(a.batch, a.q_heads, (a.n_q + ROWS - 1) / ROWS, a.causal, &it)) return;
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const int wave = wave_index<W * KS>() % W, set = wave_index<W * KS>() / W;
  const int kvh = it.h / a.group, len = ga_length(a, it.b), off = a.n_k - a.n_q;
  const int blk0 = it.tile * ROWS, q0 = blk0 + 32 * wave;
  const size_t os = (size_t)a.q_heads * D;
  const bf16* kb = a.k + (size_t)it.b * a.n_k * a.k_stride + (size_t)kvh * D;
  const bf16* vb = a.v + (size_t)it.b * a.n_k * a.v_stride + (size_t)kvh * D;
  const int blk_end = a.causal ? min(len, blk0 + ROWS + off) : len;
  const int wave_end = a.causal ? min(len, q0 + 32 + off) : len;
  const int full_end = a.causal ? min(len, q0 + 1 + off) : len;
  // tiles as in the forward
  const int all = blk_end > 0 ? (blk_end + GA_STEP - 1) / GA_STEP : 0;
  const int turns = (all + KS - 1) / KS, tiles = (all - set + KS - 1) / KS;
  const int wave_tiles = q0 < a.n_q && wave_end > 0 ? (wave_end + GA_STEP - 1) / GA_STEP : 0;
  const int mine = (wave_tiles - set + KS - 1) / KS;
  bf16(*sK)[GA_STEP * D] = sKV[set][0];
  bf16(*sV)[GA_STEP * D] = sKV[set][1];
  const TileDma<D, GA_STEP, W> dk(wave, lane, a.k_stride), dv(wave, lane, a.v_stride);
  auto load = [&](auto buf, int t) {      // buf: t % BUFS
    if (t >= tiles) return;
    dk.load(kb, a.k_stride, (t * KS + set) * GA_STEP, len, sK[buf]);
    dv.load(vb, a.v_stride, (t * KS + set) * GA_STEP, len, sV[buf]);
  };
  load(Const<0>(), 0);
  load(Const<1>(), 1);
  if constexpr (BUFS == 4) {
    load(Const<2>(), 2);
    load(Const<3>(), 3);
  }
  bf16x8 qf[D / 16], of[D / 16];
  ga_rows<D>(qf, a.q + (size_t)it.b * a.n_q * a.q_stride + (size_t)it.h * D, a.q_stride, q0, a.n_q, lane);
  ga_rows<D>(of, a.dout + (size_t)it.b * a.n_q * os + (size_t)it.h * D, os, q0, a.n_q, lane);
  const float sc = a.scale * GA_LOG2E;
  // keys that this lane's query sees, and its statistics
  const int seen = a.causal ? min(len, q0 + (lane & 31) + 1 + off) : len;
  float start = -INFINITY, d = 0.f, z = 0.f, rounded = 0.f;
  // whether any row of the block takes D from P and dP, and any from out (block-uniform)
  constexpr int SHORT = GA_STEP * GA_BUFS;
  const bool from_p = (a.causal ? min(len, blk0 + 1 + off) : len) <= SHORT, from_out = all > GA_BUFS;
  bf16x8 xf[D / 16];
  if (from_out) ga_rows<D>(xf, a.out + (size_t)it.b * a.n_q * os + (size_t)it.h * D, os, q0, a.n_q, lane);
  if (q0 + (lane & 31) < a.n_q) {
    const float lse = a.lse[((size_t)it.b * a.q_heads + it.h) * a.n_q + q0 + (lane & 31)];
    start = lse == -INFINITY ? -INFINITY : -lse / a.scale;
  }
  wait_vmcnt<0>();
  __syncthreads();
  __shared__ float2 sD[KS][W][64];
  // x and y of all sets and both lanes of a query, in one order
  auto joined = [&](float x, float y) {
    if constexpr (KS > 1) {
      sD[set][wave][lane] = float2{x, y};
      __syncthreads();
      x = y = 0.f;
#pragma unroll
      for (int i = 0; i < KS; i++) {
        x += sD[i][wave][lane].x;
        y += sD[i][wave][lane].y;
      }
    }
    return float2{x + __shfl_xor(x, 32), y + __shfl_xor(y, 32)};
  };
  if (from_out) {
#pragma unroll
    for (int ks = 0; ks < D / 16; ks++)
#pragma unroll
      for (int e = 0; e < 8; e++) rounded += (float)xf[ks][e] * (float)of[ks][e];
    rounded += __shfl_xor(rounded, 32);
  }
  if (from_p) {
    const int held = min(mine, GA_BUFS / KS);
    for (int t = 0; t < held; t++) {
      f32x16 s = {}, dp = {};
#pragma unroll
      for (int ks = 0; ks < D / 16; ks++) {
        s = mfma32(ga_frag<GA_STEP>(sK[t], 0, 16 * ks, lane), qf[ks], s);
        dp = mfma32(ga_frag<GA_STEP>(sV[t], 0, 16 * ks, lane), of[ks], dp);
      }
#pragma unroll
      for (int e = 0; e < 16; e++) {
        float p = __builtin_amdgcn_exp2f((s[e] + start) * sc);
        if ((t * KS + set) * GA_STEP + 8 * (e >> 2) + 4 * half + (e & 3) >= seen) p = 0.f;
        d += p * dp[e];
        z += p;
      }
    }
    const float2 dz = joined(d, z);
    d = dz.y > 0.f ? dz.x / dz.y : dz.x;
  }
  if (seen > SHORT) d = rounded;
  if (q0 < a.n_q && !set)
    a.stats[ga_stats(it.b * a.q_heads + it.h, a.n_q, q0) + lane] = half ? -d : start;
  start *= sc;                            // -inf stays
  // FINE: sums of P (dP - D), of P, and of P K for what the first says
  f32x16 gq[D / 32] = {}, gp[FINE ? D / 32 : 1] = {};
  float left = 0.f;
  z = 0.f;
  auto scores = [&](auto buf, f32x16& s, f32x16& dp) {
    const bf16 *tk = sK[buf], *tv = sV[buf];
    s = f32x16{};
    dp = f32x16{};
#pragma unroll
    for (int ks = 0; ks < D / 16; ks++) {
      s = mfma32(ga_frag<GA_STEP>(tk, 0, 16 * ks, lane), qf[ks], s);
      dp = mfma32(ga_frag<GA_STEP>(tv, 0, 16 * ks, lane), of[ks], dp);
    }
  };
  auto turn = [&](auto buf, int t, f32x16& s, f32x16& dp, f32x16& s_next, f32x16& dp_next) {
    // tile t + 1 has landed when at most t + 2's loads are on their way
    if (BUFS == 4 && t + 2 < tiles) wait_vmcnt<2 * TileDma<D, GA_STEP, W>::PER>();
    else wait_vmcnt<0>();
    __syncthreads();
    if (t) load(Const<(buf + BUFS - 1) % BUFS>(), t + BUFS - 1);
    if (t >= mine) return;                // wave-uniform
    if constexpr (!AHEAD) scores(buf, s, dp);
    if ((t * KS + set + 1) * GA_STEP > full_end) {
      asm volatile("; tile with keys that some query does not see");   // no selects elsewhere
#pragma unroll
      for (int e = 0; e < 16; e++)
        if ((t * KS + set) * GA_STEP + 8 * (e >> 2) + 4 * half + (e & 3) >= seen) s[e] = -INFINITY;
    }
    if constexpr (AHEAD) scores(Const<(buf + 1) % BUFS>(), s_next, dp_next);
#pragma unroll
    for (int e = 0; e < 16; e++) s[e] = __builtin_amdgcn_exp2f(fmaf(s[e], sc, start));
    const bf16* tk = sK[buf];
    if constexpr (FINE) {
      if (from_out) {
#pragma unroll
        for (int e = 0; e < 16; e++) {
          left = fmaf(s[e], dp[e] - d, left);
          z += s[e];
        }
#pragma unroll
        for (int mm = 0; mm < 2; mm++) {
          const bf16x8 pf = att_pack(s, mm);
#pragma unroll
          for (int dt = 0; dt < D / 32; dt++)
            gp[dt] = mfma32(ga_trfrag<GA_STEP>(tk, 16 * mm, 32 * dt, lane), pf, gp[dt]);
        }
      }
    }
#pragma unroll
    for (int e = 0; e < 16; e++) s[e] *= dp[e] - d;
#pragma unroll
    for (int mm = 0; mm < 2; mm++) {
      const bf16x8 sf = att_pack(s, mm);
#pragma unroll
      for (int dt = 0; dt < D / 32; dt++)
        gq[dt] = mfma32(ga_trfrag<GA_STEP>(tk, 16 * mm, 32 * dt, lane), sf, gq[dt]);
    }
    if constexpr (FINE) {
#pragma unroll
      for (int mm = 0; mm < 2; mm++) {
        const bf16x8 sf = ga_rest(s, mm);
#pragma unroll
        for (int dt = 0; dt < D / 32; dt++)
          gq[dt] = mfma32(ga_trfrag<GA_STEP>(tk, 16 * mm, 32 * dt, lane), sf, gq[dt]);
      }
    }
  };
  if (turns) {
    f32x16 s, dp, s2, dp2;
    if constexpr (AHEAD) scores(Const<0>(), s, dp);
    for (int t = 0; t < turns; t += BUFS) {
      turn(Const<0>(), t, s, dp, s2, dp2);
      if (t + 1 < turns) turn(Const<1>(), t + 1, s2, dp2, s, dp);
      if constexpr (BUFS == 4) {
        if (t + 2 < turns) turn(Const<2>(), t + 2, s, dp, s2, dp2);
        if (t + 3 < turns) turn(Const<3>(), t + 3, s2, dp2, s, dp);
      }
    }
  }
  if constexpr (FINE) {
    if (from_out) {
      const float2 lz = joined(left, z);
      const float more = seen > SHORT && lz.y > 0.f ? lz.x / lz.y : 0.f;
#pragma unroll
      for (int dt = 0; dt < D / 32; dt++)
#pragma unroll
        for (int e = 0; e < 16; e++) gq[dt][e] -= more * gp[dt][e];
      if (q0 < a.n_q && !set && half) a.stats[ga_stats(it.b * a.q_heads + it.h, a.n_q, q0) + lane] = -(d + more);
    }
  }
  if constexpr (KS > 1) {                 // as in the forward
    constexpr int QUADS = D / 8 * 64;
    static_assert(sizeof(sKV) >= (KS - 1) * W * QUADS * sizeof(f32x4), "");
    f32x4* to = (f32x4*)sKV + wave * QUADS + lane;
    __syncthreads();
    if (set)
#pragma unroll
      for (int dt = 0; dt < D / 32; dt++)
#pragma unroll
        for (int g = 0; g < 4; g++)
          to[(set - 1) * W * QUADS + (4 * dt + g) * 64] =
              f32x4{gq[dt][4 * g], gq[dt][4 * g + 1], gq[dt][4 * g + 2], gq[dt][4 * g + 3]};
    __syncthreads();
    if (set) return;
    for (int other = 1; other < KS; other++, to += W * QUADS)
#pragma unroll
      for (int dt = 0; dt < D / 32; dt++)
#pragma unroll
        for (int g = 0; g < 4; g++) {
          const f32x4 v = to[(4 * dt + g) * 64];
#pragma unroll
          for (int r = 0; r < 4; r++) gq[dt][4 * g + r] += v[r];
        }
  }
  if (q0 >= a.n_q) return;
  bf16* dqb = a.dq + ((size_t)it.b * a.n_q + q0) * a.dq_stride + (size_t)it.h * D;
#pragma unroll
  for (int dt = 0; dt < D / 32; dt++)
    att_store(dqb + 32 * dt, a.dq_stride, gq[dt], a.scale, lane, a.n_q - q0);
}

// dK and dV of 128 keys of one key/value head, S and dP with lanes = keys, over
// the query tiles that see them of the group's heads one after the other.  Where
// the key tiles are too few for the chip, a.parts blocks share that sequence of
// query tiles and leave fp32 sums, which ga_join_kernel adds in order.
//
// A lane's 16 rows have statistics of their own, read from LDS: S and dP start from
// them instead of 0, which saves the vector unit its subtractions (8 x 4096, 16
// heads of 64 over 4: 980 us for the whole backward, 1008 without).
//
// Head dimension 64: a wave makes all four products of its 32 keys.  W and KS as in
// the forward: where the blocks are few, two waves of keys by four or two sets that
// share the query tiles (8 x 1024, 16 heads over 4: 108 us for the whole backward
// with four by two, 94 with two by four; 1 x 256, 8 heads 20.4, 19.3).
template <int W, int KS, bool FINE = false>
__global__ __launch_bounds__(64 * W * KS, 2) void ga_bwd_kv_kernel(GroupedArgs a) {
  constexpr int D = 64, ROWS = 32 * W;
  __shared__ __attribute__((aligned(1024))) bf16 sQO[KS][2][GA_BUFS][GA_STEP * D];   // queries, dout
  // a tile's statistics, four times over: every wave copies them, to keep one
  // count of loads on their way, and 64 lanes copy 1 KB
  __shared__ __attribute__((aligned(1024))) float sST[KS][GA_BUFS][256];
  Item it;
  const int key_tiles = (a.n_k + ROWS - 1) / ROWS;
  if (!ga_item(a.batch, a.kv_heads, key_tiles * a.parts, false, &it)) return;
  const int part = it.tile % a.parts;
  it.tile /= a.parts;
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const int wave = wave_index<W * KS>() % W, set = wave_index<W * KS>() / W;
  bf16(*sQ)[GA_STEP * D] = sQO[set][0];
  bf16(*sO)[GA_STEP * D] = sQO[set][1];
  float(*sS)[256] = sST[set];
  const int len = ga_length(a, it.b), off = a.n_k - a.n_q;
  const int blk0 = it.tile * ROWS, j0 = blk0 + 32 * wave, j = j0 + (lane & 31);
  const size_t os = (size_t)a.q_heads * D;
  bf16x8 kf[D / 16], vf[D / 16];
  ga_rows<D>(kf, a.k + (size_t)it.b * a.n_k * a.k_stride + (size_t)it.h * D, a.k_stride, j0, len, lane);
  ga_rows<D>(vf, a.v + (size_t)it.b * a.n_k * a.v_stride + (size_t)it.h * D, a.v_stride, j0, len, lane);
  f32x16 dk[D / 32] = {}, dv[D / 32] = {};
  const float sc = a.scale * GA_LOG2E;
  // the query tiles that see any of the block's keys: `per` of each head from
  // `first` on; this block's are steps lo .. hi - 1 of them all, this set's every
  // KS-th of those
  const int first = a.causal && blk0 - off > 0 ? (blk0 - off) / GA_STEP : 0;
  const int per = blk0 < len ? max(0, (a.n_q + GA_STEP - 1) / GA_STEP - first) : 0;
  const int lo = (int)((int64_t)per * a.group * part / a.parts);
  const int hi = (int)((int64_t)per * a.group * (part + 1) / a.parts);
  const int turns = (hi - lo + KS - 1) / KS, steps = (hi - lo - set + KS - 1) / KS;
  const TileDma<D, GA_STEP, W> dq(wave, lane, a.q_stride), dout(wave, lane, os);
  int lg = per ? (lo + set) / per : 0, lt = lo + set - lg * per;   // head and tile to be loaded next
  int ct = lt;                                                     // tile to be computed next
  auto load = [&](auto buf, int step) {                   // buf: step % GA_BUFS
    if (step >= steps) return;
    const int h = it.h * a.group + lg, i0 = (first + lt) * GA_STEP;
    dq.load(a.q + (size_t)it.b * a.n_q * a.q_stride + (size_t)h * D, a.q_stride, i0, a.n_q, sQ[buf]);
    dout.load(a.dout + (size_t)it.b * a.n_q * os + (size_t)h * D, os, i0, a.n_q, sO[buf]);
    dma16_at((const bf16*)(a.stats + ga_stats(it.b * a.q_heads + h, a.n_q, i0)), 16 * (lane & 15),
             (bf16*)sS[buf]);
#pragma unroll
    for (int i = 0; i < KS; i++)
      if (++lt == per) {
        lt = 0;
        lg++;
      }
  };
  auto scores = [&](auto buf, f32x16& s, f32x16& dp) {
    const bf16 *tq = sQ[buf], *to = sO[buf];
    // register e: query 8 (e / 4) + 4 half + e % 4 of the tile, key j
#pragma unroll
    for (int g = 0; g < 4; g++) {
      const f32x4 l4 = *(const f32x4*)(sS[buf] + 8 * g + 4 * half);
      const f32x4 d4 = *(const f32x4*)(sS[buf] + 32 + 8 * g + 4 * half);
#pragma unroll
      for (int r = 0; r < 4; r++) {
        s[4 * g + r] = l4[r];
        dp[4 * g + r] = d4[r];
      }
    }
#pragma unroll
    for (int ks = 0; ks < D / 16; ks++) {
      s = mfma32(ga_frag<GA_STEP>(tq, 0, 16 * ks, lane), kf[ks], s);
      dp = mfma32(ga_frag<GA_STEP>(to, 0, 16 * ks, lane), vf[ks], dp);
    }
  };
  auto turn = [&](auto buf, int step, f32x16& s, f32x16& dp, f32x16& s_next, f32x16& dp_next) {
    if (step + 2 < steps) wait_vmcnt<2 * TileDma<D, GA_STEP, W>::PER + 1>();
    else wait_vmcnt<0>();
    __syncthreads();
    load(Const<(buf + 3) % GA_BUFS>(), step + 3);
    const int r0 = (first + ct) * GA_STEP;
#pragma unroll
    for (int i = 0; i < KS; i++)
      if (++ct == per) ct = 0;
    if (KS > 1 && step >= steps) return;           // wave-uniform
    if (j0 + 32 > len || (a.causal && r0 + off < j0 + 31)) {
      asm volatile("; tile with keys that some query does not see");
      const int from = j >= len ? 1 << 30 : a.causal ? j - off - r0 : -1;   // first row that sees j
#pragma unroll
      for (int e = 0; e < 16; e++)
        if (8 * (e >> 2) + 4 * half + (e & 3) < from) s[e] = -INFINITY;
    }
    scores(Const<(buf + 1) % GA_BUFS>(), s_next, dp_next);
#pragma unroll
    for (int e = 0; e < 16; e++) {
      s[e] = __builtin_amdgcn_exp2f(s[e] * sc);
      dp[e] *= s[e];
    }
    const bf16 *tq = sQ[buf], *to = sO[buf];
#pragma unroll
    for (int mm = 0; mm < 2; mm++) {
      const bf16x8 pf = att_pack(s, mm), sf = att_pack(dp, mm);
#pragma unroll
      for (int d = 0; d < D / 32; d++) {
        dv[d] = mfma32(ga_trfrag<GA_STEP>(to, 16 * mm, 32 * d, lane), pf, dv[d]);
        dk[d] = mfma32(ga_trfrag<GA_STEP>(tq, 16 * mm, 32 * d, lane), sf, dk[d]);
      }
    }
    if constexpr (FINE) {
#pragma unroll
      for (int mm = 0; mm < 2; mm++) {
        const bf16x8 pf = ga_rest(s, mm), sf = ga_rest(dp, mm);
#pragma unroll
        for (int d = 0; d < D / 32; d++) {
          dv[d] = mfma32(ga_trfrag<GA_STEP>(to, 16 * mm, 32 * d, lane), pf, dv[d]);
          dk[d] = mfma32(ga_trfrag<GA_STEP>(tq, 16 * mm, 32 * d, lane), sf, dk[d]);
        }
      }
    }
  };
  if (turns > 0) {
    f32x16 s, dp, s2, dp2;
    load(Const<0>(), 0);
    load(Const<1>(), 1);
    load(Const<2>(), 2);
    wait_vmcnt<0>();
    __syncthreads();
    scores(Const<0>(), s, dp);
    for (int t = 0; t < turns; t += 4) {
      turn(Const<0>(), t, s, dp, s2, dp2);
      if (t + 1 < turns) turn(Const<1>(), t + 1, s2, dp2, s, dp);
      if (t + 2 < turns) turn(Const<2>(), t + 2, s, dp, s2, dp2);
      if (t + 3 < turns) turn(Const<3>(), t + 3, s2, dp2, s, dp);
    }
  }
  if constexpr (KS > 1) {                // as in the forward
    constexpr int QUADS = D / 4 * 64;
    static_assert(sizeof(sQO) >= (KS - 1) * W * QUADS * sizeof(f32x4), "");
    f32x4* to = (f32x4*)sQO + wave * QUADS + lane;
    __syncthreads();
    if (set) {
      f32x4* mine = to + (set - 1) * W * QUADS;
#pragma unroll
      for (int d = 0; d < D / 32; d++)
#pragma unroll
        for (int g = 0; g < 4; g++) {
          mine[(8 * d + g) * 64] = f32x4{dk[d][4 * g], dk[d][4 * g + 1], dk[d][4 * g + 2], dk[d][4 * g + 3]};
          mine[(8 * d + 4 + g) * 64] = f32x4{dv[d][4 * g], dv[d][4 * g + 1], dv[d][4 * g + 2], dv[d][4 * g + 3]};
        }
    }
    __syncthreads();
    if (set) return;
    for (int other = 1; other < KS; other++, to += W * QUADS)
#pragma unroll
      for (int d = 0; d < D / 32; d++)
#pragma unroll
        for (int g = 0; g < 4; g++) {
          const f32x4 x = to[(8 * d + g) * 64], y = to[(8 * d + 4 + g) * 64];
#pragma unroll
          for (int r = 0; r < 4; r++) {
            dk[d][4 * g + r] += x[r];
            dv[d][4 * g + r] += y[r];
          }
        }
  }
  if (j0 >= a.n_k) return;
  if (a.parts > 1) {
    // [part][dk, dv][sequence][key][head][D]
    const size_t rows = (size_t)a.batch * a.n_k * a.kv_heads * D;
    float* p = a.partial + 2 * part * rows + (((size_t)it.b * a.n_k + j) * a.kv_heads + it.h) * D + 4 * half;
    if (j < a.n_k)
#pragma unroll
      for (int d = 0; d < D / 32; d++)
#pragma unroll
        for (int g = 0; g < 4; g++) {
          *(f32x4*)(p + 32 * d + 8 * g) = f32x4{dk[d][4 * g], dk[d][4 * g + 1], dk[d][4 * g + 2], dk[d][4 * g + 3]};
          *(f32x4*)(p + rows + 32 * d + 8 * g) = f32x4{dv[d][4 * g], dv[d][4 * g + 1], dv[d][4 * g + 2], dv[d][4 * g + 3]};
        }
    return;
  }
  bf16* dkb = a.dk + ((size_t)it.b * a.n_k + j0) * a.dk_stride + (size_t)it.h * D;
  bf16* dvb = a.dv + ((size_t)it.b * a.n_k + j0) * a.dv_stride + (size_t)it.h * D;
#pragma unroll
  for (int d = 0; d < D / 32; d++) {
    att_store(dkb + 32 * d, a.dk_stride, dk[d], a.scale, lane, a.n_k - j0);
    att_store(dvb + 32 * d, a.dv_stride, dv[d], 1.f, lane, a.n_k - j0);
  }
}

// Head dimension 128: all four products of 32 keys take more than half of a SIMD's
// registers, and a wave that is alone there waits for itself.  So two waves of one
// SIMD share them: the first makes S, P and dV, the second dP, dS and dK a turn
// later, from the P in fp32 that the first leaves in LDS.  (8 x 4096, 8 heads over
// 2: the backward 970 us with a wave for all four, 909 so, 925 without the hint on
// order; 32 x 512: 122, 113; by head dimension 64 952 and 1064: there the exchange
// costs more LDS than it hides.)
//
// The last turn's tiles, this one's and the next are in use, the fourth buffer's are
// on their way.  A buffer is an LDS variable of its own, so that the compiler sees
// that no read of the turn waits for them (in one variable 8 x 4096 took 937 us on a
// card where it is 924, 3 x 1000 70.2 and 68.0).
template <bool FINE>
__global__ __launch_bounds__(512, 2) void ga_bwd_pair_kernel(GroupedArgs a) {
  constexpr int D = 128;
  struct Tiles {
    bf16 rows[2][GA_STEP * D];                 // queries, dout
    float stats[256];
  };
  __shared__ __attribute__((aligned(1024))) Tiles t0, t1, t2, t3;
  __shared__ __attribute__((aligned(1024))) f32x4 sP[2][4][4][64];              // [turn % 2][wave][quad][lane]
  Item it;
  const int key_tiles = (a.n_k + GA_ROWS - 1) / GA_ROWS;
  if (!ga_item(a.batch, a.kv_heads, key_tiles * a.parts, false, &it)) return;
  const int part = it.tile % a.parts;
  it.tile /= a.parts;
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const int wave = wave_index<8>() & 3, role = wave_index<8>() >> 2;
  const int len = ga_length(a, it.b), off = a.n_k - a.n_q;
  const int blk0 = it.tile * GA_ROWS, j0 = blk0 + 32 * wave, j = j0 + (lane & 31);
  const size_t os = (size_t)a.q_heads * D;
  bf16x8 xf[D / 16];
  if (role == 0)
    ga_rows<D>(xf, a.k + (size_t)it.b * a.n_k * a.k_stride + (size_t)it.h * D, a.k_stride, j0, len, lane);
  else
    ga_rows<D>(xf, a.v + (size_t)it.b * a.n_k * a.v_stride + (size_t)it.h * D, a.v_stride, j0, len, lane);
  f32x16 acc[D / 32] = {};
  const float sc = a.scale * GA_LOG2E;
  const int first = a.causal && blk0 - off > 0 ? (blk0 - off) / GA_STEP : 0;
  const int per = blk0 < len ? max(0, (a.n_q + GA_STEP - 1) / GA_STEP - first) : 0;
  const int lo = (int)((int64_t)per * a.group * part / a.parts);
  const int hi = (int)((int64_t)per * a.group * (part + 1) / a.parts);
  const int steps = hi - lo;
  const int64_t stride = role ? (int64_t)os : a.q_stride;
  const bf16* src = role ? a.dout + (size_t)it.b * a.n_q * os : a.q + (size_t)it.b * a.n_q * a.q_stride;
  const TileDma<D, GA_STEP> dma(wave, lane, stride);
  int lg = per ? lo / per : 0, lt = lo - lg * per;       // head and tile to be loaded next
  int ct = lt;                                           // tile to be computed next
  auto tiles = [&](auto buf) -> Tiles& {
    if constexpr (buf == 0) return t0;
    else if constexpr (buf == 1) return t1;
    else if constexpr (buf == 2) return t2;
    else return t3;
  };
  auto load = [&](auto buf, int step) {                  // buf: step % GA_BUFS
    if (step >= steps) return;
    const int h = it.h * a.group + lg, i0 = (first + lt) * GA_STEP;
    dma.load(src + (size_t)h * D, stride, i0, a.n_q, tiles(buf).rows[role]);
    if (wave == 0 && role == 0)
      dma16_at((const bf16*)(a.stats + ga_stats(it.b * a.q_heads + h, a.n_q, i0)), 16 * (lane & 15),
               (bf16*)tiles(buf).stats);
    if (++lt == per) {
      lt = 0;
      lg++;
    }
  };
  auto product = [&](auto buf, f32x16& x) {              // S or dP
#pragma unroll
    for (int g = 0; g < 4; g++) {
      const f32x4 y = *(const f32x4*)(tiles(buf).stats + 32 * role + 8 * g + 4 * half);
#pragma unroll
      for (int r = 0; r < 4; r++) x[4 * g + r] = y[r];
    }
#pragma unroll
    for (int ks = 0; ks < D / 16; ks++) x = mfma32(ga_frag<GA_STEP>(tiles(buf).rows[role], 0, 16 * ks, lane), xf[ks], x);
  };
  auto gather = [&](auto buf, const f32x16& x) {         // dV or dK
#pragma unroll
    for (int mm = 0; mm < 2; mm++) {
      const bf16x8 f = att_pack(x, mm), rest = FINE ? ga_rest(x, mm) : f;
#pragma unroll
      for (int d = 0; d < D / 32; d++) {
        const bf16x8 t = ga_trfrag<GA_STEP>(tiles(buf).rows[role ^ 1], 16 * mm, 32 * d, lane);
        acc[d] = mfma32(t, f, acc[d]);
        if constexpr (FINE) acc[d] = mfma32(t, rest, acc[d]);
      }
    }
  };
  auto meet = [&](auto buf, int t) {
    ga_meet<0>();
    load(Const<(buf + 2) % GA_BUFS>(), t + 2);
  };
  auto turn_s = [&](auto buf, int t, f32x16& s, f32x16& next) {
    meet(buf, t);
    if (t >= steps) return;
    const int r0 = (first + ct) * GA_STEP;
    if (++ct == per) ct = 0;
    if (j0 + 32 > len || (a.causal && r0 + off < j0 + 31)) {
      asm volatile("; tile with keys that some query does not see");
      const int from = j >= len ? 1 << 30 : a.causal ? j - off - r0 : -1;
#pragma unroll
      for (int e = 0; e < 16; e++)
        if (8 * (e >> 2) + 4 * half + (e & 3) < from) s[e] = -INFINITY;
    }
    product(Const<(buf + 1) % GA_BUFS>(), next);
#pragma unroll
    for (int e = 0; e < 16; e++) s[e] = __builtin_amdgcn_exp2f(s[e] * sc);
#pragma unroll
    for (int g = 0; g < 4; g++) sP[buf & 1][wave][g][lane] = f32x4{s[4 * g], s[4 * g + 1], s[4 * g + 2], s[4 * g + 3]};
    gather(buf, s);
    __builtin_amdgcn_iglp_opt(0);          // the compiler's order for matrix products fed from LDS
  };
  auto turn_d = [&](auto buf, int t, f32x16& dp, f32x16& last) {
    meet(buf, t);
    product(buf, dp);
    if (t == 0) return;
#pragma unroll
    for (int g = 0; g < 4; g++) {
      const f32x4 p = sP[(buf + 1) & 1][wave][g][lane];
#pragma unroll
      for (int r = 0; r < 4; r++) last[4 * g + r] *= p[r];
    }
    gather(Const<(buf + 3) % GA_BUFS>(), last);
    __builtin_amdgcn_iglp_opt(0);
  };
  if (steps > 0) {
    load(Const<0>(), 0);
    load(Const<1>(), 1);
    ga_meet<0>();
    f32x16 x, y;
    if (role == 0) {
      product(Const<0>(), x);
      for (int t = 0; t <= steps; t += 4) {
        turn_s(Const<0>(), t, x, y);
        if (t + 1 <= steps) turn_s(Const<1>(), t + 1, y, x);
        if (t + 2 <= steps) turn_s(Const<2>(), t + 2, x, y);
        if (t + 3 <= steps) turn_s(Const<3>(), t + 3, y, x);
      }
    } else {
      for (int t = 0; t <= steps; t += 4) {
        turn_d(Const<0>(), t, x, y);
        if (t + 1 <= steps) turn_d(Const<1>(), t + 1, y, x);
        if (t + 2 <= steps) turn_d(Const<2>(), t + 2, x, y);
        if (t + 3 <= steps) turn_d(Const<3>(), t + 3, y, x);
      }
    }
  }
  if (j0 >= a.n_k) return;
  if (a.parts > 1) {
    const size_t rows = (size_t)a.batch * a.n_k * a.kv_heads * D;
    float* p = a.partial + (2 * part + (role == 0)) * rows + (((size_t)it.b * a.n_k + j) * a.kv_heads + it.h) * D + 4 * half;
    if (j < a.n_k)
#pragma unroll
      for (int d = 0; d < D / 32; d++)
#pragma unroll
        for (int g = 0; g < 4; g++)
          *(f32x4*)(p + 32 * d + 8 * g) = f32x4{acc[d][4 * g], acc[d][4 * g + 1], acc[d][4 * g + 2], acc[d][4 * g + 3]};
    return;
  }
  const int64_t ostride = role ? a.dk_stride : a.dv_stride;
  bf16* ob = (role ? a.dk : a.dv) + ((size_t)it.b * a.n_k + j0) * ostride + (size_t)it.h * D;
#pragma unroll
  for (int d = 0; d < D / 32; d++) att_store(ob + 32 * d, ostride, acc[d], role ? a.scale : 1.f, lane, a.n_k - j0);
}

// Adds the parts of dK (blockIdx.y 0) or dV, eight columns to a thread.
__global__ __launch_bounds__(GA_THREADS) void ga_join_kernel(GroupedArgs a) {
  const int width = a.kv_heads * a.head_dim;
  const size_t i = ((size_t)blockIdx.x * GA_THREADS + threadIdx.x) * 8;
  const size_t rows = (size_t)a.batch * a.n_k * width;
  if (i >= rows) return;
  const float* p = a.partial + blockIdx.y * rows + i;
  f32x4 x = {}, y = {};
  for (int part = 0; part < a.parts; part++, p += 2 * rows) {
    x += *(const f32x4*)p;
    y += *(const f32x4*)(p + 4);
  }
  const float scale = blockIdx.y ? 1.f : a.scale;
  bf16x8 v;
#pragma unroll
  for (int e = 0; e < 4; e++) {
    v[e] = to_bf16(x[e] * scale);
    v[4 + e] = to_bf16(y[e] * scale);
  }
  const size_t row = i / width, col = i - row * width;
  *(bf16x8*)((blockIdx.y ? a.dv + row * a.dv_stride : a.dk + row * a.dk_stride) + col) = v;
}

// Sequences [b0, b0 + nb) of a call.
GroupedArgs ga_slice(const GroupedArgs& a, int64_t b0, int64_t nb) {
  GroupedArgs s = a;
  const size_t qo = (size_t)b0 * a.n_q, ko = (size_t)b0 * a.n_k, hd = (size_t)a.q_heads * a.head_dim;
  s.batch = (int)nb;
  s.q += qo * a.q_stride;
  s.k += ko * a.k_stride;
  s.v += ko * a.v_stride;
  s.out += qo * hd;
  s.lse += qo * a.q_heads;
  if (a.lengths) s.lengths += b0;
  if (a.dout) {
    s.dout += qo * hd;
    s.dq += qo * a.dq_stride;
    s.dk += ko * a.dk_stride;
    s.dv += ko * a.dv_stride;
    s.stats += (size_t)b0 * a.q_heads * ((a.n_q + 31) / 32) * 64;
  }
  return s;
}

constexpr int64_t GA_MAX_BLOCKS = 1 << 22;     // of a launch, up to 512 threads each: below 2^32

// Whether the scores of a call are so few that their roundings do not average
// (ga_rest), for all of its kernels alike.  Such calls are given the form for few blocks,
// up to so many blocks of 128 queries: it costs 100 x 8 positions, 2 heads of 64 3.8 + 9.2
// us, 5.2 + 11.1 so, but 512 x 4 5.6 + 15.4, 10.4 + 31.1, and so many sequences' roundings
// nearly average.
constexpr int64_t GA_FINE_BLOCKS = 256;
int64_t ga_tiles(int n) { return (n + GA_ROWS - 1) / GA_ROWS; }
int64_t ga_halves(int n) { return (n + GA_ROWS / 2 - 1) / (GA_ROWS / 2); }
bool ga_fine(const GroupedArgs& a) {
  const int64_t heads = (int64_t)a.batch * a.q_heads;
  return heads * a.n_q <= (1 << 16) / a.n_k && heads * ga_tiles(a.n_q) <= GA_FINE_BLOCKS;
}

// Whether blocks of 128 queries are so few that a CU is better given blocks of 64
// by several sets: where they fill half of the chip, up to all of it where a causal
// mask leaves the longest rows to a few, and up to two rounds where a block's few
// rows leave half of its waves idle over a long way of keys.  us of forward and
// backward with blocks of 128, and so, 8 heads over 2: 1 x 2048 of 64 27.7 + 68.6,
// 17.2 + 52.5; 2 x 2048 of 128 40.0 + 127, 30.4 + 121; 64 x 64 queries of 2000 keys of
// 64 39.9 + 101, 26.8 + 97.8; 44 x 6 of 2928, 3 heads 52.2 + 91.3, 24.3 + 62.3; but
// 16 x 256 of 64 7.8 + 28.5, 9.3 + 34.0; 4 x 1000 of 128 without mask 23.3 + 85.7,
// 24.0 + 96.3; 256 x 1 of 1000 42.6 + 116, 44.6 + 151; 35 x 3 of 237 of 128, 8 over 4
// 9.5 + 28.3, 7.8 + 34.6.
bool ga_few(const GroupedArgs& a, int64_t blocks) {
  return ga_fine(a) || blocks <= (a.causal && a.n_q >= 768 ? 256 : a.n_q <= 64 && a.n_k >= 1024 ? 512 : 128);
}
// As many sets as the tiles leave LDS for, two blocks to a CU with head dimension 128.
constexpr int ga_sets(int D) { return D == 64 ? 4 : 2; }

template <int D>
hipError_t ga_forward(const GroupedArgs& a, hipStream_t st) {
  const int64_t per = ga_tiles(a.n_q) * a.q_heads;
  const int64_t most = GA_MAX_BLOCKS / per > 0 ? GA_MAX_BLOCKS / per : 1;
  for (int64_t b0 = 0; b0 < a.batch; b0 += most) {
    const int64_t nb = a.batch - b0 < most ? a.batch - b0 : most;
    const int halves = (int)(nb * ga_halves(a.n_q) * a.q_heads), few = 128 * ga_sets(D);
    const GroupedArgs s = ga_slice(a, b0, nb);
    if (!ga_few(a, nb * per))
      ga_fwd_kernel<D, 4, 1><<<(int)(nb * per), 256, 0, st>>>(s);
    else if (ga_fine(a))
      ga_fwd_kernel<D, 2, ga_sets(D), true><<<halves, few, 0, st>>>(s);
    else
      ga_fwd_kernel<D, 2, ga_sets(D)><<<halves, few, 0, st>>>(s);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// Blocks that share a key tile where the tiles are fewer than the CUs.  Every part
// adds fp32 sums to write and to join, so it has to be worth its steps (query tiles
// of 32, of all the group's heads).
//
// Head dimension 64: a block of eight waves to each CU if a part keeps 16 steps,
// two to each, which evens out what a causal mask makes uneven, if it keeps 64.  us
// of the backward with 512 blocks of four waves, and so, 8 heads over 2: 4 x 500
// 36.5, 28.8; 1 x 1000 42.4, 32.6; 16 x 512 46.4, 40.0; 16 over 4: 4 x 1024 65.4,
// 63.0; 1 x 4096 186, 171 (one block to each CU 214).
// Head dimension 128: one block to each CU, 8 steps (5 x 333 x 777, 8 over 2: 51.9,
// with 16 56.6; 1 x 1000 47.8, 53.0).
int ga_parts(int64_t batch, int64_t n_q, int64_t n_k, int q_heads, int kv_heads, int head_dim) {
  const int64_t blocks = batch * kv_heads * ga_tiles((int)n_k);
  const int64_t steps = (n_q + GA_STEP - 1) / GA_STEP * (q_heads / kv_heads);
  const int64_t p = head_dim == 64 ? std::max(std::min(128 / blocks, steps / 16), std::min(256 / blocks, steps / 64))
                                   : std::min(256 / blocks, steps / 8);
  return p < 1 ? 1 : p > 32 ? 32 : (int)p;
}

size_t ga_stats_bytes(int64_t batch, int64_t n_q, int q_heads) {
  return (size_t)batch * q_heads * ((n_q + 31) / 32) * 64 * sizeof(float);
}

template <int D>
hipError_t ga_backward(const GroupedArgs& a, hipStream_t st) {
  const int64_t kv = ga_tiles(a.n_k) * a.kv_heads * a.parts, q = ga_tiles(a.n_q) * a.q_heads;
  const int64_t per = std::max(kv, q);
  // (every slice's sums lie at the workspace's start, in its own extents)
  const int64_t most = GA_MAX_BLOCKS / per > 0 ? GA_MAX_BLOCKS / per : 1;
  for (int64_t b0 = 0; b0 < a.batch; b0 += most) {
    const int64_t nb = a.batch - b0 < most ? a.batch - b0 : most;
    const GroupedArgs s = ga_slice(a, b0, nb);
    const int q_halves = (int)(nb * ga_halves(a.n_q) * a.q_heads), few = 128 * ga_sets(D);
    const bool fine = ga_fine(a);
    if (!ga_few(a, nb * q))
      ga_bwd_q_kernel<D, 4, 1><<<(int)(nb * q), 256, 0, st>>>(s);
    else if (fine)
      ga_bwd_q_kernel<D, 2, ga_sets(D), true><<<q_halves, few, 0, st>>>(s);
    else
      ga_bwd_q_kernel<D, 2, ga_sets(D)><<<q_halves, few, 0, st>>>(s);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if constexpr (D == 64) {
      // No more blocks of 128 keys than CUs: 64 by four sets (16 x 700, 8 heads over 2,
      // no mask: 106 us with 4 by 1, 96), or by two where a block has few steps, so
      // that one's beginning and end run under another's turns (64 x 256: 50.2, 44.6
      // by two; 4 x 500: 28.0, 27.0; but 20 x 500, 64 steps: 43.5, 48.3).
      const int halves = (int)(nb * ga_halves(a.n_k) * a.kv_heads * a.parts);
      const int64_t steps = (int64_t)(a.n_q + GA_STEP - 1) / GA_STEP * a.group / a.parts;
      if (fine)
        ga_bwd_kv_kernel<2, 2, true><<<halves, 256, 0, st>>>(s);
      else if (nb * kv > 256)
        ga_bwd_kv_kernel<4, 1><<<(int)(nb * kv), 256, 0, st>>>(s);
      else if (steps <= 32)
        ga_bwd_kv_kernel<2, 2><<<halves, 256, 0, st>>>(s);
      else
        ga_bwd_kv_kernel<2, 4><<<halves, 512, 0, st>>>(s);
    } else {
      if (fine)
        ga_bwd_pair_kernel<true><<<(int)(nb * kv), 512, 0, st>>>(s);
      else
        ga_bwd_pair_kernel<false><<<(int)(nb * kv), 512, 0, st>>>(s);
    }
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (a.parts > 1) {
      const int64_t vecs = (int64_t)nb * a.n_k * a.kv_heads * (D / 8);
      ga_join_kernel<<<dim3((unsigned)((vecs + GA_THREADS - 1) / GA_THREADS), 2), GA_THREADS, 0, st>>>(s);
      e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
  }
  return hipSuccess;
}

}  // namespace

size_t grouped_workspace_bytes(int64_t batch, int64_t n_q, int64_t n_k, int32_t q_heads,
                               int32_t kv_heads, int32_t head_dim) {
  const int parts = ga_parts(batch, n_q, n_k, q_heads, kv_heads, head_dim);
  const size_t sums = parts > 1 ? (size_t)parts * 2 * batch * n_k * kv_heads * head_dim * sizeof(float) : 0;
  return (ga_stats_bytes(batch, n_q, q_heads) + sums + 255) / 256 * 256;
}

hipError_t launch_grouped_forward(const GroupedArgs& a, hipStream_t st) {
  return a.head_dim == 64 ? ga_forward<64>(a, st) : ga_forward<128>(a, st);
}

hipError_t launch_grouped_backward(GroupedArgs a, void* workspace, hipStream_t st) {
  a.parts = ga_parts(a.batch, a.n_q, a.n_k, a.q_heads, a.kv_heads, a.head_dim);
  a.stats = (float*)workspace;
  a.partial = a.stats + ga_stats_bytes(a.batch, a.n_q, a.q_heads) / sizeof(float);
  return a.head_dim == 64 ? ga_backward<64>(a, st) : ga_backward<128>(a, st);
}

}  // namespace hcmix
