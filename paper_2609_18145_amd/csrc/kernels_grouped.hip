// Softmax attention over windows of any length, forward and backward (bf16 in,
// fp32 accumulation, head dimension 64 or 128), key/value heads shared by
// groups of query heads, keys past a sequence's length and (causal) past the
// query's own position left out.
//
// The scores of 64 keys at a time never leave the registers: the forward keeps
// each query's running maximum m and sum l of exp(S - m) and rescales what it
// has accumulated when m grows.  The backward makes P = exp(S - lse) again from
// the forward's lse instead of reading it.
//
// Tiles, fragments and the transposed scores (a lane owns a query, or a key in
// the key/value gradients, and 16 rows of a 32 x 32 tile) are tile64.h's.
// A tile of 128 columns is two of 64.
#include "hcmix_internal.h"
#include "device_common.h"
#include "tile64.h"

#include <algorithm>

namespace hcmix {

namespace {

constexpr int GA_THREADS = 256;
constexpr float GA_LOG2E = 1.4426950408889634f, GA_LN2 = 0.6931471805599453f;
constexpr int GA_TILE = 64;         // rows of an LDS tile
// Rows of a block (32 to a wave).
constexpr int GA_ROWS = 128;

template <int D>
__device__ __forceinline__ bf16x8 ga_frag(const bf16* t, int r0, int c0, int lane) {
  return att_frag(t + (c0 >> 6) * GA_TILE * HD, r0, c0 & 63, lane);
}
template <int D>
__device__ __forceinline__ bf16x8 ga_trfrag(const bf16* t, int k0, int c0, int lane) {
  return att_trfrag(t + (c0 >> 6) * GA_TILE * HD, k0, c0 & 63, lane);
}

// A tile's way from global memory through registers into LDS: rows row0 .. + 64
// of an array with rows `stride` elements apart, of which those at `valid` and
// behind are zeros, whatever memory holds there.
template <int D>
struct TileLoad {
  static constexpr int PER = GA_TILE * D / 8 / GA_THREADS;   // 16-byte pieces per thread
  u32x4 v[PER];
  __device__ __forceinline__ void load(const bf16* base, size_t stride, int row0, int valid) {
#pragma unroll
    for (int j = 0; j < PER; j++) {
      const int pi = threadIdx.x + GA_THREADS * j, r = pi / (D / 8), p = pi % (D / 8);
      v[j] = u32x4{0, 0, 0, 0};
      if (row0 + r < valid) v[j] = *(const u32x4*)(base + (size_t)(row0 + r) * stride + 8 * p);
    }
  }
  __device__ __forceinline__ void store(bf16* tile) const {
#pragma unroll
    for (int j = 0; j < PER; j++) {
      const int pi = threadIdx.x + GA_THREADS * j, r = pi / (D / 8), p = pi % (D / 8);
      *(u32x4*)(tile + (p >> 3) * GA_TILE * HD + att_off(r, 8 * (p & 7))) = v[j];
    }
  }
};

// This block's (sequence, head, tile): the tiles of one head, and the heads of
// one group, are neighbours on one XCD, whose L2 then holds their keys and
// values; a head's tiles with the most work come first.
struct Item {
  int b, h, tile;
};
__device__ __forceinline__ bool ga_item(int heads, int tiles, int total, bool last_first, Item* it) {
  const int chunk = (total + 7) >> 3;
  const int i = (blockIdx.x & 7) * chunk + (blockIdx.x >> 3);
  if ((blockIdx.x >> 3) >= chunk || i >= total) return false;
  const int bh = i / tiles, t = i - bh * tiles;
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
template <int D>
__global__ __launch_bounds__(GA_THREADS, 2) void ga_fwd_kernel(GroupedArgs a, int total) {
  __shared__ __attribute__((aligned(1024))) bf16 sK[2][GA_TILE * D], sV[2][GA_TILE * D];
  Item it;
  if (!ga_item(a.q_heads, (a.n_q + GA_ROWS - 1) / GA_ROWS, total, a.causal, &it)) return;
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const int wave = wave_index<GA_THREADS / 64>();
  const int kvh = it.h / a.group, len = ga_length(a, it.b), off = a.n_k - a.n_q;
  const int blk0 = it.tile * GA_ROWS, q0 = blk0 + 32 * wave;
  const bf16* qb = a.q + (size_t)it.b * a.n_q * a.q_stride + (size_t)it.h * D;
  const bf16* kb = a.k + (size_t)it.b * a.n_k * a.k_stride + (size_t)kvh * D;
  const bf16* vb = a.v + (size_t)it.b * a.n_k * a.v_stride + (size_t)kvh * D;
  // keys that the block's last query, and this wave's, sees
  const int blk_end = a.causal ? min(len, blk0 + GA_ROWS + off) : len;
  const int wave_end = a.causal ? min(len, q0 + 32 + off) : len;
  const int full_end = a.causal ? min(len, q0 + 1 + off) : len;   // seen by all of its queries
  const int tiles = blk_end > 0 ? (blk_end + GA_TILE - 1) / GA_TILE : 0;
  bf16x8 qf[D / 16];
  ga_rows<D>(qf, qb, a.q_stride, q0, a.n_q, lane);
  f32x16 o[D / 32] = {};
  float m = -3e38f, l = 0.f;
  const float sc = a.scale * GA_LOG2E;
  TileLoad<D> lk, lv;
  if (tiles) {
    lk.load(kb, a.k_stride, 0, len);
    lv.load(vb, a.v_stride, 0, len);
    lk.store(sK[0]);
    lv.store(sV[0]);
  }
  for (int t = 0; t < tiles; t++) {
    __syncthreads();
    if (t + 1 < tiles) {
      lk.load(kb, a.k_stride, (t + 1) * GA_TILE, len);
      lv.load(vb, a.v_stride, (t + 1) * GA_TILE, len);
    }
    const bf16 *tk = sK[t & 1], *tv = sV[t & 1];
    const int k0 = t * GA_TILE;
    if (k0 < wave_end) {             // wave-uniform
      f32x16 s[2];
#pragma unroll
      for (int kt = 0; kt < 2; kt++) {
        s[kt] = f32x16{};
#pragma unroll
        for (int ks = 0; ks < D / 16; ks++)
          s[kt] = mfma32(ga_frag<D>(tk, 32 * kt, 16 * ks, lane), qf[ks], s[kt]);
      }
      if (k0 + GA_TILE > full_end) {
        // register e of a lane: key k0 + 32 kt + 8 (e / 4) + 4 half + e % 4
        const int end = a.causal ? min(len, q0 + (lane & 31) + 1 + off) : len;
#pragma unroll
        for (int kt = 0; kt < 2; kt++)
#pragma unroll
          for (int e = 0; e < 16; e++)
            if (k0 + 32 * kt + 8 * (e >> 2) + 4 * half + (e & 3) >= end) s[kt][e] = -INFINITY;
      }
      float mx = s[0][0];
#pragma unroll
      for (int kt = 0; kt < 2; kt++)
#pragma unroll
        for (int e = 0; e < 16; e++) mx = fmaxf(mx, s[kt][e]);
      mx = fmaxf(mx, __shfl_xor(mx, 32)) * sc;
      const float mn = fmaxf(m, mx), alpha = __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      l *= alpha;
#pragma unroll
      for (int d = 0; d < D / 32; d++)
#pragma unroll
        for (int e = 0; e < 16; e++) o[d][e] *= alpha;
#pragma unroll
      for (int kt = 0; kt < 2; kt++)
#pragma unroll
        for (int e = 0; e < 16; e++) {
          const float p = __builtin_amdgcn_exp2f(fmaf(s[kt][e], sc, -m));
          s[kt][e] = p;
          l += p;
        }
#pragma unroll
      for (int kt = 0; kt < 2; kt++)
#pragma unroll
        for (int mm = 0; mm < 2; mm++) {
          const bf16x8 pf = att_pack(s[kt], mm);
#pragma unroll
          for (int d = 0; d < D / 32; d++)
            o[d] = mfma32(ga_trfrag<D>(tv, 32 * kt + 16 * mm, 32 * d, lane), pf, o[d]);
        }
    }
    if (t + 1 < tiles) {
      lk.store(sK[(t + 1) & 1]);
      lv.store(sV[(t + 1) & 1]);
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
// Backward.  A row's D and its lse in log2 units go to the workspace first, rows
// padded to a multiple of 64: behind the last row, and for rows that see
// nothing, an lse of +inf, which makes their P = 0.
//
// D = sum_j P_j dP_j = dout . out.  The second form is one pass over two rows,
// but out is rounded to bf16, and dS = P (dP - D) cancels the more the fewer keys
// share a row: a row that sees one key has dS = 0, and got 2^-9 |dout| |out|
// instead (dq and dk of windows of 10 keys were 0.0046 off in all, 0.0024 so).
// So tiles whose rows see at most GA_EXACT_KEYS keys take the first form, P and
// dP made as in the kernels below; with more, the rounding of out adds less than
// a tenth to that of dS.
// ---------------------------------------------------------------------------
constexpr int GA_EXACT_KEYS = 128;

template <int D>
__global__ __launch_bounds__(GA_THREADS) void ga_row_sum_kernel(GroupedArgs a, int pad, int total) {
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const int item = blockIdx.x * (GA_THREADS / 64) + wave_index<GA_THREADS / 64>();
  if (item >= total) return;
  const int tiles = pad / 32, bh = item / tiles, q0 = (item - bh * tiles) * 32;
  const int b = bh / a.q_heads, h = bh - b * a.q_heads;
  const int len = ga_length(a, b), off = a.n_k - a.n_q;
  const int end = a.causal ? min(len, q0 + 32 + off) : len;
  const size_t os = (size_t)a.q_heads * D, row = (size_t)bh * pad + q0;
  const bf16* dob = a.dout + (size_t)b * a.n_q * os + (size_t)h * D;
  const float* lse = a.lse + (size_t)bh * a.n_q;
  float l = INFINITY;              // of row lane % 32
  if (q0 + (lane & 31) < a.n_q) {
    l = lse[q0 + (lane & 31)];
    l = l == -INFINITY ? INFINITY : l * GA_LOG2E;
  }
  if (half == 0) a.row_lse[row + lane] = l;
  if (end <= GA_EXACT_KEYS) {      // wave-uniform
    const bf16* kb = a.k + (size_t)b * a.n_k * a.k_stride + (size_t)(h / a.group) * D;
    const bf16* vb = a.v + (size_t)b * a.n_k * a.v_stride + (size_t)(h / a.group) * D;
    bf16x8 qf[D / 16], of[D / 16];
    ga_rows<D>(qf, a.q + (size_t)b * a.n_q * a.q_stride + (size_t)h * D, a.q_stride, q0, a.n_q, lane);
    ga_rows<D>(of, dob, os, q0, a.n_q, lane);
    const int seen = a.causal ? min(len, q0 + (lane & 31) + 1 + off) : len;
    float d = 0.f;
    for (int k0 = 0; k0 < end; k0 += 32) {
      bf16x8 kf[D / 16], vf[D / 16];
      ga_rows<D>(kf, kb, a.k_stride, k0, len, lane);
      ga_rows<D>(vf, vb, a.v_stride, k0, len, lane);
      f32x16 s = {}, dp = {};
#pragma unroll
      for (int ks = 0; ks < D / 16; ks++) {
        s = mfma32(kf[ks], qf[ks], s);
        dp = mfma32(vf[ks], of[ks], dp);
      }
#pragma unroll
      for (int e = 0; e < 16; e++) {
        const float p = __builtin_amdgcn_exp2f(fmaf(s[e], a.scale * GA_LOG2E, -l));
        d += k0 + 8 * (e >> 2) + 4 * half + (e & 3) < seen ? p * dp[e] : 0.f;
      }
    }
    d += __shfl_xor(d, 32);
    if (half == 0) a.row_sum[row + lane] = d;
    return;
  }
  constexpr int PER = D / 8, RW = 64 / PER;      // lanes of a row, rows at a time
  const int piece = lane % PER;
#pragma unroll
  for (int r0 = 0; r0 < 32; r0 += RW) {
    const int r = r0 + lane / PER;
    float d = 0.f;
    if (q0 + r < a.n_q) {
      const bf16x8 y = *(const bf16x8*)(dob + (size_t)(q0 + r) * os + 8 * piece);
      const bf16x8 x = *(const bf16x8*)(a.out + ((size_t)b * a.n_q + q0 + r) * os + (size_t)h * D + 8 * piece);
#pragma unroll
      for (int e = 0; e < 8; e++) d += (float)x[e] * (float)y[e];
    }
#pragma unroll
    for (int s = 1; s < PER; s *= 2) d += __shfl_xor(d, s);
    if (piece == 0) a.row_sum[row + r] = d;
  }
}

// dK and dV of 128 keys of one key/value head: over the group's query heads and
// the query tiles that see them, S and dP with lanes = keys.
template <int D>
__global__ __launch_bounds__(GA_THREADS, D == 64 ? 2 : 1) void ga_bwd_kv_kernel(GroupedArgs a,
                                                                                int total) {
  __shared__ __attribute__((aligned(1024))) bf16 sQ[2][GA_TILE * D], sO[2][GA_TILE * D];
  __shared__ __attribute__((aligned(16))) float sL[2][GA_TILE], sD[2][GA_TILE];
  Item it;
  if (!ga_item(a.kv_heads, (a.n_k + GA_ROWS - 1) / GA_ROWS, total, false, &it)) return;
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const int wave = wave_index<GA_THREADS / 64>();
  const int len = ga_length(a, it.b), off = a.n_k - a.n_q;
  const int blk0 = it.tile * GA_ROWS, j0 = blk0 + 32 * wave;
  const int pad = (a.n_q + GA_TILE - 1) / GA_TILE * GA_TILE;
  const bf16* kb = a.k + (size_t)it.b * a.n_k * a.k_stride + (size_t)it.h * D;
  const bf16* vb = a.v + (size_t)it.b * a.n_k * a.v_stride + (size_t)it.h * D;
  bf16x8 kf[D / 16], vf[D / 16];
  ga_rows<D>(kf, kb, a.k_stride, j0, len, lane);
  ga_rows<D>(vf, vb, a.v_stride, j0, len, lane);
  f32x16 dk[D / 32] = {}, dv[D / 32] = {};
  const float sc = a.scale * GA_LOG2E;
  const size_t os = (size_t)a.q_heads * D;
  // the first query tile that sees any of the block's keys
  const int first = a.causal && blk0 - off > 0 ? (blk0 - off) / GA_TILE : 0;
  const int per = blk0 < len ? max(0, pad / GA_TILE - first) : 0, steps = per * a.group;
  TileLoad<D> lq, lo;
  float rl = 0.f, rd = 0.f;
  auto load = [&](int step) {
    const int g = step / per, i0 = (first + step - g * per) * GA_TILE, h = it.h * a.group + g;
    lq.load(a.q + (size_t)it.b * a.n_q * a.q_stride + (size_t)h * D, a.q_stride, i0, a.n_q);
    lo.load(a.dout + (size_t)it.b * a.n_q * os + (size_t)h * D, os, i0, a.n_q);
    const size_t row = ((size_t)it.b * a.q_heads + h) * pad + i0 + lane;
    if (wave == 0) rl = a.row_lse[row];
    if (wave == 1) rd = a.row_sum[row];
  };
  auto store = [&](int buf) {
    lq.store(sQ[buf]);
    lo.store(sO[buf]);
    if (wave == 0) sL[buf][lane] = rl;
    if (wave == 1) sD[buf][lane] = rd;
  };
  if (steps) {
    load(0);
    store(0);
  }
  for (int step = 0; step < steps; step++) {
    __syncthreads();
    if (step + 1 < steps) load(step + 1);
    const int buf = step & 1, i0 = (first + step % per) * GA_TILE;
    const bf16 *tq = sQ[buf], *to = sO[buf];
#pragma unroll
    for (int qt = 0; qt < 2; qt++) {
      const int r0 = i0 + 32 * qt;
      if (j0 >= len || (a.causal && r0 + 31 + off < j0)) continue;     // wave-uniform
      f32x16 s = {}, dp = {};
#pragma unroll
      for (int ks = 0; ks < D / 16; ks++) {
        s = mfma32(ga_frag<D>(tq, 32 * qt, 16 * ks, lane), kf[ks], s);
        dp = mfma32(ga_frag<D>(to, 32 * qt, 16 * ks, lane), vf[ks], dp);
      }
      // register e: query r0 + 8 (e / 4) + 4 half + e % 4, key j0 + lane % 32
#pragma unroll
      for (int g = 0; g < 4; g++) {
        const f32x4 l4 = *(const f32x4*)(sL[buf] + 32 * qt + 8 * g + 4 * half);
#pragma unroll
        for (int r = 0; r < 4; r++)
          s[4 * g + r] = __builtin_amdgcn_exp2f(fmaf(s[4 * g + r], sc, -l4[r]));
      }
      if (j0 + 32 > len || (a.causal && r0 + off < j0 + 31)) {
        const int j = j0 + (lane & 31);
        const int from = j >= len ? 1 << 30 : a.causal ? j - off - r0 : -1;   // first row that sees it
#pragma unroll
        for (int e = 0; e < 16; e++)
          if (8 * (e >> 2) + 4 * half + (e & 3) < from) s[e] = 0.f;
      }
#pragma unroll
      for (int g = 0; g < 4; g++) {
        const f32x4 d4 = *(const f32x4*)(sD[buf] + 32 * qt + 8 * g + 4 * half);
#pragma unroll
        for (int r = 0; r < 4; r++) dp[4 * g + r] = s[4 * g + r] * (dp[4 * g + r] - d4[r]);
      }
#pragma unroll
      for (int mm = 0; mm < 2; mm++) {
        const bf16x8 pf = att_pack(s, mm), sf = att_pack(dp, mm);
#pragma unroll
        for (int d = 0; d < D / 32; d++) {
          dv[d] = mfma32(ga_trfrag<D>(to, 32 * qt + 16 * mm, 32 * d, lane), pf, dv[d]);
          dk[d] = mfma32(ga_trfrag<D>(tq, 32 * qt + 16 * mm, 32 * d, lane), sf, dk[d]);
        }
      }
    }
    if (step + 1 < steps) store((step + 1) & 1);
  }
  if (j0 >= a.n_k) return;
  bf16* dkb = a.dk + ((size_t)it.b * a.n_k + j0) * a.dk_stride + (size_t)it.h * D;
  bf16* dvb = a.dv + ((size_t)it.b * a.n_k + j0) * a.dv_stride + (size_t)it.h * D;
#pragma unroll
  for (int d = 0; d < D / 32; d++) {
    att_store(dkb + 32 * d, a.dk_stride, dk[d], a.scale, lane, a.n_k - j0);
    att_store(dvb + 32 * d, a.dv_stride, dv[d], 1.f, lane, a.n_k - j0);
  }
}

// dQ of 128 queries of one head: over the key tiles they see, S^T and dP^T with
// lanes = queries.
template <int D>
__global__ __launch_bounds__(GA_THREADS, D == 64 ? 2 : 1) void ga_bwd_q_kernel(GroupedArgs a,
                                                                               int total) {
  __shared__ __attribute__((aligned(1024))) bf16 sK[2][GA_TILE * D], sV[2][GA_TILE * D];
  Item it;
  if (!ga_item(a.q_heads, (a.n_q + GA_ROWS - 1) / GA_ROWS, total, a.causal, &it)) return;
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const int wave = wave_index<GA_THREADS / 64>();
  const int kvh = it.h / a.group, len = ga_length(a, it.b), off = a.n_k - a.n_q;
  const int blk0 = it.tile * GA_ROWS, q0 = blk0 + 32 * wave;
  const int pad = (a.n_q + GA_TILE - 1) / GA_TILE * GA_TILE;
  const bf16* qb = a.q + (size_t)it.b * a.n_q * a.q_stride + (size_t)it.h * D;
  const size_t os = (size_t)a.q_heads * D;
  const bf16* ob = a.dout + (size_t)it.b * a.n_q * os + (size_t)it.h * D;
  const bf16* kb = a.k + (size_t)it.b * a.n_k * a.k_stride + (size_t)kvh * D;
  const bf16* vb = a.v + (size_t)it.b * a.n_k * a.v_stride + (size_t)kvh * D;
  const int blk_end = a.causal ? min(len, blk0 + GA_ROWS + off) : len;
  const int wave_end = a.causal ? min(len, q0 + 32 + off) : len;
  const int full_end = a.causal ? min(len, q0 + 1 + off) : len;
  const int tiles = blk_end > 0 ? (blk_end + GA_TILE - 1) / GA_TILE : 0;
  bf16x8 qf[D / 16], of[D / 16];
  ga_rows<D>(qf, qb, a.q_stride, q0, a.n_q, lane);
  ga_rows<D>(of, ob, os, q0, a.n_q, lane);
  float lq = INFINITY, dq = 0.f;
  if (q0 + (lane & 31) < a.n_q) {
    const size_t row = ((size_t)it.b * a.q_heads + it.h) * pad + q0 + (lane & 31);
    lq = a.row_lse[row];
    dq = a.row_sum[row];
  }
  f32x16 gq[D / 32] = {};
  const float sc = a.scale * GA_LOG2E;
  TileLoad<D> lk, lv;
  if (tiles) {
    lk.load(kb, a.k_stride, 0, len);
    lv.load(vb, a.v_stride, 0, len);
    lk.store(sK[0]);
    lv.store(sV[0]);
  }
  for (int t = 0; t < tiles; t++) {
    __syncthreads();
    if (t + 1 < tiles) {
      lk.load(kb, a.k_stride, (t + 1) * GA_TILE, len);
      lv.load(vb, a.v_stride, (t + 1) * GA_TILE, len);
    }
    const bf16 *tk = sK[t & 1], *tv = sV[t & 1];
    const int k0 = t * GA_TILE;
#pragma unroll
    for (int kt = 0; kt < 2; kt++) {
      if (k0 + 32 * kt >= wave_end) continue;       // wave-uniform
      f32x16 s = {}, dp = {};
#pragma unroll
      for (int ks = 0; ks < D / 16; ks++) {
        s = mfma32(ga_frag<D>(tk, 32 * kt, 16 * ks, lane), qf[ks], s);
        dp = mfma32(ga_frag<D>(tv, 32 * kt, 16 * ks, lane), of[ks], dp);
      }
#pragma unroll
      for (int e = 0; e < 16; e++) s[e] = __builtin_amdgcn_exp2f(fmaf(s[e], sc, -lq));
      if (k0 + 32 * kt + 32 > full_end) {
        const int end = a.causal ? min(len, q0 + (lane & 31) + 1 + off) : len;
#pragma unroll
        for (int e = 0; e < 16; e++)
          if (k0 + 32 * kt + 8 * (e >> 2) + 4 * half + (e & 3) >= end) s[e] = 0.f;
      }
#pragma unroll
      for (int e = 0; e < 16; e++) s[e] *= dp[e] - dq;
#pragma unroll
      for (int mm = 0; mm < 2; mm++) {
        const bf16x8 sf = att_pack(s, mm);
#pragma unroll
        for (int d = 0; d < D / 32; d++)
          gq[d] = mfma32(ga_trfrag<D>(tk, 32 * kt + 16 * mm, 32 * d, lane), sf, gq[d]);
      }
    }
    if (t + 1 < tiles) {
      lk.store(sK[(t + 1) & 1]);
      lv.store(sV[(t + 1) & 1]);
    }
  }
  if (q0 >= a.n_q) return;
  bf16* dqb = a.dq + ((size_t)it.b * a.n_q + q0) * a.dq_stride + (size_t)it.h * D;
#pragma unroll
  for (int d = 0; d < D / 32; d++) att_store(dqb + 32 * d, a.dq_stride, gq[d], a.scale, lane, a.n_q - q0);
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
    const size_t pad = (size_t)(a.n_q + GA_TILE - 1) / GA_TILE * GA_TILE;
    s.dout += qo * hd;
    s.dq += qo * a.dq_stride;
    s.dk += ko * a.dk_stride;
    s.dv += ko * a.dv_stride;
    s.row_sum += (size_t)b0 * a.q_heads * pad;
    s.row_lse += (size_t)b0 * a.q_heads * pad;
  }
  return s;
}

// A launch's blocks: below 2^32 threads, and whole rounds of the 8 XCDs.
constexpr int64_t GA_MAX_BLOCKS = 1 << 23;
int ga_grid(int64_t total) { return (int)((total + 7) / 8 * 8); }
int64_t ga_tiles(int n) { return (n + GA_ROWS - 1) / GA_ROWS; }

template <int D>
hipError_t ga_forward(const GroupedArgs& a, hipStream_t st) {
  const int64_t per = ga_tiles(a.n_q) * a.q_heads;
  const int64_t most = GA_MAX_BLOCKS / per > 0 ? GA_MAX_BLOCKS / per : 1;
  for (int64_t b0 = 0; b0 < a.batch; b0 += most) {
    const int64_t nb = a.batch - b0 < most ? a.batch - b0 : most, total = nb * per;
    ga_fwd_kernel<D><<<ga_grid(total), GA_THREADS, 0, st>>>(ga_slice(a, b0, nb), (int)total);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <int D>
hipError_t ga_backward(const GroupedArgs& a, hipStream_t st) {
  const int pad = (a.n_q + GA_TILE - 1) / GA_TILE * GA_TILE;
  const int64_t rows = (int64_t)a.q_heads * (pad / 32), rpb = GA_THREADS / 64;
  const int64_t kv = ga_tiles(a.n_k) * a.kv_heads, q = ga_tiles(a.n_q) * a.q_heads;
  const int64_t per = std::max(std::max(kv, q), (rows + rpb - 1) / rpb);
  const int64_t most = GA_MAX_BLOCKS / per > 0 ? GA_MAX_BLOCKS / per : 1;
  for (int64_t b0 = 0; b0 < a.batch; b0 += most) {
    const int64_t nb = a.batch - b0 < most ? a.batch - b0 : most;
    const GroupedArgs s = ga_slice(a, b0, nb);
    ga_row_sum_kernel<D><<<(int)((nb * rows + rpb - 1) / rpb), GA_THREADS, 0, st>>>(s, pad, (int)(nb * rows));
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    ga_bwd_kv_kernel<D><<<ga_grid(nb * kv), GA_THREADS, 0, st>>>(s, (int)(nb * kv));
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    ga_bwd_q_kernel<D><<<ga_grid(nb * q), GA_THREADS, 0, st>>>(s, (int)(nb * q));
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

size_t grouped_workspace_bytes(int64_t batch, int64_t n_q, int32_t q_heads) {
  const size_t pad = (size_t)(n_q + GA_TILE - 1) / GA_TILE * GA_TILE;
  return ((size_t)batch * q_heads * pad * 2 * sizeof(float) + 255) / 256 * 256;
}

hipError_t launch_grouped_forward(const GroupedArgs& a, hipStream_t st) {
  return a.head_dim == 64 ? ga_forward<64>(a, st) : ga_forward<128>(a, st);
}

hipError_t launch_grouped_backward(GroupedArgs a, void* workspace, hipStream_t st) {
  const size_t pad = (size_t)(a.n_q + GA_TILE - 1) / GA_TILE * GA_TILE;
  a.row_sum = (float*)workspace;
  a.row_lse = a.row_sum + (size_t)a.batch * a.q_heads * pad;
  return a.head_dim == 64 ? ga_backward<64>(a, st) : ga_backward<128>(a, st);
}

}  // namespace hcmix
