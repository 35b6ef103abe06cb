// Key/value cache in 8 bits and attention over it.
//
// A sequence's tokens lie in blocks of 64.  Every block of every key/value head
// holds its keys and its values as e4m3 numbers (4 significant bits, largest
// 448) times one power of two each, the least by which the largest value in the
// block is at most 448.  A power of two costs no significant bit, and a block
// whose scale has to grow for a later token is held again at the new one
// without a second rounding (but of what then falls below 2^-6 of a unit, where
// e4m3 has fewer bits).
//
// Layout, made for the attention's loads: for each (sequence, head, block)
//   keys    [64 tokens][D] bytes
//   values  [D][64] bytes, token t at kv_slot(t) of a row
//   scales  fp32: keys, values
// With the 16 x 16 x 32 matrix instruction S^T = K Q^T leaves lane (c = l % 16,
// g = l / 16) with query c and keys 16 j + 4 g + 0..3 of each group j of 16, and
// P V takes P from those registers when the values' fragment holds the same
// keys: kv_slot puts a lane's 16 keys of the block in 16 consecutive bytes of
// each dimension's row.  So both operands go from memory to registers to the
// matrix instruction, with no LDS and no transposition, in 16-byte loads of
// whole lines; the conversion to bf16 multiplies the scale in, exactly.  P, the other
// operand of that instruction, is rounded to bf16 as well; its sum is taken before.
#include <algorithm>

#include "hcmix_internal.h"
#include "device_common.h"

namespace hcmix {

namespace {

constexpr int KV_THREADS = 256;
constexpr int KV_WAVES = KV_THREADS / 64;
constexpr int KB = kKvBlock;
constexpr float KV_LOG2E = 1.4426950408889634f;
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ int kv_slot(int t) {
  return 16 * ((t >> 2) & 3) + 8 * (t >> 5) + 4 * ((t >> 4) & 1) + (t & 3);
}

__device__ __forceinline__ int kv_bounded(int v, int lo, int hi) { return v < lo ? lo : v > hi ? hi : v; }

// The least power of two, 2^-118 .. 2^120, by which amax divided is at most 448
// = 1.75 2^8.
__device__ __forceinline__ float kv_scale(float amax) {
  const unsigned u = __float_as_uint(amax);
  int e = (int)(u >> 23) - 127 - ((u & 0x7fffff) > 0x600000 ? 7 : 8);
  e = kv_bounded(e, -118, 120);
  return __uint_as_float((unsigned)(e + 127) << 23);
}

// At the scale 2^120 quotients reach 255, which e4m3 rounds to 256 from 248 on: 2^128,
// infinite in bf16.  So finite numbers are held to 240 2^120.  (One past that asks for the
// scale 2^120 by itself.)
constexpr float KV_TOP = 0x1p120f, KV_MOST = 0x1.ep127f;
__device__ __forceinline__ float kv_finite(float x) {
  return x > KV_MOST && x < INFINITY ? KV_MOST : x < -KV_MOST && x > -INFINITY ? -KV_MOST : x;
}

// |v| <= 448 or infinite (held as 448), or NaN (held as NaN).
__device__ __forceinline__ unsigned char kv_byte(float v) {
  v = v > 448.f ? 448.f : v < -448.f ? -448.f : v;
  return (unsigned char)__builtin_amdgcn_cvt_pk_fp8_f32(v, v, 0, false);
}
__device__ __forceinline__ float kv_value(unsigned byte) {
  return __builtin_amdgcn_cvt_f32_fp8((int)byte, 0);
}

// 16 bytes times `scale` (a power of two: exact) as two operand fragments.
__device__ __forceinline__ void kv_expand(const u32x4& v, float scale, bf16x8* lo, bf16x8* hi) {
#pragma unroll
  for (int w = 0; w < 4; w++) {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[w], scale, false);
    const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[w], scale, true);
    bf16x8& f = w < 2 ? *lo : *hi;
    const int e = 4 * (w & 1);
    f[e] = a[0];
    f[e + 1] = a[1];
    f[e + 2] = b[0];
    f[e + 3] = b[1];
  }
}

// Four bytes (tokens 4 i .. 4 i + 3 of a dimension) of a block's values in LDS:
// rows of 17 words, so that the lanes that hold neighbouring dimensions of one
// token group meet in no bank.
constexpr int KV_ROW = KB / 4 + 1;
__device__ __forceinline__ int kv_word(int dim, int group) { return dim * KV_ROW + (kv_slot(4 * group) >> 2); }

// 16 held numbers at another scale.
__device__ __forceinline__ u32x4 kv_rescaled(u32x4 v, float ratio) {
#pragma unroll
  for (int w = 0; w < 4; w++) {
    unsigned r = 0;
#pragma unroll
    for (int e = 0; e < 4; e++)
      r |= (unsigned)kv_byte(kv_value((v[w] >> (8 * e)) & 255) * ratio) << (8 * e);
    v[w] = r;
  }
  return v;
}

// ---------------------------------------------------------------------------
// Append: a block of threads per touched block of one head and sequence.  Its
// new tokens are read once, an item of 4 tokens x 8 dimensions to a thread: the
// largest magnitude, then the bytes, from registers.  Values turn in LDS where the
// block is filled from its first token on; into a block that holds some already
// they go byte by byte.
// ---------------------------------------------------------------------------
template <int D>
__global__ __launch_bounds__(KV_THREADS) void kv_append_kernel(KvAppendArgs a) {
  constexpr int DV = D / 8, ITEMS = KB / 4 * DV;   // of keys, as many of values
  constexpr int PER = 2 * ITEMS / KV_THREADS;      // per thread: keys and values, or one of them
  __shared__ unsigned tile[D * KV_ROW];
  __shared__ float part[2][KV_WAVES];
  const int h = blockIdx.y, b = blockIdx.z;
  const int pos = a.positions[b];
  const int count = a.counts ? kv_bounded(a.counts[b], 0, a.tokens) : a.tokens;
  if (pos < 0 || pos >= a.capacity) return;
  const int end = a.capacity - pos < count ? a.capacity : pos + count;
  const int blk = pos / KB + blockIdx.x, first = blk * KB;
  const int t0 = first > pos ? first : pos, t1 = end < first + KB ? end : first + KB;
  if (t0 >= t1) return;
  const int old = t0 - first;                      // earlier tokens of the block
  const size_t at = ((size_t)b * a.kv_heads + h) * a.blocks + blk;
  unsigned char *ck = a.keys + at * KB * D, *cv = a.values + at * KB * D;
  float* scales = a.scales + 2 * at;
  const float ok = old ? scales[0] : 0.f, ov = old ? scales[1] : 0.f;
  bf16x8 x[PER][4];
  float amax[2] = {0.f, 0.f};
#pragma unroll
  for (int i = 0; i < PER; i++) {
    const int item = threadIdx.x + KV_THREADS * i, of_v = item / ITEMS, rest = item % ITEMS;
    const int g = rest / DV, p = rest % DV;
    const bf16* src = (of_v ? a.v : a.k) + (size_t)h * D + 8 * p;
    const size_t stride = of_v ? a.v_stride : a.k_stride;
    float m = 0.f;
#pragma unroll
    for (int r = 0; r < 4; r++) {
      const int t = first + 4 * g + r;
      x[i][r] = bf16x8{};
      if (t >= t0 && t < t1) x[i][r] = *(const bf16x8*)(src + ((size_t)b * a.tokens + (t - pos)) * stride);
    }
#pragma unroll
    for (int r = 0; r < 4; r++)
#pragma unroll
      for (int e = 0; e < 8; e++) m = fmaxf(m, fabsf((float)x[i][r][e]));
    amax[0] = fmaxf(amax[0], of_v ? 0.f : m);
    amax[1] = fmaxf(amax[1], of_v ? m : 0.f);
  }
#pragma unroll
  for (int s = 32; s; s >>= 1) {
    amax[0] = fmaxf(amax[0], __shfl_xor(amax[0], s));
    amax[1] = fmaxf(amax[1], __shfl_xor(amax[1], s));
  }
  if ((threadIdx.x & 63) == 0) {
    part[0][threadIdx.x >> 6] = amax[0];
    part[1][threadIdx.x >> 6] = amax[1];
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < KV_WAVES; w++) {
    amax[0] = fmaxf(amax[0], part[0][w]);
    amax[1] = fmaxf(amax[1], part[1][w]);
  }
  const float sk = fmaxf(kv_scale(amax[0]), ok), sv = fmaxf(kv_scale(amax[1]), ov);
  if (threadIdx.x == 0) {
    scales[0] = sk;
    scales[1] = sv;
  }
  // what is there already, at the new scale (and what lies behind it, which
  // nothing takes)
  if (old && sk > ok)
    for (int i = threadIdx.x; i < old * (D / 16); i += KV_THREADS)
      ((u32x4*)ck)[i] = kv_rescaled(((u32x4*)ck)[i], ok / sk);
  if (old && sv > ov) {
    for (int i = threadIdx.x; i < KB * D / 16; i += KV_THREADS)
      ((u32x4*)cv)[i] = kv_rescaled(((u32x4*)cv)[i], ov / sv);
    __syncthreads();                               // new bytes go between them
  }
  if (sk == KV_TOP || sv == KV_TOP)                // of the block
#pragma unroll
    for (int i = 0; i < PER; i++)
#pragma unroll
      for (int r = 0; r < 4; r++)
#pragma unroll
        for (int e = 0; e < 8; e++) x[i][r][e] = (bf16)kv_finite((float)x[i][r][e]);
  const float ik = 1.f / sk, iv = 1.f / sv;        // exact
#pragma unroll
  for (int i = 0; i < PER; i++) {
    const int item = threadIdx.x + KV_THREADS * i, of_v = item / ITEMS, rest = item % ITEMS;
    const int g = rest / DV, p = rest % DV, t = first + 4 * g;
    if (t + 4 <= t0 || t >= t1) {
      if (of_v && !old)
#pragma unroll
        for (int e = 0; e < 8; e++) tile[kv_word(8 * p + e, g)] = 0;
      continue;
    }
    unsigned char bytes[4][8];
#pragma unroll
    for (int r = 0; r < 4; r++)
#pragma unroll
      for (int e = 0; e < 8; e++) bytes[r][e] = kv_byte((float)x[i][r][e] * (of_v ? iv : ik));
    if (!of_v) {
#pragma unroll
      for (int r = 0; r < 4; r++)
        if (t + r >= t0 && t + r < t1)
          *(uint2*)(ck + (4 * g + r) * D + 8 * p) =
              uint2{bytes[r][0] | (unsigned)bytes[r][1] << 8 | (unsigned)bytes[r][2] << 16 | (unsigned)bytes[r][3] << 24,
                    bytes[r][4] | (unsigned)bytes[r][5] << 8 | (unsigned)bytes[r][6] << 16 | (unsigned)bytes[r][7] << 24};
    } else if (!old) {
#pragma unroll
      for (int e = 0; e < 8; e++)
        tile[kv_word(8 * p + e, g)] = bytes[0][e] | (unsigned)bytes[1][e] << 8 |
                                      (unsigned)bytes[2][e] << 16 | (unsigned)bytes[3][e] << 24;
    } else {
#pragma unroll
      for (int r = 0; r < 4; r++)
        if (t + r >= t0 && t + r < t1)
#pragma unroll
          for (int e = 0; e < 8; e++) cv[(8 * p + e) * KB + kv_slot(4 * g + r)] = bytes[r][e];
    }
  }
  if (!old) {
    __syncthreads();
    for (int i = threadIdx.x; i < D * (KB / 16); i += KV_THREADS) {
      const unsigned* w = tile + i / (KB / 16) * KV_ROW + i % (KB / 16) * 4;
      ((u32x4*)cv)[i] = u32x4{w[0], w[1], w[2], w[3]};
    }
  }
}

// One token of every sequence, the decoding step's form: a wave to a head, lane l
// the dimensions l and, for 128, 64 + l.  (64 sequences of 8 heads of 64: 6.5 us with
// the kernel above, whose 256 threads meet twice for one row, 3.4 so.)
template <int D>
__global__ __launch_bounds__(KV_THREADS) void kv_append_one_kernel(KvAppendArgs a) {
  constexpr int DL = D / 64;
  const int lane = threadIdx.x & 63, b = blockIdx.y;
  const int h = blockIdx.x * KV_WAVES + wave_index<KV_WAVES>();
  if (h >= a.kv_heads) return;
  const int pos = __builtin_amdgcn_readfirstlane(a.positions[b]);
  const int count = a.counts ? __builtin_amdgcn_readfirstlane(a.counts[b]) : 1;
  if (pos < 0 || pos >= a.capacity || count < 1) return;
  const int old = pos % KB;
  const size_t at = ((size_t)b * a.kv_heads + h) * a.blocks + pos / KB;
  unsigned char *ck = a.keys + at * KB * D, *cv = a.values + at * KB * D;
  float* scales = a.scales + 2 * at;
  const float2 held = old ? *(const float2*)scales : float2{0.f, 0.f};
  float x[DL], y[DL], mk = 0.f, mv = 0.f;
#pragma unroll
  for (int i = 0; i < DL; i++) {
    x[i] = kv_finite((float)a.k[(size_t)b * a.k_stride + (size_t)h * D + 64 * i + lane]);
    y[i] = kv_finite((float)a.v[(size_t)b * a.v_stride + (size_t)h * D + 64 * i + lane]);
    mk = fmaxf(mk, fabsf(x[i]));
    mv = fmaxf(mv, fabsf(y[i]));
  }
#pragma unroll
  for (int s = 32; s; s >>= 1) {
    mk = fmaxf(mk, __shfl_xor(mk, s));
    mv = fmaxf(mv, __shfl_xor(mv, s));
  }
  const float sk = fmaxf(kv_scale(mk), held.x), sv = fmaxf(kv_scale(mv), held.y);
  if (lane == 0) *(float2*)scales = float2{sk, sv};
  if (old && sk > held.x)
    for (int i = lane; i < old * (D / 16); i += 64)
      ((u32x4*)ck)[i] = kv_rescaled(((u32x4*)ck)[i], held.x / sk);
  if (old && sv > held.y) {
    for (int i = lane; i < KB * D / 16; i += 64)
      ((u32x4*)cv)[i] = kv_rescaled(((u32x4*)cv)[i], held.y / sv);
    // the new byte goes between them: this wave's stores stay in order
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  }
#pragma unroll
  for (int i = 0; i < DL; i++) {
    ck[old * D + 64 * i + lane] = kv_byte(x[i] * (1.f / sk));
    cv[(64 * i + lane) * KB + kv_slot(old)] = kv_byte(y[i] * (1.f / sv));
  }
}

// ---------------------------------------------------------------------------
// Read: tokens first[b] .. + tokens of every sequence, zeros from lengths[b] on;
// a block of threads per touched block, as the append has them.
// ---------------------------------------------------------------------------
template <int D>
__global__ __launch_bounds__(KV_THREADS) void kv_read_kernel(KvReadArgs a) {
  // an item is R tokens x 8 dimensions: one to a thread
  constexpr int DV = D / 8, R = D / 32;
  static_assert(KB / R * DV == KV_THREADS, "");
  __shared__ unsigned tile[D * KV_ROW];
  const int h = blockIdx.y, b = blockIdx.z;
  const int from = a.first[b], len = kv_bounded(a.lengths[b], 0, a.capacity);
  const int64_t start = ((int64_t)from - ((from % KB) + KB) % KB) + (int64_t)blockIdx.x * KB;
  if (start >= (int64_t)from + a.tokens) return;
  const bool held = start >= 0 && start < len;     // (then a block of the cache)
  const size_t at = held ? ((size_t)b * a.kv_heads + h) * a.blocks + start / KB : 0;
  const unsigned char *ck = a.keys + at * KB * D, *cv = a.values + at * KB * D;
  const int g = threadIdx.x / DV, p = threadIdx.x % DV;
  uint2 c[R];
  float2 scale = {0.f, 0.f};
  if (held) {
    constexpr int PER = D * (KB / 16) / KV_THREADS;
    u32x4 v[PER];
#pragma unroll
    for (int i = 0; i < PER; i++) v[i] = ((const u32x4*)cv)[threadIdx.x + KV_THREADS * i];
#pragma unroll
    for (int r = 0; r < R; r++) c[r] = *(const uint2*)(ck + (R * g + r) * D + 8 * p);
    scale = *(const float2*)(a.scales + 2 * at);
#pragma unroll
    for (int i = 0; i < PER; i++) {
      const int n = threadIdx.x + KV_THREADS * i;
      unsigned* w = tile + n / (KB / 16) * KV_ROW + n % (KB / 16) * 4;
#pragma unroll
      for (int e = 0; e < 4; e++) w[e] = v[i][e];
    }
  }
  __syncthreads();
  unsigned w[8];
#pragma unroll
  for (int e = 0; e < 8; e++) w[e] = held ? tile[kv_word(8 * p + e, R * g / 4)] : 0;
#pragma unroll
  for (int r = 0; r < R; r++) {
    const int64_t pos = start + R * g + r, t = pos - from;
    if (t < 0 || t >= a.tokens) continue;
    bf16x8 x = {}, y = {};
    if (held && pos < len) {
      const int byte = 8 * ((R * g + r) & 3);      // of its group of four tokens
#pragma unroll
      for (int e = 0; e < 8; e++) {
        x[e] = to_bf16(kv_value(((e < 4 ? c[r].x : c[r].y) >> (8 * (e & 3))) & 255) * scale.x);
        y[e] = to_bf16(kv_value((w[e] >> byte) & 255) * scale.y);
      }
    }
    const size_t o = (((size_t)b * a.tokens + t) * a.kv_heads + h) * D + 8 * p;
    *(bf16x8*)(a.k + o) = x;
    *(bf16x8*)(a.v + o) = y;
  }
}

// ---------------------------------------------------------------------------
// Attention: a block of W waves takes a range of the sequence's blocks for one
// key/value head and 16 NQ of its query rows (token, head of the group); its
// waves take the range's blocks in turn, each with its own running maximum
// and sums, joined at the end.
// ---------------------------------------------------------------------------
template <int D, int NQ, int W>
__global__ __launch_bounds__(64 * W) void kv_attention_kernel(KvAttentionArgs a) {
  constexpr int KS = D / 32, DT = D / 16;
  __shared__ float sm[W][16 * NQ], sl[W][16 * NQ];
  __shared__ __attribute__((aligned(16))) float so[W][16][D + 4];
  const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  const int wave = wave_index<W>();
  const int split = blockIdx.x % a.splits, rt = blockIdx.x / a.splits;
  const int h = blockIdx.y, b = blockIdx.z;
  const int rows = a.tokens * a.group, r0 = rt * 16 * NQ;
  const int len = kv_bounded(__builtin_amdgcn_readfirstlane(a.lengths[b]), 0, a.capacity);
  const int base = len - a.tokens;              // position of the first query token
  // a row past the last repeats it and is not stored
  bf16x8 q[NQ][KS];
  int end[NQ];                                  // keys that this lane's row sees
  int first_end = 1 << 30;                      // keys that all rows see
#pragma unroll
  for (int j = 0; j < NQ; j++) {
    const int r = r0 + 16 * j + c < rows ? r0 + 16 * j + c : rows - 1;
    const int t = r / a.group, qh = h * a.group + r - t * a.group;
    const bf16* p = a.q + ((size_t)b * a.tokens + t) * a.q_stride + (size_t)qh * D;
    end[j] = base + t + 1;
#pragma unroll
    for (int s = 0; s < KS; s++) q[j][s] = *(const bf16x8*)(p + (s >> 1) * 64 + 16 * g + 8 * (s & 1));
  }
  first_end = base + r0 / a.group + 1;
  const int last_row = r0 + 16 * NQ < rows ? r0 + 16 * NQ - 1 : rows - 1;
  const int last_end = base + last_row / a.group + 1;        // keys that any row sees, <= len
  const int nblk = last_end > 0 ? (last_end + KB - 1) / KB : 0;
  const int per = (nblk + a.splits - 1) / a.splits;
  const int lo = split * per, hi = lo + per < nblk ? lo + per : nblk;
  const size_t at0 = ((size_t)b * a.kv_heads + h) * a.blocks;
  const float sc = a.scale * KV_LOG2E;
  f32x4 o[NQ][DT] = {};
  float m[NQ], l[NQ];
#pragma unroll
  for (int j = 0; j < NQ; j++) {
    m[j] = -3e38f;
    l[j] = 0.f;
  }
  for (int blk = lo + wave; blk < hi; blk += W) {
    const size_t at = at0 + blk;
    const unsigned char* ck = a.keys + at * KB * D;
    const unsigned char* cv = a.values + at * KB * D;
    u32x4 kr[4][D / 64], vr[DT];
#pragma unroll
    for (int t = 0; t < 4; t++)
#pragma unroll
      for (int s = 0; s < D / 64; s++)
        kr[t][s] = __builtin_nontemporal_load((const u32x4*)(ck + (16 * t + c) * D + 64 * s + 16 * g));
#pragma unroll
    for (int d = 0; d < DT; d++) vr[d] = __builtin_nontemporal_load((const u32x4*)(cv + (16 * d + c) * KB + 16 * g));
    const float2 scl = *(const float2*)(a.scales + 2 * at);
    const int k0 = blk * KB;
    if (k0 + KB > len) {
      // the last block: values behind the last token may be anything, NaN among it
      unsigned keep[4];
#pragma unroll
      for (int w = 0; w < 4; w++) {
        // byte 4 w + r of a lane: key 32 (w / 2) + 16 (w % 2) + 4 g + r
        const int left = len - (k0 + 32 * (w >> 1) + 16 * (w & 1) + 4 * g);
        keep[w] = left >= 4 ? ~0u : left <= 0 ? 0u : ~0u >> (32 - 8 * left);
      }
#pragma unroll
      for (int d = 0; d < DT; d++)
#pragma unroll
        for (int w = 0; w < 4; w++) vr[d][w] &= keep[w];
    }
    f32x4 s[NQ][4];
#pragma unroll
    for (int t = 0; t < 4; t++) {
      bf16x8 kf[KS];
#pragma unroll
      for (int u = 0; u < D / 64; u++) kv_expand(kr[t][u], scl.x, &kf[2 * u], &kf[2 * u + 1]);
#pragma unroll
      for (int j = 0; j < NQ; j++) {
        s[j][t] = f32x4{};
#pragma unroll
        for (int u = 0; u < KS; u++) s[j][t] = mfma16(kf[u], q[j][u], s[j][t]);
      }
    }
    if (k0 + KB > first_end) {
#pragma unroll
      for (int j = 0; j < NQ; j++)
#pragma unroll
        for (int t = 0; t < 4; t++)
#pragma unroll
          for (int r = 0; r < 4; r++)
            if (k0 + 16 * t + 4 * g + r >= end[j]) s[j][t][r] = -INFINITY;
    }
    bf16x8 p[NQ][2];
#pragma unroll
    for (int j = 0; j < NQ; j++) {
      float mx = s[j][0][0];
#pragma unroll
      for (int t = 0; t < 4; t++)
#pragma unroll
        for (int r = 0; r < 4; r++) mx = fmaxf(mx, s[j][t][r]);
      mx = fmaxf(mx, __shfl_xor(mx, 16));
      mx = fmaxf(mx, __shfl_xor(mx, 32)) * sc;
      const float mn = fmaxf(m[j], mx), alpha = __builtin_amdgcn_exp2f(m[j] - mn);
      m[j] = mn;
      l[j] *= alpha;
#pragma unroll
      for (int d = 0; d < DT; d++) o[j][d] *= alpha;
#pragma unroll
      for (int t = 0; t < 4; t++)
#pragma unroll
        for (int r = 0; r < 4; r++) {
          const float e = __builtin_amdgcn_exp2f(fmaf(s[j][t][r], sc, -mn));
          l[j] += e;
          p[j][t >> 1][4 * (t & 1) + r] = to_bf16(e);
        }
    }
#pragma unroll
    for (int d = 0; d < DT; d++) {
      bf16x8 lo8, hi8;
      kv_expand(vr[d], scl.y, &lo8, &hi8);
#pragma unroll
      for (int j = 0; j < NQ; j++) {
        o[j][d] = mfma16(lo8, p[j][0], o[j][d]);
        o[j][d] = mfma16(hi8, p[j][1], o[j][d]);
      }
    }
  }
  // join the waves: o[j][d] register r of a lane: row 16 j + c, dimension 16 d + 4 g + r
#pragma unroll
  for (int j = 0; j < NQ; j++) {
    l[j] += __shfl_xor(l[j], 16);
    l[j] += __shfl_xor(l[j], 32);
    if (g == 0) {
      sm[wave][16 * j + c] = m[j];
      sl[wave][16 * j + c] = l[j];
    }
  }
#pragma unroll
  for (int j = 0; j < NQ; j++) {
    __syncthreads();
#pragma unroll
    for (int d = 0; d < DT; d++) *(f32x4*)&so[wave][c][16 * d + 4 * g] = o[j][d];
    __syncthreads();
    for (int i = threadIdx.x; i < 16 * D / 4; i += 64 * W) {
      const int row = i / (D / 4), d4 = i % (D / 4), r = r0 + 16 * j + row;
      if (r >= rows) continue;
      float mm = -3e38f, ll = 0.f;
#pragma unroll
      for (int w = 0; w < W; w++) mm = fmaxf(mm, sm[w][16 * j + row]);
      f32x4 acc = {};
#pragma unroll
      for (int w = 0; w < W; w++) {
        const float f = __builtin_amdgcn_exp2f(sm[w][16 * j + row] - mm);
        ll += f * sl[w][16 * j + row];
        acc += f * *(const f32x4*)&so[w][row][4 * d4];
      }
      const size_t part = (((size_t)b * a.kv_heads + h) * rows + r) * a.splits + split;
      if (a.splits > 1) {
        *(f32x4*)(a.partial + part * D + 4 * d4) = acc;
        if (d4 == 0) *(float2*)(a.stats + 2 * part) = float2{mm, ll};
      } else {
        const int t = r / a.group, qh = h * a.group + r - t * a.group;
        const float inv = ll == 0.f ? 0.f : 1.f / ll;       // 0: the row sees nothing
        bf16x4 y;
#pragma unroll
        for (int e = 0; e < 4; e++) y[e] = to_bf16(acc[e] * inv);
        *(bf16x4*)(a.out + (((size_t)b * a.tokens + t) * a.kv_heads * a.group + qh) * D + 4 * d4) = y;
      }
    }
  }
}

// Joins the ranges of a row, a block to each: D / 4 threads take a range's
// dimensions, so many such groups the ranges in turn, each with its own maximum.
template <int D>
__global__ __launch_bounds__(KV_THREADS) void kv_join_kernel(KvAttentionArgs a) {
  constexpr int T = D / 4, G = KV_THREADS / T;
  __shared__ __attribute__((aligned(16))) f32x4 so[G][T];
  __shared__ float2 sm[G];
  const int64_t row = blockIdx.x;
  const int d4 = threadIdx.x % T, g = threadIdx.x / T;
  const float2* stats = (const float2*)a.stats + row * a.splits;
  const float* part = a.partial + row * a.splits * D + 4 * d4;
  float mm = -3e38f, ll = 0.f;
  f32x4 acc = {};
  for (int s = g; s < a.splits; s += G) mm = fmaxf(mm, stats[s].x);
#pragma unroll 4
  for (int s = g; s < a.splits; s += G) {
    const float2 st = stats[s];
    const float f = __builtin_amdgcn_exp2f(st.x - mm);
    ll += f * st.y;
    acc += f * *(const f32x4*)(part + (size_t)s * D);
  }
  so[g][d4] = acc;
  if (d4 == 0) sm[g] = float2{mm, ll};
  __syncthreads();
  if (g) return;
  mm = sm[0].x;
#pragma unroll
  for (int i = 1; i < G; i++) mm = fmaxf(mm, sm[i].x);
  acc = f32x4{};
  ll = 0.f;
#pragma unroll
  for (int i = 0; i < G; i++) {
    const float f = __builtin_amdgcn_exp2f(sm[i].x - mm);
    ll += f * sm[i].y;
    acc += f * so[i][d4];
  }
  const int rows = a.tokens * a.group;
  const int64_t bh = row / rows, b = bh / a.kv_heads;
  const int r = (int)(row - bh * rows), h = (int)(bh - b * a.kv_heads);
  const int t = r / a.group, qh = h * a.group + r - t * a.group;
  const float inv = ll == 0.f ? 0.f : 1.f / ll;
  bf16x4 y;
#pragma unroll
  for (int e = 0; e < 4; e++) y[e] = to_bf16(acc[e] * inv);
  *(bf16x4*)(a.out + (((size_t)b * a.tokens + t) * a.kv_heads * a.group + qh) * D + 4 * d4) = y;
}

int kv_row_tiles(int rows) { return rows <= 16 ? 1 : rows <= 32 ? 2 : 4; }     // NQ

// How a call is cut: the ranges of a sequence, and the waves of a block.
//
// Ranges: enough blocks of threads for the chip and, where several fit a CU, twice
// as many, since the lengths of a batch differ (32 sequences up to 16384 long, 8
// heads of 128: 109.9 us with 512 blocks, 105.9 with 1024; 64 query rows of
// 8 x 8192, which take a CU each: 38.5 with 256, 44.4 with 512).  A range has one
// of the sequence's blocks for every wave up to 16 ranges (a wave's second block
// is loaded after the first: 1 x 4000, 32 heads of 128 over 8: 10.2 us with two,
// 8.7), two where that makes more (4 x 8000: 13.6, one: 14.9).
//
// Waves: a block of 16, or of 8 where head dimension or rows leave 16 too few
// registers, takes a sequence by itself where none of its waves gets more than one
// and a half blocks, or four where such blocks fill the chip: no partial sums, no
// second kernel.  us with four waves and ranges, and so: 1 x 700, 8 heads of 64
// over 2 7.0, 5.5; 16 x 1000, 8 of 64 over 8 8.4, 7.0; 32 x 2000, 32 of 128 over 8,
// 6 tokens 31.3, 25.1 (but 1 x 1500, 32 of 128 over 8 8.6, 14.4).
struct KvPlan {
  int splits, waves;
};
KvPlan kv_plan(int64_t batch, int kv_heads, int rows, int max_length, int D) {
  const int nq = kv_row_tiles(rows), blocks = (max_length + KB - 1) / KB;
  const int64_t sequences = batch * kv_heads, tiles = sequences * ((rows + 16 * nq - 1) / (16 * nq));
  const int64_t want = (1024 / nq + tiles - 1) / tiles;
  const int64_t per = (blocks + KV_WAVES - 1) / KV_WAVES;
  const int64_t s = std::min(want, std::max(std::min<int64_t>(per, 16), (per + 1) / 2));
  const int w = D == 64 && nq == 1 ? 16 : 8;
  if (s > 1 && nq <= 2 && blocks <= w * (sequences < 256 ? 3 : 8) / 2) return {1, w};
  return {s < 1 ? 1 : (int)s, KV_WAVES};
}

template <int D>
hipError_t kv_attention_launch(const KvAttentionArgs& a, int waves, hipStream_t st) {
  const int rows = a.tokens * a.group, nq = kv_row_tiles(rows);
  const dim3 grid(a.splits * ((rows + 16 * nq - 1) / (16 * nq)), a.kv_heads, a.batch);
  if (waves > KV_WAVES) {
    constexpr int W1 = D == 64 ? 16 : 8;
    if (nq == 1) kv_attention_kernel<D, 1, W1><<<grid, 64 * W1, 0, st>>>(a);
    else kv_attention_kernel<D, 2, 8><<<grid, 512, 0, st>>>(a);
  } else if (nq == 1) {
    kv_attention_kernel<D, 1, KV_WAVES><<<grid, KV_THREADS, 0, st>>>(a);
  } else if (nq == 2) {
    kv_attention_kernel<D, 2, KV_WAVES><<<grid, KV_THREADS, 0, st>>>(a);
  } else {
    kv_attention_kernel<D, 4, KV_WAVES><<<grid, KV_THREADS, 0, st>>>(a);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.splits == 1) return e;
  kv_join_kernel<D><<<(int)(a.batch * a.kv_heads * rows), KV_THREADS, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_kv_append(const KvAppendArgs& a, hipStream_t st) {
  if (a.tokens == 1) {
    const dim3 grid((a.kv_heads + KV_WAVES - 1) / KV_WAVES, a.batch);
    if (a.head_dim == 64) kv_append_one_kernel<64><<<grid, KV_THREADS, 0, st>>>(a);
    else kv_append_one_kernel<128><<<grid, KV_THREADS, 0, st>>>(a);
    return hipGetLastError();
  }
  const dim3 grid((a.tokens + KB - 2) / KB + 1, a.kv_heads, a.batch);
  if (a.head_dim == 64) kv_append_kernel<64><<<grid, KV_THREADS, 0, st>>>(a);
  else kv_append_kernel<128><<<grid, KV_THREADS, 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_kv_read(const KvReadArgs& a, hipStream_t st) {
  const dim3 grid((a.tokens + KB - 2) / KB + 1, a.kv_heads, a.batch);
  if (a.head_dim == 64) kv_read_kernel<64><<<grid, KV_THREADS, 0, st>>>(a);
  else kv_read_kernel<128><<<grid, KV_THREADS, 0, st>>>(a);
  return hipGetLastError();
}

size_t kv_attention_workspace_bytes(int64_t batch, int32_t kv_heads, int32_t group,
                                    int32_t head_dim, int32_t tokens, int32_t max_length) {
  const int splits = kv_plan(batch, kv_heads, tokens * group, max_length, head_dim).splits;
  if (splits == 1) return 0;
  const size_t parts = (size_t)batch * kv_heads * tokens * group * splits;
  return parts * (head_dim + 2) * sizeof(float) / 256 * 256 + 256;
}

hipError_t launch_kv_attention(KvAttentionArgs a, void* workspace, int32_t max_length,
                               hipStream_t st) {
  const KvPlan plan = kv_plan(a.batch, a.kv_heads, a.tokens * a.group, max_length, a.head_dim);
  a.splits = plan.splits;
  a.partial = (float*)workspace;
  a.stats = a.partial + (size_t)a.batch * a.kv_heads * a.tokens * a.group * a.splits * a.head_dim;
  return a.head_dim == 64 ? kv_attention_launch<64>(a, plan.waves, st)
                          : kv_attention_launch<128>(a, plan.waves, st);
}

}  // namespace hcmix
