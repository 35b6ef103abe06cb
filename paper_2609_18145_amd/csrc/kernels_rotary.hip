// Rotary positions: pairs of a head's values turned by position * frequency.
//
//   (a, b) -> scale (a cos t - b sin t, b cos t + a sin t),   t = position freqs[j]
//
// for the pairs (j, j + rot/2) (half layout) or (2j, 2j + 1) (pairs layout) of a
// head's first rot_dim values; the others are copied.  The inverse takes -t: it
// is the transpose, hence also the backward.
//
// The angle is taken in 64 bits, in turns, and only its fraction is rounded, by 2^-22.3
// radians at most (fp32 results 5.1e-8 off in norm, where 64-bit sines leave 3.8e-8): a
// position of 10^6 times a frequency in 32 bits is off by 0.06 radians.  Every
// head of a position shares the angles, so a block first makes the table of its
// rows' (cos, sin) in LDS and then streams the heads past it: bound by memory, at
// the rate of a copy.
#include "hcmix_internal.h"
#include "device_common.h"

namespace hcmix {

namespace {

constexpr int ROT_THREADS = 256;

template <typename E, int VEC>
__device__ __forceinline__ void rot_load(const E* p, float (&f)[VEC]) {
  typedef E Vec __attribute__((ext_vector_type(VEC)));
  const Vec v = *(const Vec*)p;
#pragma unroll
  for (int e = 0; e < VEC; e++) f[e] = (float)v[e];
}
template <typename E, int VEC>
__device__ __forceinline__ void rot_store(E* p, const float (&f)[VEC]) {
  typedef E Vec __attribute__((ext_vector_type(VEC)));
  Vec v;
#pragma unroll
  for (int e = 0; e < VEC; e++) v[e] = (E)f[e];
  *(Vec*)p = v;
}

// A block takes a.rows_per_block rows and its threads their units in turn; a unit
// is VEC pairs (half layout: VEC values of each half) or VEC values (pairs
// layout, and the values that are copied).
template <typename E, int VEC, bool HALF>
__global__ __launch_bounds__(ROT_THREADS) void rotary_kernel(RotaryArgs a) {
  extern __shared__ float2 tab[];            // [rows_per_block][rot / 2]
  const E* x = (const E*)a.x;
  E* y = (E*)a.y;
  const int pairs = a.rot >> 1, all = a.units * a.heads;
  for (int64_t r0 = (int64_t)blockIdx.x * a.rows_per_block; r0 < a.rows;
       r0 += (int64_t)gridDim.x * a.rows_per_block) {
    const int rows = a.rows - r0 < a.rows_per_block ? (int)(a.rows - r0) : a.rows_per_block;
    for (int i = threadIdx.x; i < rows * pairs; i += ROT_THREADS) {
      const int r = i / pairs, j = i - r * pairs;
      const int64_t pos = a.positions ? (int64_t)a.positions[r0 + r] : (r0 + r) % a.period;
      double t = (double)pos * (a.freqs[j] * 0.15915494309189533577);
      t -= rint(t);
      float s, c;
      sincospif(2.f * (float)t, &s, &c);
      tab[i] = float2{c * a.scale, (a.inverse ? -s : s) * a.scale};
    }
    __syncthreads();
    for (int i = threadIdx.x; i < rows * all; i += ROT_THREADS) {
      // i / all and k / units: exact, as rows < 2^5, all < 2^19 and units < 2^10
      const int r = (int)((unsigned)i * a.all_magic >> 44), k = i - r * all;
      const int h = (int)((unsigned)k * a.units_magic >> 32), u = k - h * a.units;
      const E* xr = x + (size_t)(r0 + r) * a.x_stride;
      E* yr = y + (size_t)(r0 + r) * a.y_stride;
      const float2* cs = tab + r * pairs;
      const size_t at = (size_t)h * a.head_dim;
      if constexpr (HALF) {
        if (u * VEC < pairs) {
          float p[VEC], q[VEC], op[VEC], oq[VEC];
          rot_load<E, VEC>(xr + at + u * VEC, p);
          rot_load<E, VEC>(xr + at + pairs + u * VEC, q);
#pragma unroll
          for (int e = 0; e < VEC; e++) {
            const float2 w = cs[u * VEC + e];
            op[e] = p[e] * w.x - q[e] * w.y;
            oq[e] = q[e] * w.x + p[e] * w.y;
          }
          rot_store<E, VEC>(yr + at + u * VEC, op);
          rot_store<E, VEC>(yr + at + pairs + u * VEC, oq);
        } else {
          const size_t c = at + a.rot + u * VEC - pairs;
          float p[VEC];
          rot_load<E, VEC>(xr + c, p);
          rot_store<E, VEC>(yr + c, p);
        }
      } else {
        constexpr int W = VEC == 1 ? 2 : VEC;      // values of a unit
        const int c = u * W;
        if (c < a.rot) {
          float p[W], o[W];
          if constexpr (VEC == 1) {
            p[0] = (float)xr[at + c];
            p[1] = (float)xr[at + c + 1];
          } else {
            rot_load<E, W>(xr + at + c, p);
          }
#pragma unroll
          for (int e = 0; e < W; e += 2) {
            const float2 w = cs[(c + e) >> 1];
            o[e] = p[e] * w.x - p[e + 1] * w.y;
            o[e + 1] = p[e + 1] * w.x + p[e] * w.y;
          }
          if constexpr (VEC == 1) {
            yr[at + c] = (E)o[0];
            yr[at + c + 1] = (E)o[1];
          } else {
            rot_store<E, W>(yr + at + c, o);
          }
        } else if constexpr (VEC == 1) {
          yr[at + c] = xr[at + c];
          yr[at + c + 1] = xr[at + c + 1];
        } else {
          float p[W];
          rot_load<E, W>(xr + at + c, p);
          rot_store<E, W>(yr + at + c, p);
        }
      }
    }
    __syncthreads();        // the next rows' table
  }
}

template <typename E, int VEC, bool HALF>
hipError_t rotary_launch(const RotaryArgs& a, int blocks, hipStream_t st) {
  const size_t lds = (size_t)a.rows_per_block * (a.rot / 2) * sizeof(float2);
  rotary_kernel<E, VEC, HALF><<<blocks, ROT_THREADS, lds, st>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rotary(RotaryArgs a, int layout_half, int elem_bytes, hipStream_t st) {
  const int vec = 16 / elem_bytes, step = layout_half ? 2 * vec : vec;
  // 16-byte accesses where every vector of every head starts on 16 bytes
  const bool wide = a.head_dim % vec == 0 && a.rot % step == 0 && a.x_stride % vec == 0 &&
                    a.y_stride % vec == 0 && ((uintptr_t)a.x | (uintptr_t)a.y) % 16 == 0;
  const int v = wide ? vec : 1, in_place = a.x == a.y;
  const int moved = in_place ? a.rot : a.head_dim;       // values of a head to go through
  a.units = layout_half ? a.rot / 2 / v + (moved - a.rot) / v : moved / (v == 1 ? 2 : v);
  a.units_magic = ((1ull << 32) + a.units - 1) / a.units;
  const uint64_t all = (uint64_t)a.units * a.heads;
  a.all_magic = ((1ull << 44) + all - 1) / all;
  // Rows to a block: more share the wait for the angles, fewer leave more blocks
  // to hide it: 8 x 4096 positions, 20 heads of 64 (168 MB): 36.9 us with 16 and 8,
  // 34.2 with 4 (4.9 TB/s; a copy of as much takes 33.8; the same tensors again and again,
  // which the Infinity Cache partly holds, 25.9, a copy 24.2).  With few heads more, up
  // to a unit for every thread: 64 x 2048, 2 heads of 64 31.0 us with 4, 20.5; 4 heads
  // 40.2, 29.0; 2 of 20, by single values, 29.7, 16.6.
  int rpb = 1;
  while (rpb < 16 && (rpb < 4 || rpb * all < ROT_THREADS) && rpb * (a.rot / 2) < ROT_THREADS &&
         a.rows / (2 * rpb) >= 1024)
    rpb *= 2;
  a.rows_per_block = rpb;
  const int64_t blocks = (a.rows + rpb - 1) / rpb;
  const int grid = blocks < (1 << 20) ? (int)blocks : 1 << 20;
  if (elem_bytes == 2)
    return layout_half ? (wide ? rotary_launch<bf16, 8, true>(a, grid, st)
                               : rotary_launch<bf16, 1, true>(a, grid, st))
                       : (wide ? rotary_launch<bf16, 8, false>(a, grid, st)
                               : rotary_launch<bf16, 1, false>(a, grid, st));
  return layout_half ? (wide ? rotary_launch<float, 4, true>(a, grid, st)
                             : rotary_launch<float, 1, true>(a, grid, st))
                     : (wide ? rotary_launch<float, 4, false>(a, grid, st)
                             : rotary_launch<float, 1, false>(a, grid, st));
}

}  // namespace hcmix
