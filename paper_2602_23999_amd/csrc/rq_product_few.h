// The forward products with few rows per list (single tokens, one query against many stored rows) or few tiles at all.
//
// Every matrix is read once for a handful of rows, so the time is that of reading the matrices: they go straight from memory to the
// registers in which the matrix instructions take them, many loads ahead, and nothing passes through LDS.  A tile is 16 positions of a
// list by 16 columns.
#pragma once
#include "rq_product_tile.h"

namespace rq {

// 16 x 16 products of 64 bytes along c: 16 bytes per lane, row (column) lane % 16, the (lane / 16)-th quarter of the 64 bytes.
template <class T>
struct Mma16 {
  using Acc = f32x4;
  static __device__ __forceinline__ Acc mul(i32x4 a, i32x4 b, Acc c) {
    const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[e], y[e], c, 0, 0, 0);
    return c;
  }
};
template <>
struct Mma16<_Float16> {
  using Acc = f32x4;
  static __device__ __forceinline__ Acc mul(i32x4 a, i32x4 b, Acc c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
};
template <>
struct Mma16<__bf16> {
  using Acc = f32x4;
  static __device__ __forceinline__ Acc mul(i32x4 a, i32x4 b, Acc c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
};
template <>
struct Mma16<int8_t> {
  using Acc = i32x4;
  static __device__ __forceinline__ Acc mul(i32x4 a, i32x4 b, Acc c) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0); }
};

// A workgroup takes 16 columns; its four wavefronts share their contraction, and their sums meet in LDS, in order.  (64 lists of 1024 x
// 1024 bf16, 1 row each: 23 us; one wavefront per column instead: 28, with 64 columns each: 39, which has too few loads in
// flight; four wavefronts for 64 columns: 29.)
template <class T>
__global__ __launch_bounds__(256) void product_few_kernel(ProductArgs p) {
  constexpr int SZ = sizeof(T), EPC = 16 / SZ, SLAB = 64 / SZ;
  constexpr int AHEAD = 4;  // slabs of 64 bytes requested together
  using Acc = typename Mma16<T>::Acc;
  __shared__ Acc sums[4][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, quarter = lane >> 4;
  const uint32_t blocks = (uint32_t)((p.n + 15) / 16);
  const uint32_t tile = blockIdx.x / blocks;
  const int64_t j0 = (int64_t)(blockIdx.x % blocks) * 16;
  const int g = p.pair_off ? list_of_tile(p, tile, 16, lane) : 0;
  const Span s = span_of(p, g);
  const int64_t i0 = s.begin + (tile - (p.pair_off ? s.begin / 16 + g : 0)) * 16;
  if (i0 < s.begin || i0 >= s.end) return;
  const int64_t pair = i0 + l16 < s.end ? pair_at(p, i0 + l16) : -1;
  // (rows that are not there read row 0, unused)
  const T* x = static_cast<const T*>(p.a) + (pair < 0 ? 0 : (int64_t)p.probe.of((int)pair)) * p.lda + quarter * EPC;
  const T* w = static_cast<const T*>(p.b) + (int64_t)g * p.stride + (j0 + l16 < p.n ? j0 + l16 : 0) * p.ldb + quarter * EPC;
  // this wavefront's slabs, whole ones first
  const int slabs = (p.k + SLAB - 1) / SLAB, share = (slabs + 3) / 4;
  const int first = wave * share, last = min(first + share, slabs);
  const int whole = min(last, p.k / SLAB);
  Acc acc = {0, 0, 0, 0};
  int t = first;
  for (; t + AHEAD <= whole; t += AHEAD) {
    i32x4 vx[AHEAD], vw[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      __builtin_memcpy(&vw[u], w + (t + u) * SLAB, 16);  // (with the streaming hint 5 to 10 % slower)
      __builtin_memcpy(&vx[u], x + (t + u) * SLAB, 16);
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) acc = Mma16<T>::mul(vw[u], vx[u], acc);
  }
  for (; t < last; ++t) {
    const int valid = p.k - t * SLAB - quarter * EPC;
    acc = Mma16<T>::mul(load_piece<T>(reinterpret_cast<const char*>(w + t * SLAB), valid),
                        load_piece<T>(reinterpret_cast<const char*>(x + t * SLAB), valid), acc);
  }
  sums[wave][lane] = acc;
  __syncthreads();
  if (wave != 0 || pair < 0) return;
#pragma unroll
  for (int u = 1; u < 4; ++u) acc += sums[u][lane];
  // register r of a lane: column 4 (lane / 16) + r, row lane % 16
  const int64_t j = j0 + 4 * quarter;
  f32x4 v;
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = (float)acc[e];
  if constexpr (SZ == 1) {
    const float sa = p.scale_a[p.probe.of((int)pair)];
    const float* sb = p.scale_b + (int64_t)g * p.n;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = v[e] * sa * sb[j + e < p.n ? j + e : 0];
  }
  const int64_t at = pair * p.ldo + j;
  if (j + 4 <= p.n) {  // (at any alignment of the element)
    typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    if (p.out_dtype == RABITQ_F32) {
      __builtin_memcpy(static_cast<float*>(p.out) + at, &v, 16);
    } else if (p.out_dtype == RABITQ_F16) {
      const f16x4 h = __builtin_convertvector(v, f16x4);
      __builtin_memcpy(static_cast<_Float16*>(p.out) + at, &h, 8);
    } else {
      const bf16x4 h = __builtin_convertvector(v, bf16x4);
      __builtin_memcpy(static_cast<__bf16*>(p.out) + at, &h, 8);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (j + e < p.n) store_as(p.out, p.out_dtype, at + e, v[e]);
  }
}

}  // namespace rq
