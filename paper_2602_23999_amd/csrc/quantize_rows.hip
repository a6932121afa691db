// Rows of numbers as int8 codes with a scale each (rabitq_quantize_rows).
//
// scale = fp32(max |x| / 127), code = the whole number nearest to x / scale, ties to even: of the exact quotient, so that codes do not
// depend on how a division rounds.  q = rint(x (1 / scale)) is that number or, next to a border, a neighbour of it.  The rest
// x - q scale is exact in an FMA (a multiple of the smaller of the two numbers' last places, and about half the scale at most), and
// says which: beyond half the scale on either side, or on it with q odd, the neighbour is the nearest.
//
// Bound by memory: a row is read once and kept in registers (8192 x 4096 bf16, 101 MB: 29 us, 3.5 TB/s, 32 768 x 4096
// 95 us, 4.2 TB/s; the first with a second read of the row and divisions 39 us).
#include "rq_products.h"

namespace rq {

typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int HELD = 4;  // pieces of 16 bytes of a row that a thread keeps

// 16 bytes, of which the first `valid` elements exist, as floats; the others 0.
template <class T>
__device__ __forceinline__ void piece_of(const T* from, int valid, float* v) {
  constexpr int EPC = 16 / sizeof(T);
  T e[EPC];
  if (valid >= EPC) {
    __builtin_memcpy(e, from, 16);
  } else {
#pragma unroll
    for (int i = 0; i < EPC; ++i) e[i] = i < valid ? from[i] : T(0);
  }
#pragma unroll
  for (int i = 0; i < EPC; ++i) v[i] = to_f32(e[i]);
}

struct RowScale {
  float scale, inverse, lift;  // lift: a power of two that takes tiny rows away from the denormal numbers
  bool bad;
};
// top: the largest |x| of the row as bits; those order as the values do, infinity and NaN above all numbers.
__device__ __forceinline__ RowScale row_scale(uint32_t top) {
  RowScale r;
  r.bad = top >= 0x7f800000u;
  r.scale = __uint_as_float(top) / 127.0f;
  if (r.scale == 0.f) r.scale = 1.0f;
  r.lift = r.scale < 0x1p-60f ? 0x1p80f : 1.0f;
  r.inverse = 1.0f / (r.scale * r.lift);
  return r;
}

template <int EPC>
__device__ __forceinline__ void store_codes(const float* v, const RowScale& r, int valid, int8_t* to) {
  const float s = r.scale * r.lift;
  float q[EPC], off = 0.f;
#pragma unroll
  for (int i = 0; i < EPC; ++i) {
    const float x = v[i] * r.lift;
    q[i] = __builtin_rintf(x * r.inverse);
    off = fmaxf(off, fabsf(__builtin_fmaf(-q[i], s, x)));
  }
  if (2.f * off >= s) {  // a border is near
#pragma unroll
    for (int i = 0; i < EPC; ++i) {
      const float rest = 2.f * __builtin_fmaf(-q[i], s, v[i] * r.lift);
      const bool odd = ((int)q[i] & 1) != 0;
      if (rest > s || (rest == s && odd)) q[i] += 1.f;
      else if (rest < -s || (rest == -s && odd)) q[i] -= 1.f;
    }
  }
  int8_t c[EPC];
#pragma unroll
  for (int i = 0; i < EPC; ++i) c[i] = r.bad ? 0 : (int8_t)(int)fminf(fmaxf(q[i], -127.f), 127.f);
  if (valid >= EPC) {
    __builtin_memcpy(to, c, EPC);
  } else {
#pragma unroll
    for (int i = 0; i < EPC; ++i)
      if (i < valid) to[i] = c[i];
  }
}

// WAVES wavefronts share a row (1: four rows per workgroup).  ONCE: the row fits the registers; else it is read twice.
template <class T, int WAVES, bool ONCE>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const T* __restrict__ x, int64_t ldx, int64_t rows, int k,
                                                            int8_t* __restrict__ codes, int64_t ldc, float* __restrict__ scale) {
  constexpr int EPC = 16 / sizeof(T), SPAN = 64 * WAVES;
  __shared__ uint32_t tops[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int me = WAVES == 1 ? lane : tid;
  const int64_t row = WAVES == 1 ? (int64_t)blockIdx.x * 4 + wave : blockIdx.x;
  if (row >= rows) return;  // (whole wavefronts, or the whole workgroup)
  const T* from = x + row * ldx;
  int8_t* to = codes + row * ldc;
  const int pieces = (k + EPC - 1) / EPC;
  float v[ONCE ? HELD : 1][EPC];
  uint32_t top = 0;
  if constexpr (ONCE) {
#pragma unroll
    for (int h = 0; h < HELD; ++h) piece_of(from + (int64_t)(me + h * SPAN) * EPC, k - (me + h * SPAN) * EPC, v[h]);
#pragma unroll
    for (int h = 0; h < HELD; ++h)
#pragma unroll
      for (int i = 0; i < EPC; ++i) top = max(top, __float_as_uint(v[h][i]) & 0x7fffffffu);
  } else {
    for (int c = me; c < pieces; c += SPAN) {
      piece_of(from + (int64_t)c * EPC, k - c * EPC, v[0]);
#pragma unroll
      for (int i = 0; i < EPC; ++i) top = max(top, __float_as_uint(v[0][i]) & 0x7fffffffu);
    }
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
  if constexpr (WAVES > 1) {
    if (lane == 0) tops[wave] = top;
    __syncthreads();
    top = max(max(tops[0], tops[1]), max(tops[2], tops[3]));
  }
  const RowScale r = row_scale(top);
  if (me == 0) scale[row] = r.bad ? __uint_as_float(0x7fc00000u) : r.scale;
  if constexpr (ONCE) {
#pragma unroll
    for (int h = 0; h < HELD; ++h) {
      const int c = me + h * SPAN;
      if (c < pieces) store_codes<EPC>(v[h], r, k - c * EPC, to + (int64_t)c * EPC);
    }
  } else {
    for (int c = me; c < pieces; c += SPAN) {
      piece_of(from + (int64_t)c * EPC, k - c * EPC, v[0]);
      store_codes<EPC>(v[0], r, k - c * EPC, to + (int64_t)c * EPC);
    }
  }
}

template <class T>
static int launch_typed(const T* x, int64_t ldx, int64_t rows, int k, int8_t* codes, int64_t ldc, float* scale, hipStream_t st) {
  constexpr int EPC = 16 / sizeof(T);
  // a wavefront per row while its registers hold the row: no barrier, four rows per workgroup
  const bool wave = k <= 64 * HELD * EPC, once = k <= 256 * HELD * EPC;
  // (a launch takes 2^24 - 1 workgroups of 256 threads, so many rows are several launches)
  const int64_t most = MAX_GRID / 256 * (wave ? 4 : 1);
  for (int64_t first = 0; first < rows; first += most) {
    const int64_t here = std::min(most, rows - first);
    const unsigned grid = (unsigned)(wave ? (here + 3) / 4 : here);
    const T* from = x + first * ldx;
    int8_t* to = codes + first * ldc;
    if (wave) quantize_rows_kernel<T, 1, true><<<grid, 256, 0, st>>>(from, ldx, here, k, to, ldc, scale + first);
    else if (once) quantize_rows_kernel<T, 4, true><<<grid, 256, 0, st>>>(from, ldx, here, k, to, ldc, scale + first);
    else quantize_rows_kernel<T, 4, false><<<grid, 256, 0, st>>>(from, ldx, here, k, to, ldc, scale + first);
    RQ_HIP(hipGetLastError());
  }
  return RABITQ_OK;
}

int launch_quantize_rows(const void* x, int dtype, int64_t ldx, int64_t rows, int k, int8_t* codes, int64_t ldc, float* scale,
                         hipStream_t st) {
  if (dtype == RABITQ_F32) return launch_typed(static_cast<const float*>(x), ldx, rows, k, codes, ldc, scale, st);
  if (dtype == RABITQ_F16) return launch_typed(static_cast<const _Float16*>(x), ldx, rows, k, codes, ldc, scale, st);
  return launch_typed(static_cast<const __bf16*>(x), ldx, rows, k, codes, ldc, scale, st);
}

}  // namespace rq
