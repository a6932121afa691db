// Products by list (forward, gradient of the inputs, gradient of the matrices) and products of int8 codes with scales.
#include "rq_products.h"

namespace rq {

constexpr int TB = 64, KB = 16;  // tile of the output, contraction per step

enum { FORWARD = 0, GRAD_X = 1, GRAD_W = 2 };

template <class T>
struct AccOf { using type = float; };
template <>
struct AccOf<int8_t> { using type = int; };
__device__ __forceinline__ float operand(float v) { return v; }
__device__ __forceinline__ float operand(_Float16 v) { return (float)v; }
__device__ __forceinline__ float operand(__bf16 v) { return (float)v; }
__device__ __forceinline__ int operand(int8_t v) { return v; }

template <class T, int OP>
__global__ __launch_bounds__(256) void product_kernel(ProductArgs p) {
  using Acc = typename AccOf<T>::type;
  __shared__ Acc As[KB][TB + 1], Bs[KB][TB + 1];
  __shared__ int64_t row_a[TB], row_out[TB];
  const int tid = threadIdx.x, lane = tid & 63;
  const T* a = static_cast<const T*>(p.a);
  const T* b = static_cast<const T*>(p.b);
  int g;
  Span s;
  const int jt = (int)(((OP == FORWARD ? p.n : p.k) + TB - 1) / TB);
  const int64_t tile = blockIdx.x / jt;
  int64_t i0, j0 = (int64_t)(blockIdx.x % jt) * TB, ni, nj, nc;
  if (OP == GRAD_W) {
    const int64_t it = (p.n + TB - 1) / TB;
    g = (int)(tile / it);
    s = span_of(p, g);
    i0 = tile % it * TB;
    ni = p.n; nj = p.k; nc = s.end - s.begin;
  } else {
    g = p.pair_off ? list_of_tile(p, tile, TB, lane) : 0;
    s = span_of(p, g);
    const int64_t first = p.pair_off ? s.begin / TB + g : 0;
    i0 = s.begin + (tile - first) * TB;
    if (i0 < s.begin || i0 >= s.end) return;
    ni = s.end; nj = OP == FORWARD ? p.n : p.k; nc = OP == FORWARD ? p.k : p.n;
    for (int i = tid; i < TB; i += 256) {
      const int64_t pr = i0 + i < s.end ? pair_at(p, i0 + i) : -1;
      row_out[i] = pr;
      row_a[i] = pr < 0 ? -1 : OP == FORWARD ? pr / p.nprobe : pr;
    }
    __syncthreads();
    b += (int64_t)g * p.stride;
  }
  Acc acc[4][4] = {};
  const int ti = tid / 16, tj = tid % 16;
  for (int64_t c0 = 0; c0 < nc; c0 += KB) {
    for (int e = tid; e < TB * KB; e += 256) {
      if (OP == GRAD_W) {
        const int i = e % TB, c = e / TB;
        const int64_t pr = c0 + c < nc ? pair_at(p, s.begin + c0 + c) : -1;
        As[c][i] = pr >= 0 && i0 + i < ni ? operand(a[pr * p.lda + i0 + i]) : Acc(0);
        Bs[c][i] = pr >= 0 && j0 + i < nj ? operand(b[pr / p.nprobe * p.ldb + j0 + i]) : Acc(0);
      } else {
        const int c = e % KB, i = e / KB;
        As[c][i] = c0 + c < nc && row_a[i] >= 0 ? operand(a[row_a[i] * p.lda + c0 + c]) : Acc(0);
        if (OP == FORWARD) {
          Bs[c][i] = c0 + c < nc && j0 + i < nj ? operand(b[(j0 + i) * p.ldb + c0 + c]) : Acc(0);
        } else {
          const int j = e % TB, cc = e / TB;
          Bs[cc][j] = c0 + cc < nc && j0 + j < nj ? operand(b[(c0 + cc) * p.ldb + j0 + j]) : Acc(0);
        }
      }
    }
    __syncthreads();
    for (int c = 0; c < KB; ++c)
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int v = 0; v < 4; ++v) acc[u][v] += As[c][ti * 4 + u] * Bs[c][tj + 16 * v];
    __syncthreads();
  }
  for (int u = 0; u < 4; ++u) {
    const int i = ti * 4 + u;
    const int64_t ro = OP == GRAD_W ? (i0 + i < ni ? i0 + i : -1) : row_out[i];
    if (ro < 0) continue;
    if (OP == GRAD_X && p.named && j0 == 0 && tj == 0) p.named[ro] = 1;
    for (int v = 0; v < 4; ++v) {
      const int64_t j = j0 + tj + 16 * v;
      if (j >= nj) continue;
      float r = (float)acc[u][v];
      if (sizeof(T) == 1) r = r * p.scale_a[row_a[i]] * p.scale_b[(int64_t)g * p.n + j];
      store_as(p.out, p.out_dtype, (OP == GRAD_W ? (int64_t)g * p.stride : 0) + ro * p.ldo + j, r);
    }
  }
}

__global__ __launch_bounds__(256) void clear_bytes_kernel(uint8_t* at, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) at[i] = 0;
}

// dx of several probes: the named pairs' rows in ascending order of the pair.
template <class T>
__global__ __launch_bounds__(256) void sum_named_kernel(const float* __restrict__ parts, const uint8_t* __restrict__ named, int64_t rows,
                                                        int nprobe, int k, T* __restrict__ out, int64_t ldo) {
  for (int64_t q = blockIdx.x; q < rows; q += gridDim.x) {
    for (int j = threadIdx.x; j < k; j += 256) {
      float sum = 0.f;
      bool any = false;
      for (int r = 0; r < nprobe; ++r) {
        const int64_t pr = q * nprobe + r;
        if (named[pr]) { sum += parts[pr * k + j]; any = true; }
      }
      if (any) out[q * ldo + j] = (T)sum;
    }
  }
}

template <class T>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const T* __restrict__ x, int64_t ldx, int64_t rows, int k,
                                                            int8_t* __restrict__ codes, int64_t ldc, float* __restrict__ scale) {
  __shared__ uint32_t top_s[4];
  const int tid = threadIdx.x;
  for (int64_t i = blockIdx.x; i < rows; i += gridDim.x) {
    uint32_t top = 0;  // |x| as bits: they order as the values do, infinity and NaN above all numbers
    for (int j = tid; j < k; j += 256) top = max(top, __float_as_uint(to_f32(x[i * ldx + j])) & 0x7fffffffu);
    for (int o = 32; o; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
    if ((tid & 63) == 0) top_s[tid >> 6] = top;
    __syncthreads();
    top = max(max(top_s[0], top_s[1]), max(top_s[2], top_s[3]));
    __syncthreads();
    const bool bad = top >= 0x7f800000u;
    float sc = __uint_as_float(top) / 127.0f;
    if (sc == 0.f) sc = 1.0f;
    for (int j = tid; j < k; j += 256)
      codes[i * ldc + j] = bad ? 0 : (int8_t)(int)rint((double)to_f32(x[i * ldx + j]) / (double)sc);
    if (tid == 0) scale[i] = bad ? __uint_as_float(0x7fc00000u) : sc;
  }
}

template <int OP>
static int launch_op(const ProductArgs& p, int dtype, int64_t tiles, hipStream_t st) {
  if (tiles > MAX_TILES) {
    set_error("too many tiles of work");
    return RABITQ_EINVAL;
  }
  const unsigned grid = (unsigned)tiles;
  switch (dtype) {
    case RABITQ_F32: product_kernel<float, OP><<<grid, 256, 0, st>>>(p); break;
    case RABITQ_F16: product_kernel<_Float16, OP><<<grid, 256, 0, st>>>(p); break;
    case RABITQ_BF16: product_kernel<__bf16, OP><<<grid, 256, 0, st>>>(p); break;
    default: if constexpr (OP == FORWARD) product_kernel<int8_t, OP><<<grid, 256, 0, st>>>(p);
  }
  RQ_HIP(hipGetLastError());
  return RABITQ_OK;
}

static int64_t up(int64_t v, int64_t by) { return (v + by - 1) / by; }

int launch_product_forward(const ProductArgs& p, int dtype, hipStream_t st) {
  return launch_op<FORWARD>(p, dtype, (p.pairs / TB + p.groups) * up(p.n, TB), st);
}
int launch_product_dx(const ProductArgs& p, int dtype, hipStream_t st) {
  return launch_op<GRAD_X>(p, dtype, (p.pairs / TB + p.groups) * up(p.k, TB), st);
}
int launch_product_dw(const ProductArgs& p, int dtype, hipStream_t st) {
  return launch_op<GRAD_W>(p, dtype, up(p.n, TB) * up(p.k, TB) * p.groups, st);
}

int launch_clear_bytes(void* at, int64_t n, hipStream_t st) {
  clear_bytes_kernel<<<(unsigned)std::min<int64_t>((n + 255) / 256, 4096), 256, 0, st>>>(static_cast<uint8_t*>(at), n);
  RQ_HIP(hipGetLastError());
  return RABITQ_OK;
}

int launch_sum_named(const float* parts, const uint8_t* named, int64_t rows, int nprobe, int k, void* out, int dtype, int64_t ldo,
                     hipStream_t st) {
  const unsigned grid = (unsigned)std::min<int64_t>(rows, 65536);
  if (dtype == RABITQ_F32) sum_named_kernel<<<grid, 256, 0, st>>>(parts, named, rows, nprobe, k, (float*)out, ldo);
  else if (dtype == RABITQ_F16) sum_named_kernel<<<grid, 256, 0, st>>>(parts, named, rows, nprobe, k, (_Float16*)out, ldo);
  else sum_named_kernel<<<grid, 256, 0, st>>>(parts, named, rows, nprobe, k, (__bf16*)out, ldo);
  RQ_HIP(hipGetLastError());
  return RABITQ_OK;
}

int launch_quantize_rows(const void* x, int dtype, int64_t ldx, int64_t rows, int k, int8_t* codes, int64_t ldc, float* scale,
                         hipStream_t st) {
  const unsigned grid = (unsigned)std::min<int64_t>(rows, 65536);
  if (dtype == RABITQ_F32) quantize_rows_kernel<<<grid, 256, 0, st>>>((const float*)x, ldx, rows, k, codes, ldc, scale);
  else if (dtype == RABITQ_F16) quantize_rows_kernel<<<grid, 256, 0, st>>>((const _Float16*)x, ldx, rows, k, codes, ldc, scale);
  else quantize_rows_kernel<<<grid, 256, 0, st>>>((const __bf16*)x, ldx, rows, k, codes, ldc, scale);
  RQ_HIP(hipGetLastError());
  return RABITQ_OK;
}

}  // namespace rq
