// Products by list (forward, gradient of the inputs, gradient of the matrices) and products of int8 codes with scales.
#include "rq_product_tile.h"

namespace rq {

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

static int64_t up(int64_t v, int64_t by) { return (v + by - 1) / by; }

template <class T, int OP, int BI, int BJ, int WI, int WJ, bool FAST>
static int launch_tiles(ProductArgs p, hipStream_t st) {
  const int64_t width = OP == FORWARD ? p.n : p.k;
  p.chunk = std::max<int64_t>(1, up(width, BJ) / 8);
  p.tiles = up(width, BJ) * (OP == GRAD_W ? up(p.n, BI) * p.groups : p.pair_off ? p.pairs / BI + p.groups : up(p.pairs, BI));
  const int64_t grid = up(p.tiles, 8 * p.chunk) * 8 * p.chunk;
  if (grid > MAX_GRID / (64 * WI * WJ)) {
    set_error("too many tiles of work");
    return RABITQ_EINVAL;
  }
  const size_t lds = 2 * (BI + BJ) * 128 + BI * sizeof(int);
  auto kernel = product_tile_kernel<T, OP, BI, BJ, WI, WJ, FAST>;
  static const hipError_t granted =
      hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  RQ_HIP(granted);
  kernel<<<(unsigned)grid, 64 * WI * WJ, lds, st>>>(p);
  RQ_HIP(hipGetLastError());
  return RABITQ_OK;
}

// Rows of whole 16-byte pieces at multiples of 16 bytes: the pieces can go to LDS without registers.
static bool fast_rows(const ProductArgs& p, int op, int dtype) {
  const int64_t sz = dtype_bytes(dtype), per = 16 / sz;
  const int64_t in_a = op == FORWARD ? p.k : p.n;  // elements of a row of each operand
  return in_a % per == 0 && p.k % per == 0 && p.lda % per == 0 && p.ldb % per == 0 && (op == GRAD_W || p.stride % per == 0 || p.groups == 1) &&
         reinterpret_cast<uintptr_t>(p.a) % 16 == 0 && reinterpret_cast<uintptr_t>(p.b) % 16 == 0;
}

template <class T, int OP>
static int launch_typed(const ProductArgs& p, int dtype, hipStream_t st) {
  if (!fast_rows(p, OP, dtype)) return launch_tiles<T, OP, 128, 128, 2, 2, false>(p, st);
  const int64_t width = OP == FORWARD ? p.n : p.k;
  const int64_t big = up(width, 256) * (OP == GRAD_W ? up(p.n, 256) * p.groups : p.pairs / 256 + p.groups);
  if (big >= 512) return launch_tiles<T, OP, 256, 256, 2, 4, true>(p, st);
  return launch_tiles<T, OP, 128, 128, 2, 2, true>(p, st);
}

template <int OP>
static int launch_op(const ProductArgs& p, int dtype, hipStream_t st) {
  switch (dtype) {
    case RABITQ_F32: return launch_typed<float, OP>(p, dtype, st);
    case RABITQ_F16: return launch_typed<_Float16, OP>(p, dtype, st);
    case RABITQ_BF16: return launch_typed<__bf16, OP>(p, dtype, st);
  }
  if constexpr (OP == FORWARD) return launch_typed<int8_t, OP>(p, dtype, st);
  return RABITQ_EINVAL;
}

int launch_product_forward(const ProductArgs& p, int dtype, hipStream_t st) { return launch_op<FORWARD>(p, dtype, st); }
int launch_product_dx(const ProductArgs& p, int dtype, hipStream_t st) { return launch_op<GRAD_X>(p, dtype, st); }
int launch_product_dw(const ProductArgs& p, int dtype, hipStream_t st) { return launch_op<GRAD_W>(p, dtype, st); }

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
