// C ABI of the products by list and of the 8-bit integer products: argument checks, then the launchers.
#include <new>

#include "rq_products.h"

using namespace rq;

namespace {

constexpr int64_t MAX_WIDTH = 1 << 20;
constexpr int64_t MAX_K_I8 = 131071;       // 128 x 128 x k must stay below 2^31
constexpr int32_t MAX_LISTS = 1 << 24;
constexpr int64_t MAX_LD = (int64_t)1 << 40;

int bad(const char* call, const char* what) {
  set_error(std::string(call) + ": " + what);
  return RABITQ_EINVAL;
}

// No exception leaves a C entry point (the text of an error is a std::string).
template <class Body>
int guarded(Body&& body) noexcept {
  try {
    return body();
  } catch (...) {
    return RABITQ_ENOMEM;
  }
}

bool dtype_ok(int32_t t) { return t == RABITQ_F32 || t == RABITQ_F16 || t == RABITQ_BF16; }
bool ld_ok(int64_t ld, int64_t width) { return ld >= width && ld <= MAX_LD; }
bool aligned(const void* p, int64_t to) { return reinterpret_cast<uintptr_t>(p) % (uintptr_t)to == 0; }
bool stride_ok(const rabitq_lists* l, int64_t ldw, int64_t stride) {
  return l->groups == 1 || (stride >= (l->n - 1) * ldw + l->k && stride <= MAX_LD);
}

int check_lists(const char* call, const rabitq_lists* l) {
  if (!l) return bad(call, "null pointer");
  if (l->groups < 1 || l->groups > MAX_LISTS) return bad(call, "groups must lie in 1 .. 2^24");
  if (l->nprobe < 1) return bad(call, "nprobe must be at least 1");
  if (l->pairs < 0 || l->pairs > 0x7fffffff) return bad(call, "pairs must lie in 0 .. 2^31 - 1");
  if (l->pairs % l->nprobe != 0) return bad(call, "pairs must be a multiple of nprobe");
  if (l->n < 1 || l->n > MAX_WIDTH || l->k < 1 || l->k > MAX_WIDTH) return bad(call, "n and k must lie in 1 .. 2^20");
  if (!l->pair_off) return bad(call, "null pointer");
  if (!aligned(l->pair_off, 4) || !aligned(l->pair_ids, 4)) return bad(call, "pointer not aligned to its type");
  return RABITQ_OK;
}

ProductArgs args_of(const rabitq_lists* l) {
  ProductArgs p{};
  p.pair_off = l->pair_off; p.pair_ids = l->pair_ids; p.pairs = l->pairs; p.n = l->n; p.k = l->k;
  p.groups = l->groups; p.probe = divisor(l->nprobe);
  return p;
}

int64_t named_bytes(int64_t pairs) { return (pairs + 15) / 16 * 16; }

}  // namespace

extern "C" {

int rabitq_grouped_matmul(const rabitq_lists* l, int32_t dtype, const void* x, int64_t ldx, const void* w, int64_t ldw,
                          int64_t stride_w, void* out, int64_t ldo, void* stream) {
  return guarded([&]() -> int {
    const char* call = "grouped_matmul";
    const int rc = check_lists(call, l);
    if (rc) return rc;
    if (!dtype_ok(dtype)) return bad(call, "unknown type");
    if (!ld_ok(ldx, l->k) || !ld_ok(ldw, l->k) || !ld_ok(ldo, l->n) || !stride_ok(l, ldw, stride_w)) return bad(call, "stride out of range");
    if (l->pairs == 0) return RABITQ_OK;
    if (!x || !w || !out) return bad(call, "null pointer");
    const int64_t sz = dtype_bytes(dtype);
    if (!aligned(x, sz) || !aligned(w, sz) || !aligned(out, sz)) return bad(call, "pointer not aligned to its type");
    ProductArgs p = args_of(l);
    p.a = x; p.lda = ldx; p.rows_a = l->pairs / l->nprobe; p.b = w; p.ldb = ldw; p.stride = stride_w; p.out = out; p.ldo = ldo; p.out_dtype = dtype;
    return launch_product_forward(p, dtype, (hipStream_t)stream);
  });
}

int64_t rabitq_grouped_dx_scratch_bytes(const rabitq_lists* l) {
  return guarded([&]() -> int {
           return check_lists("grouped_dx_scratch_bytes", l);
         }) != RABITQ_OK
             ? (int64_t)RABITQ_EINVAL
             : l->nprobe == 1 ? 0 : named_bytes(l->pairs) + l->pairs * l->k * 4;
}

int rabitq_grouped_matmul_dx(const rabitq_lists* l, int32_t dtype, const void* dout, int64_t ldd, const void* w, int64_t ldw,
                             int64_t stride_w, void* dx, int64_t ldx, void* scratch, void* stream) {
  return guarded([&]() -> int {
    const char* call = "grouped_matmul_dx";
    int rc = check_lists(call, l);
    if (rc) return rc;
    if (!dtype_ok(dtype)) return bad(call, "unknown type");
    if (!ld_ok(ldd, l->n) || !ld_ok(ldw, l->k) || !ld_ok(ldx, l->k) || !stride_ok(l, ldw, stride_w)) return bad(call, "stride out of range");
    if (l->pairs == 0) return RABITQ_OK;
    if (!dout || !w || !dx || (l->nprobe > 1 && !scratch)) return bad(call, "null pointer");
    const int64_t sz = dtype_bytes(dtype);
    if (!aligned(dout, sz) || !aligned(w, sz) || !aligned(dx, sz) || !aligned(scratch, 16)) return bad(call, "pointer not aligned to its type");
    hipStream_t st = (hipStream_t)stream;
    ProductArgs p = args_of(l);
    p.a = dout; p.lda = ldd; p.rows_a = l->pairs; p.b = w; p.ldb = ldw; p.stride = stride_w;
    if (l->nprobe == 1) {
      p.out = dx; p.ldo = ldx; p.out_dtype = dtype;
      return launch_product_dx(p, dtype, st);
    }
    // every pair's own row in fp32, and the sum over a query's pairs behind it
    p.named = static_cast<uint8_t*>(scratch);
    float* parts = reinterpret_cast<float*>(p.named + named_bytes(l->pairs));
    p.out = parts; p.ldo = l->k; p.out_dtype = RABITQ_F32;
    p.check_only = true;  // (nothing is written by a call that is refused)
    if ((rc = launch_product_dx(p, dtype, st))) return rc;
    p.check_only = false;
    if ((rc = launch_clear_bytes(p.named, l->pairs, st))) return rc;
    if ((rc = launch_product_dx(p, dtype, st))) return rc;
    return launch_sum_named(parts, p.named, l->pairs / l->nprobe, l->nprobe, l->k, dx, dtype, ldx, st);
  });
}

int64_t rabitq_grouped_dw_scratch_bytes(const rabitq_lists* l) {
  const int rc = guarded([&]() -> int { return check_lists("grouped_dw_scratch_bytes", l); });
  if (rc) return rc;
  const int part = dw_part(l->pairs, l->groups, l->n, l->k);
  return part == 0 ? 0 : dw_parts(l->pairs, l->groups, part) * l->n * l->k * 4;
}

int rabitq_grouped_matmul_dw(const rabitq_lists* l, int32_t dtype, const void* dout, int64_t ldd, const void* x, int64_t ldx,
                             void* dw, int64_t ldw, int64_t stride_w, void* scratch, void* stream) {
  return guarded([&]() -> int {
    const char* call = "grouped_matmul_dw";
    const int rc = check_lists(call, l);
    if (rc) return rc;
    if (!dtype_ok(dtype)) return bad(call, "unknown type");
    if (!ld_ok(ldd, l->n) || !ld_ok(ldx, l->k) || !ld_ok(ldw, l->k) || !stride_ok(l, ldw, stride_w)) return bad(call, "stride out of range");
    const bool in_parts = dw_part(l->pairs, l->groups, l->n, l->k) != 0;
    if (!dw || (l->pairs > 0 && (!dout || !x)) || (in_parts && !scratch)) return bad(call, "null pointer");
    const int64_t sz = dtype_bytes(dtype);
    if (!aligned(dout, sz) || !aligned(x, sz) || !aligned(dw, sz) || !aligned(scratch, 16)) return bad(call, "pointer not aligned to its type");
    ProductArgs p = args_of(l);
    p.a = dout; p.lda = ldd; p.rows_a = l->pairs; p.b = x; p.ldb = ldx; p.out = dw; p.ldo = ldw; p.stride = stride_w; p.out_dtype = dtype;
    return launch_product_dw(p, dtype, static_cast<float*>(scratch), (hipStream_t)stream);
  });
}

int rabitq_quantize_rows(const void* x, int32_t dtype, int64_t ldx, int64_t rows, int32_t k, int8_t* codes, int64_t ldc,
                         float* scale, void* stream) {
  return guarded([&]() -> int {
    const char* call = "quantize_rows";
    if (!dtype_ok(dtype)) return bad(call, "unknown type");
    if (rows < 0 || k < 1 || k > MAX_WIDTH) return bad(call, "rows must be at least 0 and k in 1 .. 2^20");
    if (rows > 0x7fffffff) return bad(call, "too many rows");
    if (!ld_ok(ldx, k) || !ld_ok(ldc, k)) return bad(call, "stride out of range");
    if (rows == 0) return RABITQ_OK;
    if (!x || !codes || !scale) return bad(call, "null pointer");
    if (!aligned(x, dtype_bytes(dtype)) || !aligned(scale, 4)) return bad(call, "pointer not aligned to its type");
    return launch_quantize_rows(x, dtype, ldx, rows, k, codes, ldc, scale, (hipStream_t)stream);
  });
}

int rabitq_matmul_i8(const int8_t* a, int64_t lda, const float* scale_a, const int8_t* b, int64_t ldb, const float* scale_b,
                     int64_t m, int64_t n, int32_t k, void* out, int32_t out_dtype, int64_t ldo, void* stream) {
  return guarded([&]() -> int {
    const char* call = "matmul_i8";
    if (!dtype_ok(out_dtype)) return bad(call, "unknown type");
    if (m < 0 || n < 0 || m > 0x7fffffff || n > 0x7fffffff) return bad(call, "m and n must lie in 0 .. 2^31 - 1");
    if (k < 1 || k > MAX_K_I8) return bad(call, "k must lie in 1 .. 131071");
    if (!ld_ok(lda, k) || !ld_ok(ldb, k) || !ld_ok(ldo, n)) return bad(call, "stride out of range");
    if (m == 0 || n == 0) return RABITQ_OK;
    if (!a || !b || !scale_a || !scale_b || !out) return bad(call, "null pointer");
    if (!aligned(scale_a, 4) || !aligned(scale_b, 4) || !aligned(out, dtype_bytes(out_dtype))) return bad(call, "pointer not aligned to its type");
    ProductArgs p{};
    p.a = a; p.lda = lda; p.rows_a = m; p.b = b; p.ldb = ldb; p.scale_a = scale_a; p.scale_b = scale_b;
    p.pairs = m; p.n = n; p.k = k; p.groups = 1; p.probe = divisor(1); p.out = out; p.ldo = ldo; p.out_dtype = out_dtype;
    return launch_product_forward(p, DTYPE_I8, (hipStream_t)stream);
  });
}

int rabitq_grouped_matmul_i8(const rabitq_lists* l, const int8_t* x, int64_t ldx, const float* scale_x, const int8_t* w,
                             int64_t ldw, int64_t stride_w, const float* scale_w, void* out, int32_t out_dtype, int64_t ldo,
                             void* stream) {
  return guarded([&]() -> int {
    const char* call = "grouped_matmul_i8";
    const int rc = check_lists(call, l);
    if (rc) return rc;
    if (!dtype_ok(out_dtype)) return bad(call, "unknown type");
    if (l->k > MAX_K_I8) return bad(call, "k must lie in 1 .. 131071");
    if (!ld_ok(ldx, l->k) || !ld_ok(ldw, l->k) || !ld_ok(ldo, l->n) || !stride_ok(l, ldw, stride_w)) return bad(call, "stride out of range");
    if (l->pairs == 0) return RABITQ_OK;
    if (!x || !w || !scale_x || !scale_w || !out) return bad(call, "null pointer");
    if (!aligned(scale_x, 4) || !aligned(scale_w, 4) || !aligned(out, dtype_bytes(out_dtype))) return bad(call, "pointer not aligned to its type");
    ProductArgs p = args_of(l);
    p.a = x; p.lda = ldx; p.rows_a = l->pairs / l->nprobe; p.b = w; p.ldb = ldw; p.stride = stride_w; p.scale_a = scale_x; p.scale_b = scale_w;
    p.out = out; p.ldo = ldo; p.out_dtype = out_dtype;
    return launch_product_forward(p, DTYPE_I8, (hipStream_t)stream);
  });
}

}  // extern "C"
