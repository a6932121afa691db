// Products by list and products of 8-bit integers: what the launchers take, and how a kernel finds its rows.
#pragma once
#include "rq_device.h"

namespace rq {

constexpr int DTYPE_I8 = 3;  // operands only; behind the rabitq_dtype values
constexpr int64_t MAX_GRID = 0xffffffff;  // threads of a launch
inline int64_t dtype_bytes(int dtype) { return dtype == RABITQ_F32 ? 4 : dtype == DTYPE_I8 ? 1 : 2; }

// x / d for 0 <= x < 2^31, by a multiplication: with 2^(s - 1) < d <= 2^s and m = floor(2^(31 + s) / d) + 1, x m / 2^(31 + s) exceeds
// x / d by less than x / 2^(31 + s) <= 2^-s <= 1 / d, which no next whole number is nearer than.
struct Divisor {
  uint32_t m;
  int shift;
  __device__ __forceinline__ int of(int x) const { return (int)(((uint64_t)(uint32_t)x * m) >> shift); }
};
inline Divisor divisor(int d) {
  int s = 0;
  while (((int64_t)1 << s) < d) ++s;
  return Divisor{(uint32_t)(((uint64_t)1 << (31 + s)) / (uint64_t)d + 1), 31 + s};
}

// One product, whichever direction.  `a` has a row per pair or per row of x, `b` is the matrices (forward and dx) or x (dw).
struct ProductArgs {
  const void* a;
  const void* b;
  void* out;
  int64_t lda, ldb, ldo;
  int64_t rows_a;
  int64_t stride;             // between the matrices of two lists, in b or (dw) in out
  const float* scale_a;       // codes only: one per row of a, one per row of b ([groups][n])
  const float* scale_b;
  const int32_t* pair_off;    // null: one list of all positions
  const int32_t* pair_ids;    // null: position i is pair i
  int64_t pairs;
  int64_t n;
  int k, groups;
  Divisor probe;              // by the pairs per row of x
  int out_dtype;
  bool check_only;            // say whether the launch would be refused, and launch nothing
  int64_t tiles_i;            // of the launch, along the rows
  uint32_t strip, strips;     // neighbouring tiles of a row of tiles that go to one XCD, and how many such strips a row has
  int part;                   // dw: positions of a list that one workgroup sums up, or 0 (all)
  float* parts;               // dw: [parts][n][k], the sums of lists of several parts
  uint8_t* named;             // dx of several probes: set to 1 for every pair a list names, or null
};

// Positions of a list, within 0 .. pairs whatever the offsets hold.
struct Span {
  int64_t begin, end;
};
__device__ __forceinline__ int64_t clamp_off(const ProductArgs& p, int g) {
  const int64_t o = p.pair_off[g];
  return o < 0 ? 0 : o > p.pairs ? p.pairs : o;
}
__device__ __forceinline__ Span span_of(const ProductArgs& p, int g) {
  if (p.pair_off == nullptr) return Span{0, p.pairs};
  return Span{clamp_off(p, g), clamp_off(p, g + 1)};
}
// The pair at a position, or -1.
__device__ __forceinline__ int64_t pair_at(const ProductArgs& p, int64_t pos) {
  if (p.pair_ids == nullptr) return pos;
  const int64_t i = p.pair_ids[pos];
  return (uint64_t)i < (uint64_t)p.pairs ? i : -1;
}

// Tiles of `rows` positions are numbered so that list g owns those from F(g) = off[g] / rows + g on: F grows by at least the
// ceil(length / rows) tiles that the list needs, so no table of tiles has to be made, pairs / rows + groups tiles are enough, and
// the list of a tile is the last g with F(g) <= tile.  Searched 64 ways at a time, one offset per lane (a level reads one line or
// 64 scattered words; 2 levels to 4096 lists).
__device__ __forceinline__ int list_of_tile(const ProductArgs& p, int64_t tile, int rows, int lane) {
  int lo = 0, len = p.groups;  // the answer lies in lo .. lo + len - 1
  while (len > 1) {
    const int step = (len + 63) / 64;
    const int g = lo + lane * step;
    const bool below = lane * step < len && clamp_off(p, g) / rows + g <= tile;
    const int c = __popcll(__ballot(below));  // F ascends, so these are the first c lanes (at least one if lo holds)
    const int at = c > 0 ? (c - 1) * step : 0;
    lo += at;
    len = min(step, len - at);
  }
  return lo;
}

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(_Float16 v) { return (float)v; }
__device__ __forceinline__ float to_f32(__bf16 v) { return (float)v; }

__device__ __forceinline__ void store_as(void* out, int dtype, int64_t at, float v) {
  if (dtype == RABITQ_F32) static_cast<float*>(out)[at] = v;
  else if (dtype == RABITQ_F16) static_cast<_Float16*>(out)[at] = (_Float16)v;
  else static_cast<__bf16*>(out)[at] = (__bf16)v;
}

// dtype: of the operands.  All sizes and pointers checked by the caller, work to do.
int launch_product_forward(const ProductArgs& p, int dtype, hipStream_t st);
int launch_product_dx(const ProductArgs& p, int dtype, hipStream_t st);
// dw.  Where there are few tiles of dw, a list is summed up in parts of dw_part(...) positions (0: not in parts), numbered as tiles are;
// the sums of lists of several parts go to scratch and are added up in order.
int dw_part(int64_t pairs, int groups, int64_t n, int64_t k);
inline int64_t dw_parts(int64_t pairs, int groups, int part) { return pairs / part + groups; }
int launch_product_dw(const ProductArgs& p, int dtype, float* scratch, hipStream_t st);
int launch_clear_bytes(void* at, int64_t n, hipStream_t st);
int launch_sum_named(const float* parts, const uint8_t* named, int64_t rows, int nprobe, int k, void* out, int dtype, int64_t ldo,
                     hipStream_t st);
int launch_quantize_rows(const void* x, int dtype, int64_t ldx, int64_t rows, int k, int8_t* codes, int64_t ldc, float* scale,
                         hipStream_t st);

}  // namespace rq
