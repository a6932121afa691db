// Products by list (forward, gradient of the inputs, gradient of the matrices) and products of int8 codes with scales.
#include "rq_product_few.h"

namespace rq {

__global__ __launch_bounds__(256) void clear_bytes_kernel(uint8_t* at, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) at[i] = 0;
}

// dw in parts: the sums of the parts of a list that has several, in ascending order; zeros for a list without positions.
template <class T>
__global__ __launch_bounds__(256) void sum_parts_kernel(ProductArgs p, T* __restrict__ out) {
  const int64_t elems = p.n * p.k;
  for (int g = blockIdx.y; g < p.groups; g += gridDim.y) {
    const Span s = span_of(p, g);
    const int64_t first = s.begin / p.part + g, count = s.end > s.begin ? (s.end - s.begin + p.part - 1) / p.part : 0;
    if (count == 1) continue;
    for (int64_t e0 = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; e0 < elems; e0 += (int64_t)gridDim.x * 1024) {
      const int here = (int)(elems - e0 < 4 ? elems - e0 : 4);
      float sum[4] = {0.f, 0.f, 0.f, 0.f};
      for (int64_t c = 0; c < count; ++c) {
        const float* from = p.parts + (first + c) * elems + e0;
        if (here == 4) {
          float v[4];
          __builtin_memcpy(v, from, 16);
#pragma unroll
          for (int e = 0; e < 4; ++e) sum[e] += v[e];
        } else {
          for (int e = 0; e < here; ++e) sum[e] += from[e];
        }
      }
      int64_t row = e0 / p.k, col = e0 % p.k;
      T* to = out + (int64_t)g * p.stride + row * p.ldo + col;
      if (col + 4 <= p.k) {
        const T v[4] = {(T)sum[0], (T)sum[1], (T)sum[2], (T)sum[3]};
        __builtin_memcpy(to, v, sizeof(v));  // (at any alignment of the element)
      } else {
        for (int e = 0; e < here; ++e) {
          out[(int64_t)g * p.stride + row * p.ldo + col] = (T)sum[e];
          if (++col == p.k) { col = 0; ++row; }
        }
      }
    }
  }
}

// dx of several probes: the named pairs' rows in ascending order of the pair.  A thread takes 4 neighbouring columns of a query.
template <class T>
__global__ __launch_bounds__(256) void sum_named_kernel(const float* __restrict__ parts, const uint8_t* __restrict__ named, int64_t rows,
                                                        int nprobe, int k, T* __restrict__ out, int64_t ldo) {
  const int per_row = (k + 3) / 4;
  const int64_t all = rows * per_row;
  for (int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x; id < all; id += (int64_t)gridDim.x * 256) {
    const int64_t q = id / per_row;
    const int j = (int)(id - q * per_row) * 4, here = min(4, k - j);
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    bool any = false;
    for (int r = 0; r < nprobe; ++r) {
      const int64_t pr = q * nprobe + r;
      if (!named[pr]) continue;
      any = true;
      const float* from = parts + pr * k + j;
      if (here == 4) {
        float v[4];
        __builtin_memcpy(v, from, 16);  // (at any alignment of the element, as below)
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] += v[e];
      } else {
        for (int e = 0; e < here; ++e) sum[e] += from[e];
      }
    }
    if (!any) continue;
    T* to = out + q * ldo + j;
    if (here == 4) {
      const T v[4] = {(T)sum[0], (T)sum[1], (T)sum[2], (T)sum[3]};
      __builtin_memcpy(to, v, sizeof(v));
    } else {
      for (int e = 0; e < here; ++e) to[e] = (T)sum[e];
    }
  }
}

static int64_t up(int64_t v, int64_t by) { return (v + by - 1) / by; }

struct TileGrid {
  int64_t tiles_i, strips, strip, workgroups;
  bool fits(int threads) const { return workgroups <= MAX_GRID / threads; }
};
static TileGrid grid_of(const ProductArgs& p, int op, int64_t bi, int64_t bj) {
  TileGrid g;
  const int64_t width = op == FORWARD ? p.n : p.k;
  g.tiles_i = op == GRAD_W ? up(p.n, bi) * (p.part > 0 ? dw_parts(p.pairs, p.groups, p.part) : p.groups)
                           : p.pair_off ? p.pairs / bi + p.groups : up(p.pairs, bi);
  // strips of up to 8 tiles, evenly dealt out; shorter where that would be less than 16 for each XCD
  const int64_t tiles_j = up(width, bj), most = std::min<int64_t>(8, std::max<int64_t>(1, g.tiles_i * tiles_j / 128));
  g.strips = up(tiles_j, most);
  g.strip = up(tiles_j, g.strips);
  g.workgroups = up(g.tiles_i * g.strips, 8) * 8 * g.strip;
  return g;
}

template <class T, int OP, int BI, int BJ, int WI, int WJ, int KS, int STEPS, bool FAST>
static int launch_tiles(ProductArgs p, hipStream_t st) {
  const TileGrid grid = grid_of(p, OP, BI, BJ);
  p.tiles_i = grid.tiles_i;
  p.strips = (uint32_t)grid.strips;
  p.strip = (uint32_t)grid.strip;
  if (!grid.fits(64 * WI * WJ * KS)) {
    set_error("too many tiles of work");
    return RABITQ_EINVAL;
  }
  const size_t lds = KS * STEPS * (BI + BJ) * 128 + (OP == GRAD_W ? 1024 * sizeof(int2) : BI * (sizeof(int) + sizeof(float)));
  auto kernel = product_tile_kernel<T, OP, BI, BJ, WI, WJ, KS, STEPS, FAST>;
  if (p.check_only) return RABITQ_OK;
  if (lds > 64 * 1024) RQ_HIP(hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
  kernel<<<(unsigned)grid.workgroups, 64 * WI * WJ * KS, lds, st>>>(p);
  RQ_HIP(hipGetLastError());
  return RABITQ_OK;
}

// Rows of whole 16-byte pieces at multiples of 16 bytes: the pieces can go to LDS without registers.  The kernel's 32-bit offsets
// have to reach every row of a from the first one (dw: each row's length), and 256 rows of b (as many as a tile or a step has).
static bool fast_rows(const ProductArgs& p, int op, int dtype) {
  const int64_t sz = dtype_bytes(dtype), per = 16 / sz, reach = (int64_t)1 << 32;
  const int64_t in_a = op == FORWARD ? p.k : p.n;  // elements of a row
  const int64_t rows_a = op == GRAD_W ? 1 : p.rows_a;
  return in_a % per == 0 && p.k % per == 0 && p.lda % per == 0 && p.ldb % per == 0 && (op == GRAD_W || p.stride % per == 0 || p.groups == 1) &&
         reinterpret_cast<uintptr_t>(p.a) % 16 == 0 && reinterpret_cast<uintptr_t>(p.b) % 16 == 0 &&
         rows_a * p.lda * sz < reach && 256 * p.ldb * sz < reach;
}

// Whether the forward product goes to the kernel that streams the matrices, in 16 x 16 tiles and without LDS.  With at most 8 rows per
// list on average (16 of a single list, whose rows are known) it reads every matrix once, as the tile kernel does, and waits for
// nothing (64 lists of 2048 x 2048 bf16, 4 rows each: 120 us and 152, 16 rows each: 187 and 182; one query against 200 000 rows of 768
// codes: 32 and 68).  Beyond, it reads more than the tile kernel, but has 16 times as many workgroups, which pays while those
// are two for each compute unit that the tile kernel can fill (codes, 512 tiles of 16: 17 x 4096 x 4096 9.1 and 12.8 us, 128 x 512 x 8192
// 11 and 20; 256 tiles, 1000 rows by 128 x 768: 3.9 and 6.1; more: 64 x 4096 x 4096 17 and 14, 48 x 8192 x 8192 46 and 26).
// fp32 tiles are bound by the multiplication, of which this kernel wastes less: four for each (1024 tiles, 64 x 4096 x 1024:
// 18 and 22; 768, 96 x 2048 x 16 384: 172 and 253).
static bool few_rows(const ProductArgs& p, int size) {
  const int64_t lists = p.groups;
  if (p.pairs <= (p.pair_off ? 8 : 16) * lists) return true;
  const int64_t tiles16 = (p.pair_off ? p.pairs / 16 + lists : up(p.pairs, 16)) * up(p.n, 16);
  const int64_t tiles64 = (p.pair_off ? p.pairs / 64 + lists : up(p.pairs, 64)) * up(p.n, 64);
  return tiles16 <= (size == 4 ? 1024 : 512) * up(tiles64, 256);
}

static int64_t few_workgroups(const ProductArgs& p) { return (p.pair_off ? p.pairs / 16 + p.groups : up(p.pairs, 16)) * up(p.n, 16); }

template <class T>
static int launch_few(const ProductArgs& p, hipStream_t st) {
  product_few_kernel<T><<<(unsigned)few_workgroups(p), 256, 0, st>>>(p);
  RQ_HIP(hipGetLastError());
  return RABITQ_OK;
}

// The edge of the tile.  A larger one moves fewer bytes per product, but fills the chip only with many rows and columns, and in rounds:
// a compute unit has one tile of 256 at a time, two of 128, more of 64.  The estimates below are in the time of a round of 256 tiles of
// 256.  A round that is not full saves half of what is missing (the card is limited by its power, and the others run faster); 512 tiles
// of 128 take 0.6, 256 of 64 0.105 (8192 x 4096 x 1024 bf16, 2 rounds of 256: 71 us, 128: 85, 64: 118, rows at odd addresses 94 and 121;
// 4352 x 4096 x 1024, a round and a bit: 60, 56, 63; 2048 x 4096 x 4096 codes, half a round: 56, 46, 64; 8192 rows, 8 lists, 1024 x 2048
// bf16, 144 tiles of 256, but 544 of 128: 53, 66, 72).  fp32 tiles are bound by the multiplication, so that their size hardly matters
// and what is left over at the end does: 0.26 and 0.07 for 256 tiles (8192 x 4096 x 1024: 488, 504, 518 us; 4352 x 4096 x 1024: 481,
// 320, 294).  A list ends inside its last tile, half a tile behind its end on average; rows of lists shorter than a tile would be
// multiplied for nothing (64 lists of 64 rows, 2048 x 2048 bf16: 182, 170, 150).  With one or two steps of contraction there is less
// to overlap a tile's start and end with (10 000 x 1024 x 128 codes: 19, 21, 17).  For dw the rows and columns are those of the matrices.
static int tile_size(const ProductArgs& p, int op, int size) {
  const int64_t width = op == FORWARD ? p.n : p.k;
  const int64_t rows = op == GRAD_W ? p.n : p.pairs / p.groups;  // of a list, on average
  const int64_t lists = op == GRAD_W && p.part > 0 ? dw_parts(p.pairs, p.groups, p.part) : p.groups;
  const int64_t contraction = op == FORWARD ? p.k : op == GRAD_X ? p.n : p.part > 0 ? p.part : p.pairs / p.groups;
  if (contraction * size < 512 || rows < 128) return 64;
  const auto rounds = [&](int64_t edge, int64_t round) {
    const bool whole = op == GRAD_W || lists == 1;
    const int64_t tiles = (whole ? up(rows, edge) * lists : p.pairs / edge + lists / 2) * up(width, edge);
    return size == 4 ? (double)up(tiles, round) : ((double)tiles / (double)round + (double)up(tiles, round)) / 2;
  };
  const double of_64 = (size == 4 ? 0.07 : 0.105) * rounds(64, 256);
  const double of_128 = size == 4 ? 0.26 * rounds(128, 256) : 0.6 * rounds(128, 512);
  if (rows >= 256 && rounds(256, 256) <= std::min(of_64, of_128)) return 256;
  return of_128 <= of_64 ? 128 : 64;
}

// The rows of a tile of 64 columns that four groups of wavefronts share (forward and dx), or 0: with 8 steps of contraction or more, and
// only where the chip takes all tiles at once, because a compute unit has room for one of them.  With 32 rows where there are no more
// of those than compute units (1119 rows, 5 of 10 lists each, 64 x 5472 fp32, 184 tiles: 56 us, 90 with tiles of 64; 326 rows, 2 lists, 1222 x
// 7352 fp16, 240 tiles: 32, with two steps in LDS 39, and 47; 300 x 2048 x 2048 fp16, 320 tiles: 19 and 13), else with 64 rows (256 x 4096 x 4096
// codes, 256 tiles: 14 us, not shared 22; 1024 x 1024 x 1024 bf16, 256 tiles: 10.4 and 12.5; 1408 x 768 x 1024 bf16, 264 tiles: 16.3 and
// 12.7, as codes with 2048 columns 16.5 and 13.3; 3001 rows, 24 lists, 501 x 777 fp16, 560 tiles: 28 and 20).  Tiles are counted as
// many as lists of any lengths may need: over 110 uneven batches near the border the choice takes 1.08 times the best one's time on
// average, with the tiles of lists of mean length 1.12 times.
static int shared_rows(const ProductArgs& p, int op, int size) {
  const int64_t width = op == FORWARD ? p.n : p.k, contraction = op == FORWARD ? p.k : p.n;
  if (contraction * size < 8 * 128) return 0;
  const int64_t lists = std::min<int64_t>(p.groups, p.pairs);
  const auto tiles = [&](int64_t rows) { return (p.pairs + lists * (rows - 1)) / rows * up(width, 64); };
  return tiles(32) <= 256 ? 32 : tiles(64) <= 256 ? 64 : 0;
}

// Whether the lists are shorter than a tile of 64, so that the matrices, read once each, are what the time goes to: a third step on its
// way is worth more than a fourth workgroup per compute unit (64 lists of 32 rows, 1024 x 2048 bf16: 91 us with two steps, 72 with
// three, codes 44 and 36; of 64 rows, 2048 x 2048 bf16: 184 and 164; but 1000 x 4096 x 4096 bf16 52 and 60).  fp32 tiles, bound by the
// multiplication, would rather have the workgroup (64 lists of 64 rows, 2048 x 2048: 456 and 496).
static bool short_lists(const ProductArgs& p) { return p.pairs <= 64 * (int64_t)p.groups; }

// A launch holds fewer than 2^32 threads, which few rows (of x or of each list) against many columns can pass: 256 threads take 16 columns
// in the kernel for few rows, 64 in tiles of 64, 128 in tiles of 128.  Where the one that the rules above choose does not hold the work,
// the next does (one query against 2^28 rows and more; 2^20 lists of 512 columns).
template <class T, int OP>
static int launch_typed(const ProductArgs& p, int dtype, hipStream_t st) {
  if constexpr (OP == FORWARD) {
    if (few_rows(p, sizeof(T)) && few_workgroups(p) <= MAX_GRID / 256) return launch_few<T>(p, st);
  }
  const bool fast = fast_rows(p, OP, dtype);
  int edge = tile_size(p, OP, sizeof(T));
  if (edge == 64 && !grid_of(p, OP, 64, 64).fits(256)) edge = 128;
  if (edge == 256)
    return fast ? launch_tiles<T, OP, 256, 256, 2, 4, 1, 2, true>(p, st) : launch_tiles<T, OP, 256, 256, 2, 4, 1, 2, false>(p, st);
  if (edge == 128)
    return fast ? launch_tiles<T, OP, 128, 128, 2, 2, 1, 2, true>(p, st) : launch_tiles<T, OP, 128, 128, 2, 2, 1, 2, false>(p, st);
  if constexpr (OP != GRAD_W) {
    const int rows = shared_rows(p, OP, sizeof(T));
    if (rows == 32)
      return fast ? launch_tiles<T, OP, 32, 64, 1, 2, 4, 3, true>(p, st) : launch_tiles<T, OP, 32, 64, 1, 2, 4, 2, false>(p, st);
    if (rows == 64)
      return fast ? launch_tiles<T, OP, 64, 64, 2, 2, 4, 2, true>(p, st) : launch_tiles<T, OP, 64, 64, 2, 2, 4, 2, false>(p, st);
    if constexpr (sizeof(T) < 4) {
      if (fast && short_lists(p)) return launch_tiles<T, OP, 64, 64, 2, 2, 1, 3, true>(p, st);
    }
  }
  return fast ? launch_tiles<T, OP, 64, 64, 2, 2, 1, 2, true>(p, st) : launch_tiles<T, OP, 64, 64, 2, 2, 1, 2, false>(p, st);
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

// Without parts a list occupies one workgroup per tile of its matrix, however long it is, so parts are for launches that would
// leave places of the chip free: fewer than 512 tiles of 128 x 128 (two for each compute unit).  A part is as long as fills those places,
// at least 512 positions, so that adding up costs less than it gains: 65 536 positions, 1 list, 512 x 512 bf16: 723 to 1449 us
// without, 82 with parts of 2048; 20 000 positions, 256 x 256 fp32: 544 and 55.  Above the line parts lose:
// 8192 positions, 4 lists, 2048 x 1024: 56 us without, 74 to 222 with; 3000, 24 lists, 512 x 768: 18 and 37.
// This rule and the ones above know the mean length of the lists only, since the offsets lie in device memory.  It is dw that minds
// uneven lists: 20 000 positions, 128 lists, 256 x 256, all lists alike: 18 us bf16, 41 fp32; nine positions of ten in one
// list: 175 and 1246 (forward and dx: 21 and 42, 19 and 42).
int dw_part(int64_t pairs, int groups, int64_t n, int64_t k) {
  const int64_t tiles = up(n, 128) * up(k, 128);
  if (tiles * groups >= 512) return 0;
  return (int)(std::max<int64_t>(1, pairs * tiles / 512 / 512) * 512);
}

int launch_product_dw(const ProductArgs& p, int dtype, float* scratch, hipStream_t st) {
  ProductArgs q = p;
  q.part = dw_part(p.pairs, p.groups, p.n, p.k);
  q.parts = scratch;
  const int rc = launch_op<GRAD_W>(q, dtype, st);
  if (rc || q.part == 0) return rc;
  const dim3 grid((unsigned)std::min<int64_t>(up(p.n * p.k, 1024), 65535), (unsigned)std::min(p.groups, 65535));
  if (p.out_dtype == RABITQ_F32) sum_parts_kernel<<<grid, 256, 0, st>>>(q, (float*)p.out);
  else if (p.out_dtype == RABITQ_F16) sum_parts_kernel<<<grid, 256, 0, st>>>(q, (_Float16*)p.out);
  else sum_parts_kernel<<<grid, 256, 0, st>>>(q, (__bf16*)p.out);
  RQ_HIP(hipGetLastError());
  return RABITQ_OK;
}

int launch_clear_bytes(void* at, int64_t n, hipStream_t st) {
  clear_bytes_kernel<<<(unsigned)std::min<int64_t>((n + 255) / 256, 4096), 256, 0, st>>>(static_cast<uint8_t*>(at), n);
  RQ_HIP(hipGetLastError());
  return RABITQ_OK;
}

template <class T>
static int sum_named(const float* parts, const uint8_t* named, int64_t rows, int nprobe, int k, T* out, int64_t ldo, hipStream_t st) {
  const unsigned grid = (unsigned)std::min<int64_t>(up(rows * up(k, 4), 256), 1 << 20);
  sum_named_kernel<T><<<grid, 256, 0, st>>>(parts, named, rows, nprobe, k, out, ldo);
  RQ_HIP(hipGetLastError());
  return RABITQ_OK;
}

int launch_sum_named(const float* parts, const uint8_t* named, int64_t rows, int nprobe, int k, void* out, int dtype, int64_t ldo,
                     hipStream_t st) {
  if (dtype == RABITQ_F32) return sum_named(parts, named, rows, nprobe, k, (float*)out, ldo, st);
  if (dtype == RABITQ_F16) return sum_named(parts, named, rows, nprobe, k, (_Float16*)out, ldo, st);
  return sum_named(parts, named, rows, nprobe, k, (__bf16*)out, ldo, st);
}

}  // namespace rq
