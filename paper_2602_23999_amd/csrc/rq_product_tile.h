// The tile kernel of the products by list and of the int8 products, all directions and types.
//
// out[i][j] = sum over c of A(i, c) B(j, c).  Forward: i = positions of a list (rows of x), j = rows of the list's matrix, c = k.
// dx: i = positions (rows of dout), j = columns of the matrix, c = its rows.  dw: i = rows of the matrix (columns of dout), j =
// its columns (columns of x), c = positions.  An operand whose c runs along memory is kept in LDS as it lies there, one line of 128
// bytes per row and step; one whose i or j runs along memory (the matrix of dx, both operands of dw) as lines of c, and is
// turned on the way to the registers.  Either way a step takes 128 bytes of every row: 128 codes, 64 halves or 32 floats.
#pragma once
#include <type_traits>

#include "rq_products.h"

namespace rq {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

enum ProductOp { FORWARD = 0, GRAD_X = 1, GRAD_W = 2 };

// 32 x 32 products of 32 bytes along c (a quarter of a step).  An operand is 16 bytes per lane: its row (column) is lane % 32, its
// half of the 32 bytes lane / 32.  PARTS instructions take them (f32: one for each of the four elements of every lane).
template <class T>
struct Mma {
  using Acc = f32x16;
  static constexpr int PARTS = 4;
  static __device__ __forceinline__ Acc mul(i32x4 a, i32x4 b, Acc c, int part) {
    return __builtin_amdgcn_mfma_f32_32x32x2f32(__builtin_bit_cast(f32x4, a)[part], __builtin_bit_cast(f32x4, b)[part], c, 0, 0, 0);
  }
};
template <>
struct Mma<_Float16> {
  using Acc = f32x16;
  static constexpr int PARTS = 1;
  static __device__ __forceinline__ Acc mul(i32x4 a, i32x4 b, Acc c, int) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
};
template <>
struct Mma<__bf16> {
  using Acc = f32x16;
  static constexpr int PARTS = 1;
  static __device__ __forceinline__ Acc mul(i32x4 a, i32x4 b, Acc c, int) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
};
template <>
struct Mma<int8_t> {
  using Acc = i32x16;
  static constexpr int PARTS = 1;
  static __device__ __forceinline__ Acc mul(i32x4 a, i32x4 b, Acc c, int) { return __builtin_amdgcn_mfma_i32_32x32x32_i8(a, b, c, 0, 0, 0); }
};

// Register r of lane l of an accumulator is row 8 (r / 4) + 4 (l / 32) + r % 4 of the first operand, column l % 32 of the second.  The
// first operand holds j, in an order that leaves a lane 16 neighbouring columns of the output: its row m is j = j_of_row(m).
__device__ __forceinline__ int j_of_row(int m) { return 16 * ((m >> 2) & 1) + 4 * (m >> 3) + (m & 3); }

// 16 bytes per lane from memory to LDS without registers: lane l's go to lds + 16 l.  Not waited for by the compiler: the kernel
// waits for all of them in front of the barrier behind which they are read.  The address in LDS goes through m0, as an operand, so that it is the
// compiler that writes m0 and knows it; the instruction wants a wait state behind that.
__device__ __forceinline__ void load_to_lds(const char* from, uint32_t lds) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"{m0}"(__builtin_amdgcn_readfirstlane(lds)), "v"(from) : "memory");
}
// The same from base + offset of the lane, base in scalar registers: nothing to compute per lane and step.
__device__ __forceinline__ void load_to_lds(const char* base, uint32_t offset, uint32_t lds) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"{m0}"(__builtin_amdgcn_readfirstlane(lds)), "v"(offset), "s"(base) : "memory");
}
// (As builtins and not in the asm, so that the compiler's own count of LDS reads in flight starts again from none.)
template <int LATER>  // loads of this wavefront that may still be on their way, if some_later
__device__ __forceinline__ void wait_and_barrier(bool some_later) {
  static_assert(LATER < 16);
  asm volatile("" ::: "memory");
  if (LATER > 0 && some_later) __builtin_amdgcn_s_waitcnt(0x0070 | LATER);  // vmcnt(LATER) lgkmcnt(0)
  else __builtin_amdgcn_s_waitcnt(0x0070);
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Where the lines' 16-byte pieces lie, so that the lanes of a read spread over the 64 banks.  A read of 16 bytes per lane takes 16
// lanes at a time, of which no two are alike in bits 0 to 3 (0 .. 15 as well as 0 .. 3, 12 .. 15, 20 .. 27): bit 0 picks the half of
// the banks that an odd or even line starts at, bits 1 to 3 the place of the piece.  Turned operands are read 64 (f32: 128) bytes of 4
// (2) lines at a time.
__device__ __forceinline__ int swizzle_i(int row) { return (row >> 1) & 7; }
__device__ __forceinline__ int swizzle_j(int row) { return ((row >> 1) & 1) | ((row >> 3) & 2) | (row & 4); }  // of m, row = j_of_row(m)
template <int SIZE, int PIECES>  // of a line of one c, of so many pieces
__device__ __forceinline__ int swizzle_turned(int c, int piece) {
  static_assert(PIECES == 8 || PIECES % 16 == 0);
  if constexpr (SIZE == 4) return piece ^ (((c >> 2) & 1) << 3);
  else if constexpr (PIECES == 8) return piece ^ ((c & 2) << 1);  // (odd lines start in the other half of the banks)
  else return piece ^ ((c & 3) << 2);
}

// 16 bytes of which the first `valid` elements exist, the others zero; any alignment.
template <class T>
__device__ __forceinline__ i32x4 load_piece(const char* from, int valid) {
  constexpr int EPC = 16 / sizeof(T);
  i32x4 v = {0, 0, 0, 0};
  if (valid >= EPC) {
    __builtin_memcpy(&v, from, 16);
  } else if (valid > 0) {
    T e[EPC];
#pragma unroll
    for (int i = 0; i < EPC; ++i) e[i] = i < valid ? reinterpret_cast<const T*>(from)[i] : T(0);
    __builtin_memcpy(&v, e, 16);
  }
  return v;
}

// 16 bytes moved towards their first by 0 to 15 bytes, zeros behind.
__device__ __forceinline__ i32x4 move_down(i32x4 v, int bytes) {
  uint64_t w[2];
  __builtin_memcpy(w, &v, 16);
  const int s = bytes % 8 * 8;
  const uint64_t lo = bytes < 8 ? w[0] : w[1], hi = bytes < 8 ? w[1] : 0;
  w[0] = s == 0 ? lo : lo >> s | hi << (64 - s);
  w[1] = hi >> s;
  __builtin_memcpy(&v, w, 16);
  return v;
}

static __device__ __align__(16) unsigned char product_zeros[16];

// FAST: every row of both operands starts at a multiple of 16 bytes and is whole pieces of 16 bytes long, and they lie near enough to
// each other for 32-bit offsets (fast_rows); pieces go to LDS without registers.  Otherwise they are loaded element by element where a
// row ends inside one, and pass through registers.
//
// KS: groups of wavefronts that share a tile, each with its own part of the contraction and its own steps in LDS; their sums are added
// up in order at the end.  For long contractions of so few tiles that most of the chip would be idle.
//
// STEPS: steps in LDS, the one that is multiplied and those on their way: 2, or (FAST) 3 where a step is over before the next has come.
template <class T, int OP, int BI, int BJ, int WI, int WJ, int KS, int STEPS, bool FAST>
__global__ __launch_bounds__(64 * WI * WJ * KS) void product_tile_kernel(ProductArgs p) {
  constexpr int NT = 64 * WI * WJ, SZ = sizeof(T), EPC = 16 / SZ, STEP = 128 / SZ;
  constexpr bool TA = OP == GRAD_W, TB = OP != FORWARD;
  constexpr int NA = BI * 8 / NT, NB = BJ * 8 / NT;       // pieces per thread and step
  constexpr int FI = BI / WI / 32, FJ = BJ / WJ / 32;     // 32 x 32 products per wavefront
  constexpr int STAGE = (BI + BJ) * 128;
  using Acc = typename Mma<T>::Acc;
  static_assert((KS == 1 || !TA) && (STEPS == 2 || (STEPS == 3 && FAST)));
  extern __shared__ __align__(16) char smem_all[];
  const int wave_all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), ks = wave_all / (WI * WJ);
  char* smem = smem_all + ks * (STEPS * STAGE);
  int* row_pair = reinterpret_cast<int*>(smem_all + KS * STEPS * STAGE);  // [BI] pair of every row, or -1
  float* row_scale = reinterpret_cast<float*>(row_pair + BI);  // [BI] codes only
  int2* block_pairs = reinterpret_cast<int2*>(row_pair);     // dw: [2][512] pairs of the positions and their rows of x, or -1
  const int tid = threadIdx.x % NT, lane = tid & 63, wave = wave_all % (WI * WJ);  // of the group
  const int wi = wave / WJ, wj = wave % WJ;

  // which tile
  const int64_t width = OP == FORWARD ? p.n : p.k;  // of the output
  const int64_t jt = (width + BJ - 1) / BJ;
  // Workgroups go to the 8 XCDs in turn.  An XCD gets strips of up to 8 neighbouring columns of tiles, whose share of a comes to its L2
  // once.  (Strips of one row of tiles: 64 lists of 512 rows, 2048 x 2048 codes: 179 us; blocks of 4 x 8 tiles, which read
  // least, 228: lists end inside them and XCDs run out of work at different times; an eighth of the columns each, 210.)
  const uint32_t turn = blockIdx.x >> 3, strip = turn / p.strip * 8 + (blockIdx.x & 7);
  const int64_t tile = strip / p.strips;
  const int64_t j_tile = (int64_t)(strip % p.strips) * p.strip + turn % p.strip;
  if (tile >= p.tiles_i || j_tile >= jt) return;
  const int64_t j0 = j_tile * BJ;
  int g;
  Span s;
  int64_t i0, iend;
  uint32_t nc;  // length of the contraction, below 2^31: positions and pairs are 32-bit numbers
  void* out = p.out;
  int out_dtype = p.out_dtype;
  int64_t ldo = p.ldo, ostride = OP == GRAD_W ? p.stride : 0;
  if constexpr (OP == GRAD_W) {
    const int64_t it = (p.n + BI - 1) / BI;
    const int64_t unit = tile / it;  // a list, or (p.part > 0) a part of p.part positions of one
    i0 = tile % it * BI;
    iend = p.n;
    if (p.part > 0) {
      g = list_of_tile(p, unit, p.part, lane);
      s = span_of(p, g);
      const int64_t begin = s.begin + (unit - (s.begin / p.part + g)) * p.part;
      if (begin < s.begin || begin >= s.end) return;
      if (s.end - s.begin > p.part) {  // one of several parts: its sums go to scratch
        out = p.parts + unit * p.n * p.k;
        out_dtype = RABITQ_F32;
        ldo = p.k;
        ostride = 0;
      }
      s.end = min(s.end, begin + p.part);
      s.begin = begin;
    } else {
      g = (int)unit;
      s = span_of(p, g);
    }
    nc = s.end > s.begin ? (uint32_t)(s.end - s.begin) : 0;
  } else {
    g = p.pair_off ? list_of_tile(p, tile, BI, lane) : 0;
    s = span_of(p, g);
    i0 = s.begin + (tile - (p.pair_off ? s.begin / BI + g : 0)) * BI;
    iend = s.end;
    if (i0 < s.begin || i0 >= iend) return;
    nc = OP == FORWARD ? p.k : (uint32_t)p.n;
    for (int i = threadIdx.x; i < BI; i += NT * KS) {
      const int pr = i0 + i < iend ? (int)pair_at(p, i0 + i) : -1;
      row_pair[i] = pr;
      if constexpr (SZ == 1) row_scale[i] = pr < 0 ? 0.f : p.scale_a[p.probe.of(pr)];
    }
    __syncthreads();
  }
  const char* a = static_cast<const char*>(p.a);
  const char* b = static_cast<const char*>(p.b) + (OP == GRAD_W ? 0 : (int64_t)g * p.stride * SZ);
  uint32_t span = nc;  // that a group goes over, in whole steps where there are several
  if constexpr (KS > 1) {
    span = ((nc + STEP - 1) / STEP + KS - 1) / KS * STEP;
    const uint32_t begin = ks * span;
    nc = begin < nc ? min(nc - begin, span) : 0;
    a += (uint64_t)begin * SZ;
    b += (TB ? (int64_t)begin * p.ldb : (int64_t)begin) * SZ;
  }
  const char* zeros = reinterpret_cast<const char*>(product_zeros);
  asm("" : "+s"(zeros));  // (kept in registers, not made anew at every use)

  const int jleft = (int)(width - j0 < BJ ? width - j0 : BJ);  // columns of the tile that exist
  // this thread's pieces of a step: where they start (FAST: from the first row of a, or of the tile of b, less than 2^32 bytes behind
  // it), and which c (or, of turned operands, which i or j) they hold
  const char* pa[FAST ? 1 : NA];
  uint32_t oa[FAST && !TA ? NA : 1], ob[FAST && !TA ? NB : 1];
  const int line = tid >> 3;
  const uint32_t ca = ((tid & 7) ^ swizzle_i(line)) * EPC;  // (the same for all q: NT / 8 lines on, of which it takes bits 1 to 3)
  static_assert(NT % 128 == 0);
  auto cb = [&](int q) -> uint32_t { return ((tid & 7) ^ swizzle_j(line) ^ swizzle_j(q * (NT / 8))) * EPC; };  // (takes bits 1, 2 and 4)
  constexpr int PA = BI * SZ / 16, PB = BJ * SZ / 16;     // pieces of a line of a turned operand
  if constexpr (!TA) {
#pragma unroll
    for (int q = 0; q < NA; ++q) {
      const int pr = row_pair[line + q * (NT / 8)];
      const int64_t row = pr < 0 ? 0 : OP == FORWARD ? p.probe.of(pr) : pr;  // (a row that is not there reads row 0, unused)
      if constexpr (FAST) oa[q] = (uint32_t)((row * p.lda + ca) * SZ);
      else pa[q] = a + (row * p.lda + ca) * SZ;
    }
  }
  const char* pb = nullptr;  // piece 0; the others lie whole lines behind it
  if constexpr (!FAST && !TB) pb = b + (j0 + line) * p.ldb * SZ;
  if constexpr (!FAST && OP == GRAD_X) pb = b + (tid / PB * p.ldb + j0) * SZ;
  if constexpr (FAST && !TA) {  // (rows and columns that are not there read the first ones, unused)
#pragma unroll
    for (int q = 0; q < NB; ++q) {
      if constexpr (!TB) {
        const int row = line + q * (NT / 8);
        ob[q] = (uint32_t)(((row < jleft ? row : 0) * p.ldb + cb(q)) * SZ);
      } else {
        const int c = (tid + q * NT) / PB, col = swizzle_turned<SZ, PB>(c, (tid + q * NT) % PB) * EPC;
        ob[q] = (uint32_t)((c * p.ldb + (col < jleft ? col : 0)) * SZ);
      }
    }
    b += (!TB ? j0 * p.ldb : j0) * SZ;
  }
  // dw: the pairs of this thread's lines, a step ahead (the lines of both operands are the same).  They come from a ring of two
  // blocks of positions in LDS: loads of their own would have to arrive within a step, and all loads are waited for in order.
  constexpr int LP = TA ? NA : 1, BLOCK = 512, FILL = BLOCK / NT;
  static_assert(!TA || (BI == BJ && BLOCK % NT == 0));
  int2 pairs_next[LP];
  int block_next[FILL > 0 ? FILL : 1];
  auto load_block = [&](uint32_t block) {
    if constexpr (TA) {
#pragma unroll
      for (int f = 0; f < FILL; ++f) {
        const uint32_t c = block * BLOCK + f * NT + tid;
        block_next[f] = c < nc ? (int)pair_at(p, s.begin + c) : -1;
      }
    }
  };
  auto store_block = [&](uint32_t block) {
    if constexpr (TA) {
#pragma unroll
      for (int f = 0; f < FILL; ++f) {
        const int pr = block_next[f];
        block_pairs[block % 2 * BLOCK + f * NT + tid] = int2{pr, pr < 0 ? -1 : p.probe.of(pr)};
      }
    }
  };
  auto find_pairs = [&](uint32_t c0) {
    if constexpr (TA) {
#pragma unroll
      for (int q = 0; q < NA; ++q) pairs_next[q] = block_pairs[(c0 + (uint32_t)(tid + q * NT) / PA) % (2 * BLOCK)];
    }
  };
  const uint32_t lds = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem + wave * 1024);
  // FAST: the columns that a thread has of both operands of dw are the same in all its lines (none: a row of zeros)
  const char *ga = zeros, *gb = zeros;
  uint32_t ga_ld = 0, gb_ld = 0;
  if constexpr (FAST && TA) {
    const int col_a = swizzle_turned<SZ, PA>(tid / PA, tid % PA) * EPC, col_b = swizzle_turned<SZ, PB>(tid / PB, tid % PB) * EPC;
    if (col_a < iend - i0) ga = a + (i0 + col_a) * SZ, ga_ld = (uint32_t)(p.lda * SZ);
    if (col_b < jleft) gb = b + (j0 + col_b) * SZ, gb_ld = (uint32_t)(p.ldb * SZ);
  }
  // FAST: piece q of the step at c0, straight to LDS
  auto fetch_piece = [&](int q, uint32_t c0, int buf) {
    const uint32_t at = lds + buf * STAGE + (q < NA ? q * (NT * 16) : BI * 128 + (q - NA) * (NT * 16));
    const int qa = q < NA ? q : 0, qb = q < NA ? 0 : q - NA;
    if (c0 >= span) return;
    if constexpr (TA) {
      const int row = q < NA ? pairs_next[qa].x : pairs_next[qb].y;
      const char* from = (q < NA ? ga : gb) + (uint64_t)(uint32_t)row * (q < NA ? ga_ld : gb_ld);
      load_to_lds(row < 0 ? zeros : from, at);
    } else {
      const char* base = q < NA ? a + (uint64_t)c0 * SZ : b + (TB ? (int64_t)c0 * p.ldb : (int64_t)c0) * SZ;
      const uint32_t offset = q < NA ? oa[qa] : ob[qb];
      if (c0 + STEP <= nc) {
        load_to_lds(base, offset, at);
      } else {  // the last step: zeros behind the end
        const uint32_t c = c0 + (q < NA ? ca : !TB ? cb(qb) : (uint32_t)(tid + qb * NT) / PB);
        load_to_lds(c < nc ? base + offset : zeros, at);
      }
    }
  };
  // else: where it lies, and how many of its elements exist (none or more than there are, as may be)
  // A turned operand whose row ends inside a piece has one in every line, and each element of its own would be waited for.  Such a
  // piece is loaded from before its start, to end with the row, and moved in the registers (rows of less than a piece: by element).
  // (1107 rows, 2 of 6 lists each, 7999 x 8086 fp16, dx: 890 us by element, 603 moved, and 592 with 8088 columns, of whole pieces.)
  int back_a = 0, back_b = 0;
  if constexpr (!FAST && TA) {
    const int64_t col = i0 + swizzle_turned<SZ, PA>(tid / PA, tid % PA) * EPC, left = iend - col;  // (the same for all q)
    if (left > 0 && left < EPC && col > 0) back_a = (EPC - (int)left) * SZ;
  }
  if constexpr (!FAST && TB) {
    const int64_t col = j0 + swizzle_turned<SZ, PB>(tid / PB, tid % PB) * EPC, left = width - col;
    if (left > 0 && left < EPC && col > 0) back_b = (EPC - (int)left) * SZ;
  }
  auto piece_a = [&](int q, uint32_t c0, const char*& from) -> int {
    if constexpr (!TA) {
      from = pa[q] + (uint64_t)c0 * SZ;
      return c0 + ca < nc ? (int)(nc - c0 - ca) : 0;
    } else {
      const int col = swizzle_turned<SZ, PA>((tid + q * NT) / PA, (tid + q * NT) % PA) * EPC;
      from = a + ((int64_t)pairs_next[q].x * p.lda + i0 + col) * SZ - back_a;
      return pairs_next[q].x < 0 ? 0 : (int)(iend - i0) - col + back_a / SZ;
    }
  };
  auto piece_b = [&](int q, uint32_t c0, const char*& from) -> int {
    if constexpr (!TB) {
      from = pb + ((int64_t)(q * (NT / 8)) * p.ldb + c0 + cb(q)) * SZ;
      return line + q * (NT / 8) < jleft && c0 + cb(q) < nc ? (int)(nc - c0 - cb(q)) : 0;
    } else if constexpr (OP == GRAD_X) {
      const int c = (tid + q * NT) / PB, piece = swizzle_turned<SZ, PB>(c, (tid + q * NT) % PB);
      from = pb + ((int64_t)(c0 + q * (NT / PB)) * p.ldb + piece * EPC) * SZ - back_b;
      return c0 + c < nc ? jleft - piece * EPC + back_b / SZ : 0;
    } else {
      const int col = swizzle_turned<SZ, PB>((tid + q * NT) / PB, (tid + q * NT) % PB) * EPC;
      from = b + ((int64_t)pairs_next[q].y * p.ldb + j0 + col) * SZ - back_b;
      return pairs_next[q].y < 0 ? 0 : jleft - col + back_b / SZ;
    }
  };
  constexpr int RA = FAST ? 1 : NA, RB = FAST ? 1 : NB;
  i32x4 va[RA], vb[RB];
  auto fetch_regs = [&](uint32_t c0) {
    if constexpr (!FAST) {
#pragma unroll
      for (int q = 0; q < NA; ++q) {
        const char* from;
        const int valid = piece_a(q, c0, from);
        va[q] = load_piece<T>(from, valid);
      }
#pragma unroll
      for (int q = 0; q < NB; ++q) {
        const char* from;
        const int valid = piece_b(q, c0, from);
        vb[q] = load_piece<T>(from, valid);
      }
    }
  };
  auto stash = [&](int buf) {
    if constexpr (!FAST) {
      char* at = smem + buf * STAGE + tid * 16;
      if (TA && back_a != 0) {
#pragma unroll
        for (int q = 0; q < NA; ++q) va[q] = move_down(va[q], back_a);
      }
      if (TB && back_b != 0) {
#pragma unroll
        for (int q = 0; q < NB; ++q) vb[q] = move_down(vb[q], back_b);
      }
#pragma unroll
      for (int q = 0; q < NA; ++q) *reinterpret_cast<i32x4*>(at + q * (NT * 16)) = va[q];
#pragma unroll
      for (int q = 0; q < NB; ++q) *reinterpret_cast<i32x4*>(at + BI * 128 + q * (NT * 16)) = vb[q];
    }
  };

  // operands of 32 lines (columns) and the sub-th 32 bytes of c
  const int l32 = lane & 31, upper = lane >> 5;
  auto turned = [&](const char* tile, auto cols_c, int col32, int sub, bool is_j) -> i32x4 {
    constexpr int cols = decltype(cols_c)::value;
    if constexpr (SZ == 4) {
      f32x4 v;
      const int col = col32 * 32 + (is_j ? j_of_row(l32) : l32);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int c = sub * 8 + 4 * upper + e;
        v[e] = *reinterpret_cast<const float*>(tile + c * (cols * 4) + swizzle_turned<4, cols / 4>(c, col >> 2) * 16 + (col & 3) * 4);
      }
      return __builtin_bit_cast(i32x4, v);
    } else {
      // of 16 lanes, lane 4 r + t reads 4 columns of line r, and lane 4 t + e gets the e-th of those t read, of the 4 lines
      const int c = sub * 16 + 8 * upper + ((lane & 15) >> 2), t = lane & 3, half = (lane >> 4) & 1;
      const int col = is_j ? j_of_row(16 * half + 4 * t) : 16 * half + 4 * t;
      const char* at = tile + c * (cols * 2) + swizzle_turned<2, cols / 8>(c, col32 * 4 + (col >> 3)) * 16 + (col & 4) * 2;
      typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + 4 * (cols * 2)));
      i32x4 v;
      __builtin_memcpy(&v, &lo, 8);
      __builtin_memcpy(reinterpret_cast<char*>(&v) + 8, &hi, 8);
      return v;
    }
  };
  auto frag_i = [&](const char* st, int f, int sub) -> i32x4 {
    if constexpr (TA) return turned(st, std::integral_constant<int, BI>{}, wi * FI + f, sub, false);
    return *reinterpret_cast<const i32x4*>(st + ((wi * FI + f) * 32 + l32) * 128 + (((sub * 2 + upper) ^ swizzle_i(l32)) * 16));
  };
  auto frag_j = [&](const char* st, int f, int sub) -> i32x4 {
    if constexpr (TB) return turned(st + BI * 128, std::integral_constant<int, BJ>{}, wj * FJ + f, sub, true);
    const int in32 = j_of_row(l32);
    return *reinterpret_cast<const i32x4*>(st + BI * 128 + ((wj * FJ + f) * 32 + in32) * 128 + (((sub * 2 + upper) ^ swizzle_j(in32)) * 16));
  };

  Acc acc[FI][FJ];
#pragma unroll
  for (int x = 0; x < FI; ++x)
#pragma unroll
    for (int y = 0; y < FJ; ++y) acc[x][y] = Acc{0};

  // A step is multiplied in four parts of 32 bytes of every line; the operands of the next part are read while one is multiplied.
  // The one barrier of a step stands in front of its last part, where everybody has read the whole step and the next one has
  // arrived; behind it the step that takes its place in LDS is requested, one half of its pieces during that part and the other during
  // the next.  Reads and requests are dealt out among the products.  Behind the last step the reads go on for nothing (old lines of LDS).
  i32x4 ai[2][FI], bj[2][FJ];
  auto read_one = [&](const char* st, int r, int sub, int set) {
    if (r < FJ) bj[set][r < FJ ? r : 0] = frag_j(st, r < FJ ? r : 0, sub);
    else ai[set][r < FJ ? 0 : r - FJ] = frag_i(st, r < FJ ? 0 : r - FJ, sub);
  };
  auto multiply = [&](auto sub_c, int next_buf, auto request_c, uint32_t c2, int buf2) {
    constexpr int sub = decltype(sub_c)::value, set = sub & 1;
    const char* st = smem + next_buf * STAGE;
    constexpr int READS = FI + FJ, ROWS = FI >= 2 ? FI - 1 : 1;  // rows of products that reads are dealt out among: all but the last
#pragma unroll
    for (int x = 0; x < FI; ++x) {
#pragma unroll
      for (int part = 0; part < Mma<T>::PARTS; ++part)
#pragma unroll
        for (int y = 0; y < FJ; ++y) acc[x][y] = Mma<T>::mul(bj[set][y], ai[set][x], acc[x][y], part);
#pragma unroll
      for (int r = 0; r < READS; ++r)
        if (r * ROWS / READS == x) read_one(st, r, (sub + 1) & 3, set ^ 1);
      constexpr int HALF = decltype(request_c)::value;  // which half of the pieces is requested, or none
      if constexpr (HALF >= 0) {
#pragma unroll
        for (int q = 0; q < NA + NB; ++q)
          if (q * (2 * FI) / (NA + NB) == HALF * FI + x) fetch_piece(q, c2, buf2);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  constexpr std::integral_constant<int, 0> sub0{};
  constexpr std::integral_constant<int, 1> sub1{};
  constexpr std::integral_constant<int, 2> sub2{};
  constexpr std::integral_constant<int, 3> sub3{};
  constexpr std::integral_constant<int, FAST ? 0 : -1> first{};
  constexpr std::integral_constant<int, FAST ? 1 : -1> second{};
  constexpr std::integral_constant<int, -1> nothing{};
  auto fetch_all = [&](uint32_t c0, int buf) {
    if constexpr (FAST) {
#pragma unroll
      for (int q = 0; q < NA + NB; ++q) fetch_piece(q, c0, buf);
    } else {
      fetch_regs(c0);
    }
  };
  if (span > 0) {
    if constexpr (TA) {
      load_block(0);
      store_block(0);
      load_block(1);
      store_block(1);
      __syncthreads();
    }
#pragma unroll
    for (int u = 0; u < STEPS - 1; ++u) {
      find_pairs(u * STEP);
      fetch_all(u * STEP, u);
    }
    find_pairs((STEPS - 1) * STEP);
    stash(0);
    constexpr int LATER = (STEPS - 2) * (NA + NB);
    wait_and_barrier<LATER>(STEP < span);
#pragma unroll
    for (int r = 0; r < FI + FJ; ++r) read_one(smem, r, 0, 0);
    if constexpr (FAST) {
#pragma unroll
      for (int q = 0; q < NA + NB; ++q)
        if (q * (2 * FI) / (NA + NB) < FI) fetch_piece(q, (STEPS - 1) * STEP, STEPS - 1);
    } else {
      fetch_regs(STEP);
    }
    int buf = 0;
    for (uint32_t c0 = 0; c0 < span; c0 += STEP) {
      // (the first step of block b: nobody looks at block b - 1 any more, and b + 1 is there)
      const bool refill = TA && c0 != 0 && c0 % BLOCK == 0;
      const int next = STEPS == 2 ? buf ^ 1 : buf == STEPS - 1 ? 0 : buf + 1;
      const int before = STEPS == 2 ? next : buf == 0 ? STEPS - 1 : buf - 1;
      multiply(sub0, buf, second, c0 + (STEPS - 1) * STEP, before);
      if (refill) load_block(c0 / BLOCK + 1);
      multiply(sub1, buf, nothing, 0, 0);
      find_pairs(c0 + STEPS * STEP);
      multiply(sub2, buf, nothing, 0, 0);
      stash(next);
      wait_and_barrier<LATER>(c0 + 2 * STEP < span);  // (then the step after the next was requested behind the next)
      if (refill) store_block(c0 / BLOCK + 1);
      if constexpr (!FAST) fetch_regs(c0 + 2 * STEP);
      multiply(sub3, next, first, c0 + STEPS * STEP, buf);
      buf = next;
    }
    __builtin_amdgcn_s_waitcnt(0x0070);  // nothing may be on its way to LDS when the workgroup ends
  }

  if constexpr (KS > 1) {
    static_assert(FI * FJ * 64 * NT <= 2 * STAGE);
    Acc* sums = reinterpret_cast<Acc*>(smem_all);  // [group][product][thread]
    constexpr int PER_GROUP = 2 * STAGE / (int)sizeof(Acc);
    __syncthreads();  // (the last operands have been read)
    if (ks > 0) {
#pragma unroll
      for (int x = 0; x < FI; ++x)
#pragma unroll
        for (int y = 0; y < FJ; ++y) sums[ks * PER_GROUP + (x * FJ + y) * NT + tid] = acc[x][y];
    }
    __syncthreads();
    if (ks > 0) return;
#pragma unroll
    for (int u = 1; u < KS; ++u)
#pragma unroll
      for (int x = 0; x < FI; ++x)
#pragma unroll
        for (int y = 0; y < FJ; ++y) acc[x][y] += sums[u * PER_GROUP + (x * FJ + y) * NT + tid];
  }

  // A lane has 16 neighbouring columns of a row, so a store of its own would touch 32 rows for 16 bytes each.  The wavefront's 32
  // rows go through LDS instead (its own part of it, as fp32, pieces of 16 bytes swizzled by the row) and out in whole rows of COLS.
  constexpr int COLS = FJ * 32, PIECES = COLS / 4;  // of a row: a power of two
  static_assert(32 * COLS * 4 * WI * WJ <= 2 * STAGE && (PIECES & (PIECES - 1)) == 0 && PIECES >= 8);
  const int each = out_dtype == RABITQ_F32 ? 4 : 8;  // columns that a lane stores at once
  f32x4* mine = reinterpret_cast<f32x4*>(smem) + wave * (32 * PIECES);
  const int per_row = COLS / each, rows_at_once = 64 / per_row;
  const int col = lane % per_row * each;
  const int64_t j = j0 + wj * COLS + col;
  float sb[SZ == 1 ? 8 : 1];  // of this lane's columns
  if constexpr (SZ == 1) {
#pragma unroll
    for (int e = 0; e < 8; ++e) sb[e] = e < each && j + e < width ? p.scale_b[(int64_t)g * p.n + j + e] : 0.f;
  }
  if constexpr (KS == 1) __syncthreads();  // (the last operands have been read)
#pragma unroll
  for (int x = 0; x < FI; ++x) {
#pragma unroll
    for (int y = 0; y < FJ; ++y)
#pragma unroll
      for (int h = 0; h < 4; ++h)
        mine[l32 * PIECES + ((y * 8 + upper * 4 + h) ^ (l32 & (PIECES - 1)))] =
            f32x4{(float)acc[x][y][4 * h], (float)acc[x][y][4 * h + 1], (float)acc[x][y][4 * h + 2], (float)acc[x][y][4 * h + 3]};
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    for (int r = lane / per_row; r < 32; r += rows_at_once) {
      const int i = (wi * FI + x) * 32 + r;
      int64_t row;
      if constexpr (OP == GRAD_W) row = i0 + i < iend ? i0 + i : -1;
      else row = row_pair[i];
      if (row < 0) continue;
      if (OP == GRAD_X && p.named && j == 0) p.named[row] = 1;
      if (j >= width) continue;
      const int64_t at = (int64_t)g * ostride + row * ldo + j;
      f32x4 lo = mine[r * PIECES + ((col >> 2) ^ (r & (PIECES - 1)))];
      f32x4 hi = lo;
      if (each == 8) hi = mine[r * PIECES + (((col >> 2) + 1) ^ (r & (PIECES - 1)))];
      if constexpr (SZ == 1) {
        const float sa = row_scale[i];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          lo[e] = lo[e] * sa * sb[e];
          hi[e] = hi[e] * sa * sb[4 + e];
        }
      }
      if (j + each <= width) {  // (at any alignment of the element)
        if (out_dtype == RABITQ_F32) {
          __builtin_memcpy(static_cast<float*>(out) + at, &lo, 16);
        } else if (out_dtype == RABITQ_F16) {
          const f16x8 v = __builtin_convertvector(__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7), f16x8);
          __builtin_memcpy(static_cast<_Float16*>(out) + at, &v, 16);
        } else {
          const bf16x8 v = __builtin_convertvector(__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7), bf16x8);
          __builtin_memcpy(static_cast<__bf16*>(out) + at, &v, 16);
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (e < each && j + e < width) store_as(out, out_dtype, at + e, e < 4 ? lo[e % 4] : hi[e % 4]);
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

}  // namespace rq
