// The tile kernel of the products by list and of the int8 products, all directions and types.
//
// out[i][j] = sum over c of A(i, c) B(j, c).  Forward: i = positions of a list (rows of x), j = rows of the list's matrix, c = k.
// dx: i = positions (rows of dout), j = columns of the matrix, c = its rows.  dw: i = rows of the matrix (columns of dout), j =
// its columns (columns of x), c = positions.  An operand whose c runs along memory is kept in LDS as it lies there, one line of 128
// bytes per row and step; one whose i or j runs along memory (the matrix of dx, both operands of dw) as lines of c, and is
// turned on the way to the registers.  Either way a step takes 128 bytes of every row: 128 codes, 64 halves or 32 floats.
#pragma once
#include "rq_products.h"

namespace rq {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

enum ProductOp { FORWARD = 0, GRAD_X = 1, GRAD_W = 2 };

// 16 bytes of an operand per lane: row (column) lane % 16, the (lane / 16)-th quarter of 64 bytes along c.
template <class T>
struct Mma {  // f32: the four instructions take elements 0, 1, 2, 3 of every lane's quarter
  using Acc = f32x4;
  static __device__ __forceinline__ Acc mul(i32x4 a, i32x4 b, Acc c) {
    const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[e], y[e], c, 0, 0, 0);
    return c;
  }
};
template <>
struct Mma<_Float16> {
  using Acc = f32x4;
  static __device__ __forceinline__ Acc mul(i32x4 a, i32x4 b, Acc c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
};
template <>
struct Mma<__bf16> {
  using Acc = f32x4;
  static __device__ __forceinline__ Acc mul(i32x4 a, i32x4 b, Acc c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
};
template <>
struct Mma<int8_t> {
  using Acc = i32x4;
  static __device__ __forceinline__ Acc mul(i32x4 a, i32x4 b, Acc c) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0); }
};

// 16 bytes per lane from memory to LDS without registers: lane l's go to lds + 16 l.  Not waited for by the compiler: the kernel
// waits for all of them in front of the barrier behind which they are read.
__device__ __forceinline__ void load_to_lds(const char* from, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(from) : "memory");
}
__device__ __forceinline__ void wait_and_barrier() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// Where the lines' 16-byte pieces lie, so that the lanes of a read spread over the banks.
__device__ __forceinline__ int swizzle_i(int row) { return row & 7; }
__device__ __forceinline__ int swizzle_j(int row) { return (row & 3) | ((row >> 1) & 4); }
template <int SIZE>
__device__ __forceinline__ int swizzle_turned(int c, int piece) {  // of a line of one c
  if constexpr (SIZE == 4) return piece ^ (((c >> 2) & 3) << 2);
  else return piece ^ (((c & 3) | ((c >> 1) & 4)) << 1);
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

static __device__ __align__(16) unsigned char product_zeros[16];

// FAST: every row of both operands starts at a multiple of 16 bytes and is whole pieces of 16 bytes long; pieces go to LDS without
// registers.  Otherwise they are loaded element by element where a row ends inside one, and pass through registers.
template <class T, int OP, int BI, int BJ, int WI, int WJ, bool FAST>
__global__ __launch_bounds__(64 * WI * WJ) void product_tile_kernel(ProductArgs p) {
  constexpr int NT = 64 * WI * WJ, SZ = sizeof(T), EPC = 16 / SZ, STEP = 128 / SZ;
  constexpr bool TA = OP == GRAD_W, TB = OP != FORWARD;
  constexpr int NA = BI * 8 / NT, NB = BJ * 8 / NT;       // pieces per thread and step
  constexpr int FI = BI / WI / 16, FJ = BJ / WJ / 16;     // 16 x 16 products per wavefront
  constexpr int STAGE = (BI + BJ) * 128;
  using Acc = typename Mma<T>::Acc;
  extern __shared__ __align__(16) char smem[];
  int* row_pair = reinterpret_cast<int*>(smem + 2 * STAGE);  // [BI] pair of every row, or -1
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wi = wave / WJ, wj = wave % WJ;

  // which tile
  const int nj = OP == FORWARD ? (int)0 : p.k;
  const int64_t width = OP == FORWARD ? p.n : (int64_t)nj;  // of the output
  const int64_t jt = (width + BJ - 1) / BJ;
  const int64_t per = (gridDim.x + 7) / 8;
  const int64_t id = (blockIdx.x & 7) * per + (blockIdx.x >> 3);  // consecutive tiles on one XCD
  if (id >= p.tiles) return;
  const int64_t tile = id / jt, j0 = id % jt * BJ;
  int g;
  Span s;
  int64_t i0, iend, nc;
  if constexpr (OP == GRAD_W) {
    const int64_t it = (p.n + BI - 1) / BI;
    g = (int)(tile / it);
    s = span_of(p, g);
    i0 = tile % it * BI;
    iend = p.n;
    nc = s.end > s.begin ? s.end - s.begin : 0;
  } else {
    g = p.pair_off ? list_of_tile(p, tile, BI, lane) : 0;
    s = span_of(p, g);
    i0 = s.begin + (tile - (p.pair_off ? s.begin / BI + g : 0)) * BI;
    iend = s.end;
    if (i0 < s.begin || i0 >= iend) return;
    nc = OP == FORWARD ? p.k : p.n;
    for (int i = tid; i < BI; i += NT) row_pair[i] = i0 + i < iend ? (int)pair_at(p, i0 + i) : -1;
    __syncthreads();
  }
  const char* a = static_cast<const char*>(p.a);
  const char* b = static_cast<const char*>(p.b) + (OP == GRAD_W ? 0 : (int64_t)g * p.stride * SZ);
  const char* zeros = reinterpret_cast<const char*>(product_zeros);

  // this thread's pieces of a step: where they start, and which c (or, of turned operands, which i or j) they hold
  const char *pa[NA], *pb[NB];
  const int line = tid >> 3;
  const int ca = ((tid & 7) ^ swizzle_i(line)) * EPC, cb = ((tid & 7) ^ swizzle_j(line)) * EPC;  // (the same for all q)
  constexpr int PA = BI * SZ / 16, PB = BJ * SZ / 16;     // pieces of a line of a turned operand
  if constexpr (!TA) {
#pragma unroll
    for (int q = 0; q < NA; ++q) {
      const int pr = row_pair[line + q * (NT / 8)];
      const int64_t row = pr < 0 ? 0 : OP == FORWARD ? pr / p.nprobe : pr;  // (a row that is not there reads row 0, unused)
      pa[q] = a + (row * p.lda + ca) * SZ;
    }
  }
  if constexpr (!TB) {
#pragma unroll
    for (int q = 0; q < NB; ++q) {
      const int64_t row = j0 + line + q * (NT / 8);
      pb[q] = b + ((row < width ? row : 0) * p.ldb + cb) * SZ;
    }
  } else if constexpr (OP == GRAD_X) {
#pragma unroll
    for (int q = 0; q < NB; ++q) {
      const int c = (tid + q * NT) / PB, piece = swizzle_turned<SZ>(c, (tid + q * NT) % PB);
      pb[q] = b + (c * p.ldb + j0 + piece * EPC) * SZ;
    }
  }
  // dw: the pairs of this thread's lines, a step ahead
  constexpr int LA = TA ? NA : 1, LB = TA ? NB : 1;
  int pair_a[LA], pair_b[LB];
  auto find_pairs = [&](int64_t c0) {
    if constexpr (OP == GRAD_W) {
#pragma unroll
      for (int q = 0; q < NA; ++q) {
        const int64_t c = c0 + (tid + q * NT) / PA;
        pair_a[q] = c < nc ? (int)pair_at(p, s.begin + c) : -1;
      }
#pragma unroll
      for (int q = 0; q < NB; ++q) {
        const int64_t c = c0 + (tid + q * NT) / PB;
        pair_b[q] = c < nc ? (int)pair_at(p, s.begin + c) : -1;
      }
    }
  };
  // where piece q of the step at c0 lies, and how many of its elements exist
  auto piece_a = [&](int q, int64_t c0, const char*& from) -> int64_t {
    if constexpr (!TA) {
      from = pa[q];
      pa[q] += 128;
      return nc - c0 - ca;
    } else {
      const int col = swizzle_turned<SZ>((tid + q * NT) / PA, (tid + q * NT) % PA) * EPC;
      from = a + ((int64_t)pair_a[q] * p.lda + i0 + col) * SZ;
      return pair_a[q] < 0 ? 0 : iend - i0 - col;
    }
  };
  auto piece_b = [&](int q, int64_t c0, const char*& from) -> int64_t {
    if constexpr (!TB) {
      from = pb[q];
      pb[q] += 128;
      return nc - c0 - cb;
    } else if constexpr (OP == GRAD_X) {
      const int c = (tid + q * NT) / PB, piece = swizzle_turned<SZ>(c, (tid + q * NT) % PB);
      from = pb[q];
      pb[q] += STEP * p.ldb * SZ;
      return c0 + c < nc ? width - j0 - piece * EPC : 0;
    } else {
      const int col = swizzle_turned<SZ>((tid + q * NT) / PB, (tid + q * NT) % PB) * EPC;
      from = b + ((int64_t)(pair_b[q] / p.nprobe) * p.ldb + j0 + col) * SZ;
      return pair_b[q] < 0 ? 0 : width - j0 - col;
    }
  };
  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
  auto fetch = [&](int64_t c0, int buf) {  // straight to LDS
    const uint32_t at = lds + buf * STAGE + wave * 1024;
#pragma unroll
    for (int q = 0; q < NA; ++q) {
      const char* from;
      const int64_t valid = piece_a(q, c0, from);
      load_to_lds(valid > 0 ? from : zeros, at + q * (NT * 16));
    }
#pragma unroll
    for (int q = 0; q < NB; ++q) {
      const char* from;
      const int64_t valid = piece_b(q, c0, from);
      load_to_lds(valid > 0 ? from : zeros, at + BI * 128 + q * (NT * 16));
    }
  };
  constexpr int RA = FAST ? 1 : NA, RB = FAST ? 1 : NB;
  i32x4 va[RA], vb[RB];
  auto fetch_regs = [&](int64_t c0) {
    if constexpr (!FAST) {
#pragma unroll
      for (int q = 0; q < NA; ++q) {
        const char* from;
        const int64_t valid = piece_a(q, c0, from);
        va[q] = load_piece<T>(from, (int)(valid > EPC ? EPC : valid));
      }
#pragma unroll
      for (int q = 0; q < NB; ++q) {
        const char* from;
        const int64_t valid = piece_b(q, c0, from);
        vb[q] = load_piece<T>(from, (int)(valid > EPC ? EPC : valid));
      }
    }
  };
  auto stash = [&](int buf) {
    if constexpr (!FAST) {
      char* at = smem + buf * STAGE + tid * 16;
#pragma unroll
      for (int q = 0; q < NA; ++q) *reinterpret_cast<i32x4*>(at + q * (NT * 16)) = va[q];
#pragma unroll
      for (int q = 0; q < NB; ++q) *reinterpret_cast<i32x4*>(at + BI * 128 + q * (NT * 16)) = vb[q];
    }
  };

  // fragments
  const int l16 = lane & 15, quarter = lane >> 4;
  auto turned = [&](const char* tile, int cols, int col16, int slab) -> i32x4 {  // columns 16 col16 .. + 15, 64 bytes of c
    if constexpr (SZ == 4) {
      f32x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int c = slab * 16 + 4 * quarter + e;
        v[e] = *reinterpret_cast<const float*>(tile + c * (cols * 4) + ((col16 ^ quarter) * 64) + l16 * 4);
      }
      return __builtin_bit_cast(i32x4, v);
    } else {
      const int r = l16 >> 2;
      const char* at = tile + (slab * 32 + 8 * quarter + r) * (cols * 2) + ((col16 ^ (r | ((quarter & 1) << 2))) * 32) + (lane & 3) * 8;
      typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + 4 * (cols * 2)));
      i32x4 v;
      __builtin_memcpy(&v, &lo, 8);
      __builtin_memcpy(reinterpret_cast<char*>(&v) + 8, &hi, 8);
      return v;
    }
  };
  auto frag_i = [&](const char* st, int f, int slab) -> i32x4 {
    if constexpr (TA) return turned(st, BI, (wi * FI + f), slab);
    const int row = (wi * FI + f) * 16 + l16;
    return *reinterpret_cast<const i32x4*>(st + row * 128 + (((slab * 4 + quarter) ^ swizzle_i(l16)) * 16));
  };
  // The rows of j go to the matrix instructions in an order that leaves a lane 8 neighbouring columns of the output in two
  // accumulators: row m of product f is j = 8 (m / 4) + 4 (f % 2) + m % 4 of its 32.
  auto frag_j = [&](const char* st, int f, int slab) -> i32x4 {
    if constexpr (TB) return turned(st + BI * 128, BJ, (wj * FJ + f), slab);
    const int in32 = 8 * (l16 >> 2) + 4 * (f & 1) + (l16 & 3);
    const int row = (wj * FJ + (f & ~1)) * 16 + in32;
    return *reinterpret_cast<const i32x4*>(st + BI * 128 + row * 128 + (((slab * 4 + quarter) ^ swizzle_j(in32)) * 16));
  };

  Acc acc[FI][FJ];
#pragma unroll
  for (int x = 0; x < FI; ++x)
#pragma unroll
    for (int y = 0; y < FJ; ++y) acc[x][y] = Acc{0, 0, 0, 0};

  if (nc > 0) {
    find_pairs(0);
    if constexpr (FAST) {
      fetch(0, 0);
    } else {
      fetch_regs(0);
      stash(0);
    }
    find_pairs(STEP);
    int buf = 0;
    for (int64_t c0 = 0; c0 < nc; c0 += STEP, buf ^= 1) {
      wait_and_barrier();  // this step has arrived for all, and nobody reads the other half any more
      const bool more = c0 + STEP < nc;
      if (more) {
        if constexpr (FAST) fetch(c0 + STEP, buf ^ 1);
        else fetch_regs(c0 + STEP);
        find_pairs(c0 + 2 * STEP);
      }
      const char* st = smem + buf * STAGE;
#pragma unroll
      for (int slab = 0; slab < 2; ++slab) {
        i32x4 fi[FI], fj[FJ];
#pragma unroll
        for (int y = 0; y < FJ; ++y) fj[y] = frag_j(st, y, slab);
#pragma unroll
        for (int x = 0; x < FI; ++x) fi[x] = frag_i(st, x, slab);
#pragma unroll
        for (int x = 0; x < FI; ++x)
#pragma unroll
          for (int y = 0; y < FJ; ++y) acc[x][y] = Mma<T>::mul(fj[y], fi[x], acc[x][y]);
      }
      if (!FAST && more) stash(buf ^ 1);
    }
  }

  // accumulator register r of a lane: row i = lane % 16, j = 4 (lane / 16) + r of the product (or the order of frag_j)
  const bool whole = (p.ldo | (OP == GRAD_W ? p.stride : 0)) % 8 == 0 && reinterpret_cast<uintptr_t>(p.out) % 16 == 0;
#pragma unroll
  for (int x = 0; x < FI; ++x) {
    const int i = (wi * FI + x) * 16 + l16;
    int64_t row;
    if constexpr (OP == GRAD_W) row = i0 + i < iend ? i0 + i : -1;
    else row = row_pair[i];
    if (row < 0) continue;
    if (OP == GRAD_X && p.named && j0 == 0 && wj == 0 && quarter == 0) p.named[row] = 1;
    float sa = 1.f;
    if constexpr (SZ == 1) sa = p.scale_a[row / p.nprobe];
    const int64_t base = (OP == GRAD_W ? (int64_t)g * p.stride : 0) + row * p.ldo;
    constexpr int RUN = TB ? 4 : 8, PARTS = RUN / 4;  // neighbouring columns of a lane
#pragma unroll
    for (int y = 0; y < FJ; y += PARTS) {
      const int64_t j = j0 + (wj * FJ + y) * 16 + RUN * quarter;
      float v[RUN];
#pragma unroll
      for (int e = 0; e < RUN; ++e) {
        v[e] = (float)acc[x][y + e / 4][e % 4];
        if constexpr (SZ == 1) v[e] = v[e] * sa * p.scale_b[(int64_t)g * p.n + (j + e < width ? j + e : 0)];
      }
      if (whole && j + RUN <= width) {
        if (p.out_dtype == RABITQ_F32) {
#pragma unroll
          for (int e = 0; e < RUN; e += 4)
            *reinterpret_cast<f32x4*>(static_cast<float*>(p.out) + base + j + e) = f32x4{v[e], v[e + 1], v[e + 2], v[e + 3]};
        } else {
          typedef uint16_t h16 __attribute__((ext_vector_type(RUN)));
          h16 h;
#pragma unroll
          for (int e = 0; e < RUN; ++e)
            h[e] = p.out_dtype == RABITQ_F16 ? __builtin_bit_cast(uint16_t, (_Float16)v[e]) : __builtin_bit_cast(uint16_t, (__bf16)v[e]);
          *reinterpret_cast<h16*>(static_cast<uint16_t*>(p.out) + base + j) = h;
        }
      } else {
#pragma unroll
        for (int e = 0; e < RUN; ++e)
          if (j + e < width) store_as(p.out, p.out_dtype, base + j + e, v[e]);
      }
    }
  }
}

}  // namespace rq
