// Products of rows with one weight matrix per expert: segment e of the rows
// (sorted by expert, gathered from x; or every row for every expert) times
// W_e^T, with W_e [N][K], and the two products of its gradient.
//
// k_expert_tile computes one tile of the output.  Operands of every type pass
// through LDS alike, as rows of 128 or 64 bytes of contraction a step (32 or 16
// fp32, 64 or 32 bf16, 256 or 128 4-bit values): 16-byte chunks, one a lane and
// matrix instruction.
// The order of the contraction inside a chunk is free as long as both operands
// share it, so
//   bf16   a chunk is one operand of a 32x32x16 instruction,
//   fp32   its four values feed four 32x32x2 instructions,
//   4 bit  it is one block of 32 values, whose scale is one byte of the lane's
//          scale operand in a 32x32x64 instruction.
// Two buffers hold a step in use and one under way.
#include "gevo_internal.h"
#include "gevo_device.h"
#include "gevo_ops.h"

#include <type_traits>

namespace gevo {

namespace {

typedef int i32x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

// A workgroup's tile: RM x RN waves of (32 MI) x (32 NI), in steps of STEP
// bytes of contraction, WGS workgroups on a CU.
//   Wide   256 x 256, eight waves: per matrix clock of a step 32 bytes of
//          operands from memory to LDS and 96 from LDS to the waves.  The loop
//          takes in 17 a clock without the products (one 8192 x 8192 matrix on
//          8,192 rows in bf16): at most one step is under way, none between
//          the wait for it and the next one's issue.
//   Mid    128 x 128
//   Small  64 x 64: products of few tiles, spread over more of the chip
// Steps of 128 bytes read whole cache lines; Mid takes 64, whose buffers let
// three workgroups share a CU.
template <int RM_, int RN_, int MI_, int NI_, int WGS_, int STEP_>
struct Shape {
  static constexpr int RM = RM_, RN = RN_, MI = MI_, NI = NI_, WGS = WGS_;
  static constexpr int kStep = STEP_;                // bytes of contraction a step
  static constexpr int kThreads = 64 * RM * RN, kWaves = RM * RN;
  static constexpr int kXR = RM * 32 * MI, kWR = RN * 32 * NI;
  static constexpr int kXBytes = kXR * kStep, kWBytes = kWR * kStep;
  static constexpr int kLoadRows = 1024 / kStep;     // of a wave's load
  static constexpr int kXL = kXR / kLoadRows / kWaves, kWL = kWR / kLoadRows / kWaves;   // loads a wave and step
  static constexpr int kScaleBytes = (kXR + kWR) * (kStep / 16);
};
template <ExpertType TY> struct Shapes {
  typedef Shape<4, 2, 2, 4, 1, 128> Wide;
  typedef Shape<2, 2, 2, 2, 3, 64> Mid;
  typedef Shape<2, 2, 1, 1, 4, 128> Small;
};

__device__ uint4 g_zero_chunk;                   // what a chunk outside an operand reads

template <ExpertType TY> struct Mm;
template <> struct Mm<kTypeBf16> {
  typedef uint16_t S;
  template <int B>
  __device__ __forceinline__ static f32x16_t mma(uint4 a, uint4 b, f32x16_t c, uint32_t, uint32_t) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c,
                                                   0, 0, 0);
  }
  __device__ __forceinline__ static f32x4_t mma16(uint4 a, uint4 b, f32x4_t c, uint32_t, uint32_t) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c,
                                                   0, 0, 0);
  }
};
template <> struct Mm<kTypeF32> {
  typedef float S;
  template <int B>
  __device__ __forceinline__ static f32x16_t mma(uint4 a, uint4 b, f32x16_t c, uint32_t, uint32_t) {
    c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.x), __uint_as_float(b.x), c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.y), __uint_as_float(b.y), c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.z), __uint_as_float(b.z), c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.w), __uint_as_float(b.w), c, 0, 0, 0);
  }
  __device__ __forceinline__ static f32x4_t mma16(uint4 a, uint4 b, f32x4_t c, uint32_t, uint32_t) {
    c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.x), __uint_as_float(b.x), c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.y), __uint_as_float(b.y), c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.z), __uint_as_float(b.z), c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.w), __uint_as_float(b.w), c, 0, 0, 0);
  }
};
template <> struct Mm<kTypeMx4> {
  typedef uint8_t S;
  static constexpr int kFp4 = 4;                 // operand format of the scaled instructions
  __device__ __forceinline__ static i32x8_t wide(uint4 a) {
    return i32x8_t{(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0};
  }
  template <int B>                               // B: byte of the scale operands
  __device__ __forceinline__ static f32x16_t mma(uint4 a, uint4 b, f32x16_t c, uint32_t sa, uint32_t sb) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wide(a), wide(b), c, kFp4, kFp4, B, (int)sa, B, (int)sb);
  }
  __device__ __forceinline__ static f32x4_t mma16(uint4 a, uint4 b, f32x4_t c, uint32_t sa, uint32_t sb) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wide(a), wide(b), c, kFp4, kFp4, 0, (int)sa, 0, (int)sb);
  }
};

// Loads straight to LDS from an address per lane: lane l's bytes land at lds +
// 16 l (or 4 l).  Waited for with wait_vm, as dma16.
__device__ __forceinline__ void dma16_at(const void* p, uint32_t lds) {
  asm volatile(
      "s_mov_b32 m0, %1\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %0, off"
      :
      : "v"(p), "s"(lds)
      : "memory");
}
__device__ __forceinline__ void dma4_at(const void* p, uint32_t lds) {
  asm volatile(
      "s_mov_b32 m0, %1\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dword %0, off"
      :
      : "v"(p), "s"(lds)
      : "memory");
}

// A wave-uniform value in a scalar register, wherever the compiler holds it.
// (The wait is for a vector write of v just before, which the compiler does not
// know the lane read of.)
__device__ __forceinline__ uint32_t scalar(uint32_t v) {
  uint32_t s;
  asm volatile("s_nop 1\n\tv_readfirstlane_b32 %0, %1" : "=s"(s) : "v"(v));
  return s;
}

// Chunk c of row r of an operand tile lies at chunk c ^ turn(r) of the row: any
// 8 or 16 consecutive rows then cover the banks once.
template <int STEP>
__device__ __forceinline__ int turn(int r) {
  return STEP == 128 ? (r >> 1) & 7 : ((r & 4) >> 1 | (((r >> 1) ^ (r >> 3)) & 1));
}

// rows of segment e, kept inside [0, S]
__device__ __forceinline__ void segment(const ExpertArgs& a, int e, int64_t& s0, int64_t& cnt) {
  if (!a.offsets) {
    s0 = (int64_t)e * a.M;
    cnt = a.M;
    return;
  }
  const int64_t b = a.offsets[e], n = a.offsets[e + 1];
  s0 = b < 0 ? 0 : (b > a.S ? a.S : b);
  cnt = (n > a.S ? a.S : n) - s0;
  if (cnt < 0) cnt = 0;
}

// row of x that row i of segment e (its first sorted row s0) reads; -1: none
__device__ __forceinline__ int64_t placed_row(const ExpertArgs& a, const int32_t* order, int64_t rows, int64_t r) {
  if (order) {
    const uint32_t slot = (uint32_t)order[r];
    r = a.k > 1 ? __umulhi(slot, a.k_mul) >> a.k_shift : slot;   // slot / k
  }
  return r < rows ? r : -1;
}
__device__ __forceinline__ int64_t source_row(const ExpertArgs& a, int64_t s0, int64_t i) {
  return a.offsets ? placed_row(a, a.order, a.xrows, s0 + i) : i;
}

// Tile idx of rt x nt: eight row tiles at a time, for all column tiles, the row
// tiles fastest.  An XCD's 32 CUs then work on about 8 x 4 tiles, whose 12
// operand tiles are the fewest for 32 (all row tiles first: 33 of them).  A CU
// has only so many lines under way, so what it takes in a clock goes by the time
// a line takes, which a miss in L2 makes long: one 8192 x 8192 matrix on 8,192
// rows in bf16, with its join, 987 us; all row tiles first, 1,107.
struct Place {
  uint32_t row, col;
};
__device__ __forceinline__ Place grouped(uint32_t idx, uint32_t rt, uint32_t nt, uint32_t most = 8) {
  most = min(most, rt);
  const uint32_t g = idx / (most * nt), left = idx - g * (most * nt), here = min(most, rt - g * most);
  return {g * most + left % here, left / here};
}

// Workgroup -> tile of a list, of which XCD j (workgroups with index j mod 8)
// gets the j-th eighth, so that the tiles that read the same operands run near
// each other under one L2.  Routed rows: expert by expert.  Every wave sums the
// experts' tile counts, 64 at a time.
struct Tile {
  int e, nt;
  int64_t s0, cnt, m0;
};
template <int kXR>
__device__ __forceinline__ bool find_tile(const ExpertArgs& a, int ntiles, Tile& o) {
  const int lane = threadIdx.x & 63;
  uint32_t total = 0;
  uint32_t mine = 0, before = 0;                     // of the last 64 experts looked at
  auto look = [&](int base) {                        // returns their sum
    int64_t s0, cnt = 0;
    if (base + lane < a.E) segment(a, base + lane, s0, cnt);
    mine = (uint32_t)((cnt + kXR - 1) / kXR) * (uint32_t)ntiles;
    uint32_t inc = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const uint32_t v = __shfl_up(inc, d, 64);
      if (lane >= d) inc += v;
    }
    before = inc - mine;
    return (uint32_t)__builtin_amdgcn_readlane((int)inc, 63);
  };
  if (a.offsets) {
    for (int b = 0; b < a.E; b += 64) total += look(b);
  } else {
    total = (uint32_t)((a.M + kXR - 1) / kXR) * (uint32_t)ntiles * (uint32_t)a.E;
  }
  const uint32_t each = (total + 7) / 8, at = blockIdx.x >> 3;
  uint32_t idx = (blockIdx.x & 7) * each + at;
  if (at >= each || idx >= total) return false;
  if (!a.offsets) {
    // Every matrix's rows are the same: an eighth of the row tiles goes to each
    // XCD for all matrices, so that these rows stay in its L2 and the matrices
    // pass by (64 variants of 784-512 over 10,000 rows in 4 bits: an eighth of
    // the matrices to each XCD, as where rows differ, takes 5% longer).
    const uint32_t rts = (uint32_t)((a.M + kXR - 1) / kXR), all = (uint32_t)a.E * (uint32_t)ntiles;
    const Place in = grouped(idx, rts, all, a.x_e == 0 ? max(1u, min(8u, (rts + 7) / 8)) : 8);
    const uint32_t c = (uint32_t)__builtin_amdgcn_readfirstlane((int)in.col);
    o.e = (int)(c / (uint32_t)ntiles);
    o.nt = (int)(c % (uint32_t)ntiles);
    o.m0 = (int64_t)__builtin_amdgcn_readfirstlane((int)in.row) * kXR;
    segment(a, o.e, o.s0, o.cnt);
    return true;
  } else {
    for (int b = 0;; b += 64) {
      if (b >= a.E) return false;
      const uint32_t sum = a.E > 64 ? look(b) : total;   // (up to 64: still in the lanes)
      if (idx < sum) {
        const uint64_t in = __ballot(idx >= before && idx < before + mine);
        if (in == 0) return false;                   // (offsets of no plan, whose counts pass 32 bits)
        const int l = __ffsll((unsigned long long)in) - 1;
        o.e = b + l;
        idx -= (uint32_t)__builtin_amdgcn_readlane((int)before, __builtin_amdgcn_readfirstlane(l));
        break;
      }
      idx -= sum;
    }
  }
  o.e = __builtin_amdgcn_readfirstlane(o.e);
  idx = (uint32_t)__builtin_amdgcn_readfirstlane((int)idx);
  segment(a, o.e, o.s0, o.cnt);
  const uint32_t rt = (uint32_t)((o.cnt + kXR - 1) / kXR);
  const Place in = grouped(idx, rt, (uint32_t)ntiles);
  o.nt = __builtin_amdgcn_readfirstlane((int)in.col);
  o.m0 = (int64_t)__builtin_amdgcn_readfirstlane((int)in.row) * kXR;
  return true;
}

// The elements of a row's last 16 bytes u from the drop-th on, then zeros.
template <typename S>
__device__ __forceinline__ uint4 without_first(uint4 u, int drop) {
  if (sizeof(S) == 2 && (drop & 1))
    u = make_uint4(__builtin_amdgcn_alignbit(u.y, u.x, 16), __builtin_amdgcn_alignbit(u.z, u.y, 16),
                   __builtin_amdgcn_alignbit(u.w, u.z, 16), u.w >> 16);
  const int d = sizeof(S) == 2 ? drop >> 1 : drop;
  if (d & 1) u = make_uint4(u.y, u.z, u.w, 0);
  if (d & 2) u = make_uint4(u.z, u.w, 0, 0);
  return u;
}

// 16 bytes at p, which has its element's alignment, of which the first `valid`
// elements exist (at most 0: none, and zeros).  edge: some lane's chunk may be
// the last, partly filled one of its row; it is then read as the row's last 16
// bytes, less the elements before it.  Rows of less than 16 bytes (not wide) are
// read element by element.  Loads of absent chunks go to `safe`, so that no
// lane branches and all of a wave's loads are under way together.
template <typename S>
__device__ __forceinline__ uint4 load_chunk(const char* p, int valid, bool edge, bool wide, const char* safe) {
  constexpr int V = 16 / sizeof(S);
  uint4 u;
  if (!wide) {
    S e[V];
#pragma unroll
    for (int i = 0; i < V; ++i) e[i] = i < valid ? reinterpret_cast<const S*>(p)[i] : (S)0;
    __builtin_memcpy(&u, e, 16);
    return u;
  }
  const int drop = edge && valid < V ? V - valid : 0;
  __builtin_memcpy(&u, valid > 0 ? p - drop * (int)sizeof(S) : safe, 16);   // one load, at any address
  if (edge) u = without_first<S>(u, drop);
  return valid > 0 ? u : make_uint4(0, 0, 0, 0);
}

enum Load { kDma, kGuarded, kNatural, kNaturalGuarded };
constexpr bool by_index(Load l) { return l == kNatural || l == kNaturalGuarded; }
enum Pass { kForward, kDx, kDw };

}  // namespace

// Tiles of a product.  XL, WL: how the operand tiles reach LDS.
//   kDma         16-byte chunks straight to LDS, a step ahead
//   kGuarded     through registers, at any address, where rows are not aligned
//                or the contraction ends inside a chunk
//   kNatural     the contraction is the operand's outer index: rows of one
//                contraction index each, straight to LDS; bf16 operands are read
//                with gfx950's transposing LDS read (each 16 lanes a 4 x 16 block
//                by columns), fp32 ones value by value
//   kNaturalGuarded  the same through registers, at any address or width
template <typename SH, ExpertType TY, Pass PASS, Load XL, Load WL, bool OUT16>
__global__ __launch_bounds__(SH::kThreads, SH::WGS* SH::kThreads / 256) void k_expert_tile(ExpertArgs a) {
  typedef Mm<TY> M;
  typedef typename M::S S;
  typedef typename std::conditional<OUT16, uint16_t, float>::type O;
  constexpr int kXR = SH::kXR, kWR = SH::kWR, kXBytes = SH::kXBytes, kWBytes = SH::kWBytes;
  constexpr int MI = SH::MI, NI = SH::NI, NXL = SH::kXL, NWL = SH::kWL, kLR = SH::kLoadRows;
  constexpr int V = 16 / sizeof(S);                  // elements a chunk (not of 4-bit operands)
  constexpr int kStep = SH::kStep, kC = kStep / 16, kQ = kStep / 32;   // chunks, parts of a step
  constexpr bool mx = TY == kTypeMx4;
  constexpr int kBuf = kXBytes + kWBytes + (mx ? SH::kScaleBytes : 0);
  constexpr bool kAllDma = (XL == kDma || XL == kNatural) && (WL == kDma || WL == kNatural);
  constexpr int kXi = XL == kDma || XL == kNatural ? NXL : 0, kWi = WL == kDma || WL == kNatural ? NWL : 0;
  constexpr int kIssued = kXi + kWi + (mx ? kC / 4 : 0);   // loads straight to LDS a step and wave
  extern __shared__ __align__(16) char smem[];

  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l32 = lane & 31, lh = lane >> 5;
  const int wu = __builtin_amdgcn_readfirstlane(wave);
  // the wave's band of rows and of columns; the waves of a band sit on
  // different SIMDs, so bands without rows leave their share to the others
  const int wm = wu / SH::RN, wn = wu % SH::RN;
  const uint32_t lds0 = lds_addr(smem);
  const int cols = PASS == kDw ? a.K : a.N;          // of the output
  const int bytes = mx ? (a.K + 127) / 128 * 64 : a.K * (int)sizeof(S);   // of a contraction row (not kDw)
  constexpr int kPer = mx ? 2 * kStep : kStep / (int)sizeof(S);           // elements a step

  Tile tl;
  if constexpr (PASS == kDw) {
    // tiles of every expert's [N][K] gradient; x operand: columns of dy, w operand: columns of x
    const int nr = (a.N + kXR - 1) / kXR, nc = (a.K + kWR - 1) / kWR;
    const uint32_t total = (uint32_t)a.E * (uint32_t)(nr * nc), each = (total + 7) / 8;
    const uint32_t at = blockIdx.x >> 3, idx = (blockIdx.x & 7) * each + at;
    if (at >= each || idx >= total) return;
    tl.e = (int)(idx / (uint32_t)(nr * nc));
    const Place in = grouped(idx % (uint32_t)(nr * nc), (uint32_t)nr, (uint32_t)nc);
    tl.nt = (int)in.col;
    tl.m0 = (int64_t)in.row * kXR;
    segment(a, tl.e, tl.s0, tl.cnt);
  } else {
    if (!find_tile<kXR>(a, (a.N + kWR - 1) / kWR, tl)) return;
  }
  const int n0 = tl.nt * kWR;
  const int64_t rows = PASS == kDw ? a.N : tl.cnt;
  const bool has_rows = tl.m0 + wm * 32 * MI < rows && n0 + wn * 32 * NI < cols;   // the wave's part of the output
  const int64_t clen = PASS == kDw ? tl.cnt : a.K;   // contraction, elements
  const int nst = (int)((clen + kPer - 1) / kPer);   // steps

  // ---- chunks in row order: a load's rows follow each other, kC lanes a row.
  // A row's turn is the same in every second load.
  const int crow = lane / kC;
  const int cb[2] = {16 * ((lane % kC) ^ turn<kStep>(crow)), 16 * ((lane % kC) ^ turn<kStep>(kLR + crow))};
  const char* xp[NXL];
  const char* wp[NWL];
  uint32_t have = 0;                                 // bit j: load j of x has a row, bit 16 + j: of w
  const char* zero = (const char*)&g_zero_chunk;
  bool there = true;                                 // the lane's rows that have a place have a source
  bool have_s = false;
  const char* sp = nullptr;                          // 4-bit operands: a wave loads 64 rows' scales
  constexpr int kSx = kXR / 64, kSn = (kXR + kWR) / 64;
  const int sj = wu % kSn;
  static_assert(!mx || SH::kWaves >= kSn, "every row's scales have a wave");

  {
    if constexpr (XL == kDma || XL == kGuarded) {
#pragma unroll
      for (int j = 0; j < NXL; ++j) {
        const int64_t i = tl.m0 + kLR * (NXL * wave + j) + crow;
        int64_t r = i < tl.cnt ? source_row(a, tl.s0, i) : -1;
        if (r >= 0) {
          have |= 1u << j;
        } else {
          there &= i >= tl.cnt;
          r = 0;
        }
        xp[j] = (const char*)a.x + (a.offsets ? 0 : tl.e * a.x_e) + r * a.x_stride + cb[j & 1];
      }
    }
    if constexpr (WL == kDma || WL == kGuarded) {
#pragma unroll
      for (int j = 0; j < NWL; ++j) {
        const int n = n0 + kLR * (NWL * wave + j) + crow;
        if (n < a.N) have |= 0x10000u << j;
        wp[j] = (const char*)a.w + tl.e * a.w_e + (n < a.N ? n : 0) * a.w_n + cb[j & 1];
      }
    }
    if constexpr (mx) {
      if (sj < kSx) {
        const int64_t i = tl.m0 + 64 * sj + lane;
        const int64_t r = i < tl.cnt ? source_row(a, tl.s0, i) : -1;
        have_s = r >= 0;
        there &= have_s || i >= tl.cnt;
        sp = (const char*)a.xs + (a.offsets ? 0 : tl.e * a.xs_e) + (have_s ? r : 0) * a.xs_stride;
      } else {
        const int n = n0 + 64 * (sj - kSx) + lane;
        have_s = n < a.N;
        sp = (const char*)a.ws + tl.e * a.ws_e + (have_s ? n : 0) * a.ws_n;
      }
    }
  }

  // ---- natural order: a load's 1,024 bytes are 1,024 / kRowBytes rows of one
  // contraction index each.  So that the reads below cover the banks, 64-byte
  // blocks of bf16 rows change places with the index mod 4 (rows of 128 bytes:
  // with its second bit), 128-byte blocks of fp32 rows with its third bit.
  struct Natural {                                   // of one operand
    const char* base;                                // contraction row 0
    int64_t stride;
    int row0, per;                                   // the lane's row in the wave's first load; rows a load
    int cb[2];                                       // its column's byte in even and odd loads, -1: none
    int drop[2], valid[2];                           // elements of the chunk before that column; that exist
    const char* first[2];                            // that column's address in the lane's first row (gathered: row 0)
    int64_t load, step;                              // bytes between the rows of two loads, of two steps
  } nx{}, nw{};
  auto natural_block = [](int tile_bytes, int row) {  // what the row's 16-byte chunks are xored with
    if (sizeof(S) == 4) return ((row >> 2) & 1) << 3;
    return (tile_bytes == 128 ? (row >> 1) & 1 : row & 3) << 2;
  };
  auto natural_setup = [&](Natural& d, const char* base, int64_t stride, int tile_rows, int loads, int col0, int width,
                           bool guarded, bool placed) {
    const int tb = tile_rows * (int)sizeof(S);       // bytes of a tile's row
    d.base = base;
    d.stride = stride;
    d.per = 1024 / tb;
    d.row0 = loads * wave * d.per + lane / (tb / 16);
#pragma unroll
    for (int v = 0; v < 2; ++v) {
      const int ch = lane % (tb / 16) ^ natural_block(tb, d.row0 + v * d.per);
      const int c = col0 * (int)sizeof(S) + 16 * ch;
      const int over = c + 16 - width * (int)sizeof(S);   // as below
      d.drop[v] = over > 0 && over < 16 ? over / (int)sizeof(S) : 0;
      d.valid[v] = over < 16 ? V - (over > 0 ? over / (int)sizeof(S) : 0) : 0;
      d.cb[v] = over >= 16 ? -1 : guarded ? c : c - (over > 0 ? over : 0);
      d.first[v] = base + (placed ? 0 : d.row0 * stride) + (d.cb[v] < 0 ? 0 : d.cb[v]);
    }
    d.load = d.per * stride;
    d.step = kPer * stride;
  };
  if constexpr (by_index(XL))                        // dw: columns of dy
    natural_setup(nx, (const char*)a.w + tl.s0 * a.w_n, a.w_n, kXR, NXL, (int)tl.m0, a.N, XL != kNatural, false);
  if constexpr (by_index(WL)) {
    if constexpr (PASS == kDw) natural_setup(nw, (const char*)a.x, a.x_stride, kWR, NWL, n0, a.K, WL != kNatural, true);
    else natural_setup(nw, (const char*)a.w + tl.e * a.w_e, a.w_n, kWR, NWL, n0, a.N, WL != kNatural, false);
  }
  int32_t gathered[PASS == kDw ? NWL : 1];   // rows of x that the next step's loads read
  auto gather = [&](int st) {
    if constexpr (PASS == kDw) {
#pragma unroll
      for (int n = 0; n < NWL; ++n) {
        const int64_t k = (int64_t)st * kPer + nw.row0 + n * nw.per;
        gathered[n] = k < clen ? (int32_t)source_row(a, tl.s0, k) : -1;
      }
    }
  };

  // load n of the wave's kIssued loads of step st, to buffer b
  auto issue_one = [&](int st, int b, int n) {
    const uint32_t buf = scalar(lds0 + (uint32_t)b * kBuf);
    const int at = st * kStep;
    if (n < kXi) {
      const uint32_t to = buf + (uint32_t)(NXL * wu + n) * 1024u;
      if constexpr (XL == kDma) {
        const int over = at + cb[n & 1] + 16 - bytes;  // bytes of the chunk past the row
        dma16_at((have >> n & 1) && over < 16 ? xp[n] + at - (over > 0 ? over : 0) : zero, to);
      } else {
        const int64_t k = (int64_t)st * kPer + nx.row0 + n * nx.per;
        dma16_at(k < clen && nx.cb[n & 1] >= 0 ? nx.base + k * nx.stride + nx.cb[n & 1] : zero, to);
      }
      return;
    }
    n -= kXi;
    if (n < kWi) {
      const uint32_t to = buf + kXBytes + (uint32_t)(NWL * wu + n) * 1024u;
      if constexpr (WL == kDma) {
        const int over = at + cb[n & 1] + 16 - bytes;
        dma16_at((have >> (16 + n) & 1) && over < 16 ? wp[n] + at - (over > 0 ? over : 0) : zero, to);
      } else {
        int64_t k = (int64_t)st * kPer + nw.row0 + n * nw.per;
        if constexpr (PASS == kDw) k = gathered[n];
        else if (k >= clen) k = -1;
        dma16_at(k >= 0 && nw.cb[n & 1] >= 0 ? nw.base + k * nw.stride + nw.cb[n & 1] : zero, to);
      }
      return;
    }
    n -= kWi;
    if constexpr (mx)
      dma4_at(have_s && st * kC + n * 4 < bytes / 16 ? sp + st * kC + n * 4 : zero,
              buf + kXBytes + kWBytes + (uint32_t)n * (kXR + kWR) * 4u + (uint32_t)sj * 256u);
  };
  // The same where step st lies inside every operand and no row is out of place:
  // an address a load, without a look at what exists (which took 30 instructions
  // a load: 8,192 rows through 4 of 64 experts of 2048 x 2048 3% longer).
  // Rows and columns outside the operands read the first ones, and their products
  // are not written.
  const bool plain = kAllDma && __all(there);
  auto inside = [&](int st) {
    bool in = plain && st < nst;
    if constexpr (by_index(XL) || by_index(WL)) in = in && (int64_t)(st + 1) * kPer <= clen;
    if constexpr (PASS != kDw) in = in && (st + 1) * kStep <= bytes;
    if constexpr (PASS == kDw) {
      int32_t low = gathered[0];
#pragma unroll
      for (int n = 1; n < NWL; ++n) low = min(low, gathered[n]);
      in = in && __all(low >= 0);
    }
    return in;
  };
  auto issue_inside = [&](int st, int b, int n) {
    const uint32_t buf = (uint32_t)__builtin_amdgcn_readfirstlane((int)(lds0 + (uint32_t)b * kBuf));
    if (n < kXi) {
      const uint32_t to = buf + (uint32_t)(NXL * wu + n) * 1024u;
      if constexpr (XL == kDma) dma16_at(xp[n] + (int64_t)st * kStep, to);
      else dma16_at(nx.first[n & 1] + (st * nx.step + n * nx.load), to);
      return;
    }
    n -= kXi;
    if (n < kWi) {
      const uint32_t to = buf + kXBytes + (uint32_t)(NWL * wu + n) * 1024u;
      if constexpr (WL == kDma) dma16_at(wp[n] + (int64_t)st * kStep, to);
      else if constexpr (PASS == kDw) dma16_at(nw.first[n & 1] + (uint32_t)gathered[n] * nw.stride, to);
      else dma16_at(nw.first[n & 1] + (st * nw.step + n * nw.load), to);
      return;
    }
    n -= kWi;
    if constexpr (mx)
      dma4_at(sp + (int64_t)st * kC + n * 4, buf + kXBytes + kWBytes + (uint32_t)n * (kXR + kWR) * 4u + (uint32_t)sj * 256u);
  };
  auto issue = [&](int st, int b) {
    if (inside(st)) {
#pragma unroll
      for (int n = 0; n < kIssued; ++n) issue_inside(st, b, n);
      return;
    }
#pragma unroll
    for (int n = 0; n < kIssued; ++n) issue_one(st, b, n);
  };

  // A row's last chunk, where the row ends inside it, has been loaded as the
  // row's last 16 bytes: once they are there, the lane that loaded them puts them
  // in place.  (Rows of one contraction index: in every step of the last tile.)
  const bool ends_x = !mx && XL == kDma && bytes % 16 != 0, ends_w = !mx && WL == kDma && bytes % 16 != 0;
  const bool edge_x = XL == kNatural && tl.m0 + kXR > a.N && a.N * (int)sizeof(S) % 16 != 0;
  const bool edge_w = WL == kNatural && n0 + kWR > cols && cols * (int)sizeof(S) % 16 != 0;
  auto settle = [&](int st, int b) {
    if constexpr (mx) return;
    auto move = [&](int at, int drop) {
      if (drop > 0 && drop < V) {
        uint4* q = reinterpret_cast<uint4*>(smem + at + lane * 16);
        *q = without_first<S>(*q, drop);
      }
    };
    const bool last = (st + 1) * kStep > bytes;
    const int xat = b * kBuf + NXL * wu * 1024, wat = b * kBuf + kXBytes + NWL * wu * 1024;
    if ((ends_x && last) || edge_x) {
#pragma unroll
      for (int n = 0; n < NXL; ++n)
        move(xat + n * 1024, XL == kNatural ? nx.drop[n & 1] : (st * kStep + cb[n & 1] + 16 - bytes) / (int)sizeof(S));
    }
    if ((ends_w && last) || edge_w) {
#pragma unroll
      for (int n = 0; n < NWL; ++n)
        move(wat + n * 1024, WL == kNatural ? nw.drop[n & 1] : (st * kStep + cb[n & 1] + 16 - bytes) / (int)sizeof(S));
    }
  };

  // ---- through registers: step st from memory, and to buffer b
  constexpr bool kXg = XL == kGuarded || XL == kNaturalGuarded, kWg = WL == kGuarded || WL == kNaturalGuarded;
  uint4 xg[kXg ? NXL : 1], wg[kWg ? NWL : 1];
  const bool nat_edge = n0 + kWR > cols || (PASS == kDw && tl.m0 + kXR > a.N);   // some chunk may be partly filled
  auto fetch = [&](int st) {
    const int at = st * kStep;
    auto by_row = [&](const char* p, bool in, int n, const void* safe) {
      return load_chunk<S>(p + at, in ? (bytes - at - cb[n & 1]) / (int)sizeof(S) : 0, at + kStep > bytes, bytes >= 16,
                           (const char*)safe);
    };
    auto by_column = [&](const Natural& d, int64_t k, int n, int width, const void* safe) {
      const bool in = k >= 0 && d.cb[n & 1] >= 0;
      return load_chunk<S>(d.base + (in ? k * d.stride + d.cb[n & 1] : 0), in ? d.valid[n & 1] : 0, nat_edge, width >= V,
                           (const char*)safe);
    };
    if constexpr (kXg) {
#pragma unroll
      for (int n = 0; n < NXL; ++n) {
        if constexpr (XL == kGuarded) {
          xg[n] = by_row(xp[n], have >> n & 1, n, a.x);
        } else {
          const int64_t k = (int64_t)st * kPer + nx.row0 + n * nx.per;
          xg[n] = by_column(nx, k < clen ? k : -1, n, a.N, a.w);
        }
      }
    }
    if constexpr (kWg) {
#pragma unroll
      for (int n = 0; n < NWL; ++n) {
        if constexpr (WL == kGuarded) {
          wg[n] = by_row(wp[n], have >> (16 + n) & 1, n, a.w);
        } else {
          int64_t k = (int64_t)st * kPer + nw.row0 + n * nw.per;
          if constexpr (PASS == kDw) k = gathered[n];
          else if (k >= clen) k = -1;
          wg[n] = by_column(nw, k, n, cols, PASS == kDw ? a.x : a.w);
        }
      }
    }
  };
  auto put = [&](int b) {
    char* buf = smem + b * kBuf + lane * 16;
    if constexpr (kXg) {
#pragma unroll
      for (int n = 0; n < NXL; ++n) *reinterpret_cast<uint4*>(buf + (NXL * wave + n) * 1024) = xg[n];
    }
    if constexpr (kWg) {
#pragma unroll
      for (int n = 0; n < NWL; ++n) *reinterpret_cast<uint4*>(buf + kXBytes + (NWL * wave + n) * 1024) = wg[n];
    }
  };

  // The tile is accumulated transposed (w operand's rows down): lane l holds
  // row 32 i + l % 32 of the wave's band and, in registers 4 q + r, columns
  // 32 t + 8 q + 4 (l / 32) + r.
  //
  // A step has kQ parts of one chunk a lane and operand.  Each part's operands
  // are read while the part before is multiplied, so the step's barrier sits
  // before its last part: by then every wave has read the whole step, whose
  // buffer takes a later step's load, and the next step has landed.
  f32x16_t acc[MI][NI];
  struct Frag {
    uint4 x[MI], w[NI];
  } fr[2];
  uint32_t sx[2][MI], sw[2][NI];                     // scales: of two parts, and the next two's
#pragma unroll
  for (int b = 0; b < 2; ++b) {
#pragma unroll
    for (int i = 0; i < MI; ++i) sx[b][i] = 0;
#pragma unroll
    for (int t = 0; t < NI; ++t) sw[b][t] = 0;
  }
  const int tr = turn<kStep>(l32);
  const char* xb = smem + (wm * 32 * MI + l32) * kStep;
  const char* wb = smem + kXBytes + (wn * 32 * NI + l32) * kStep;
  // the 32 rows (of the tile) from 32 t on, at part h, of an operand in natural order
  auto read_natural = [&](int from, int tile_rows, int t, int h) -> uint4 {
    const int tb = tile_rows * (int)sizeof(S);
    uint4 u;
    if constexpr (sizeof(S) == 4) {
      const char* p = smem + from + (8 * h + 4 * lh) * tb + ((t ^ lh) << 7) + l32 * 4;
      u.x = *reinterpret_cast<const uint32_t*>(p);
      u.y = *reinterpret_cast<const uint32_t*>(p + tb);
      u.z = *reinterpret_cast<const uint32_t*>(p + 2 * tb);
      u.w = *reinterpret_cast<const uint32_t*>(p + 3 * tb);
    } else {
      // 16 lanes read 16 columns of four contraction rows, four lanes a row, and
      // get a column's four values each
      typedef short s16x4_t __attribute__((ext_vector_type(4)));
      typedef __attribute__((address_space(3))) s16x4_t* Ptr;
      const int r = (lane & 15) >> 2, row = 16 * h + 8 * lh + r;
      const int block = tb == 128 ? t ^ (r >> 1) : t ^ r;
      const char* p = smem + from + row * tb + (block << 6) + ((lane >> 4) & 1) * 32 + (lane & 3) * 8;
      const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Ptr)p);
      const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Ptr)(p + 4 * tb));
      const uint2 l2 = __builtin_bit_cast(uint2, lo), h2 = __builtin_bit_cast(uint2, hi);
      u = make_uint4(l2.x, l2.y, h2.x, h2.y);
    }
    return u;
  };
  auto read_x = [&](int b, int h) {
    if constexpr (by_index(XL)) {
#pragma unroll
      for (int i = 0; i < MI; ++i) fr[h & 1].x[i] = read_natural(b * kBuf, kXR, wm * MI + i, h);
      return;
    }
    const int at = b * kBuf + 16 * ((2 * h + lh) ^ tr);
#pragma unroll
    for (int i = 0; i < MI; ++i) fr[h & 1].x[i] = *reinterpret_cast<const uint4*>(xb + at + 32 * i * kStep);
    if constexpr (mx) {
      if ((h & 1) == 0) {
        const uint32_t* sc =
            reinterpret_cast<const uint32_t*>(smem + b * kBuf + kXBytes + kWBytes) + (h >> 1) * (kXR + kWR);
#pragma unroll
        for (int i = 0; i < MI; ++i) sx[1][i] = sc[wm * 32 * MI + 32 * i + l32] >> (8 * lh);
#pragma unroll
        for (int t = 0; t < NI; ++t) sw[1][t] = sc[kXR + wn * 32 * NI + 32 * t + l32] >> (8 * lh);
      }
    }
  };
  auto read_w = [&](int b, int h, int t) {
    if constexpr (by_index(WL)) {
      fr[h & 1].w[t] = read_natural(b * kBuf + kXBytes, kWR, wn * NI + t, h);
      return;
    }
    const int at = b * kBuf + 16 * ((2 * h + lh) ^ tr);
    fr[h & 1].w[t] = *reinterpret_cast<const uint4*>(wb + at + 32 * t * kStep);
  };
  auto mul = [&](auto hc, int t) {
    constexpr int h = decltype(hc)::value;
#pragma unroll
    for (int i = 0; i < MI; ++i)
      acc[i][t] = M::template mma<2 * h>(fr[h].w[t], fr[h].x[i], acc[i][t], sw[0][t], sx[0][i]);
  };
  // dw: sums of dy's columns, a lane's share of its row of the x operand
  constexpr bool kSums = PASS == kDw;
  float col_sum[kSums ? MI : 1];
  auto add_columns = [&](int h) {
    if constexpr (kSums) {
#pragma unroll
      for (int i = 0; i < MI; ++i) {
        S e[V];
        __builtin_memcpy(e, &fr[h].x[i], 16);
#pragma unroll
        for (int v = 0; v < V; ++v) col_sum[i] += Op<S>::to_f32(e[v]);
      }
    }
  };
  auto next_scales = [&]() {
    if constexpr (mx) {
#pragma unroll
      for (int i = 0; i < MI; ++i) sx[0][i] = sx[1][i];
#pragma unroll
      for (int t = 0; t < NI; ++t) sw[0][t] = sw[1][t];
    }
  };

  // output: rows of the wave's band pass through the wave's own part of LDS 32
  // at a time, so that they leave in segments of up to 256 bytes
  constexpr int kFit = kXBytes + kWBytes >= SH::kWaves * 32 * 256 ? 256 : 128;
  constexpr int kRowB = NI * 32 * (int)sizeof(O) < kFit ? NI * 32 * (int)sizeof(O) : kFit;   // bytes of a row a round
  constexpr int kTs = kRowB / (32 * (int)sizeof(O));                                         // column tiles a round
  constexpr int kCh = kRowB / 16, kEl = 16 / (int)sizeof(O);
  static_assert(SH::kWaves * 32 * kRowB <= kXBytes + kWBytes, "the output's staging fits a buffer");
  float* bs = reinterpret_cast<float*>(smem + 2 * kBuf);       // the tile's biases, which the sums start from
  const bool whole = ((cols | (int)(a.out_stride % kEl)) & (kEl - 1)) == 0 && (uintptr_t)a.out % 16 == 0;

  const bool sums = PASS == kDw && a.db && tl.nt == 0;
  const bool adds = kSums && sums && wn == 0;
#pragma unroll
  for (int i = 0; i < (kSums ? MI : 1); ++i) col_sum[i] = 0.0f;
  float bias = 0.0f;
  if (PASS == kForward && a.bias && tid < kWR && n0 + tid < a.N) bias = a.bias[(int64_t)tl.e * a.N + n0 + tid];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int t = 0; t < NI; ++t) acc[i][t] = zero16();

  if (nst > 0) {
    gather(0);
    issue(0, 0);
    if constexpr (!kAllDma) {
      fetch(0);
      put(0);
    }
    if (nst > 1) {
      gather(1);
      if constexpr (!kAllDma) fetch(1);
      issue(1, 1);
    }
    if (nst > 1) wait_vm<kIssued>();
    else wait_vm<0>();
    settle(0, 0);
    if (PASS == kForward && tid < kWR) bs[tid] = bias;
    __syncthreads();
    if (has_rows) {
      if constexpr (PASS == kForward) {
#pragma unroll
        for (int t = 0; t < NI; ++t)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const float4 c = *reinterpret_cast<const float4*>(bs + wn * 32 * NI + 32 * t + 8 * q + 4 * lh);
            acc[0][t][4 * q] = c.x;
            acc[0][t][4 * q + 1] = c.y;
            acc[0][t][4 * q + 2] = c.z;
            acc[0][t][4 * q + 3] = c.w;
          }
#pragma unroll
        for (int i = 1; i < MI; ++i)
#pragma unroll
          for (int t = 0; t < NI; ++t) acc[i][t] = acc[0][t];
      }
      read_x(0, 0);
#pragma unroll
      for (int t = 0; t < NI; ++t) read_w(0, 0, t);
    }
    for (int st = 0; st < nst; ++st) {
      const int b = st & 1;
      const bool more = st + 1 < nst, ahead = st + 2 < nst;
      // parts that hold a value (of 4-bit rows, whose last step is often half empty)
      const int filled = mx && !more ? (bytes - st * kStep + 31) / 32 : kQ;
      auto part = [&](auto hc) {                     // part h, reading part h + 1 of the step
        constexpr int h = decltype(hc)::value;
        if (mx && h >= filled) return;
        if ((h & 1) == 0) next_scales();
        read_x(b, h + 1);
#pragma unroll
        for (int t = 0; t < NI; ++t) {
          read_w(b, h + 1, t);
          mul(std::integral_constant<int, h & 1>{}, t);
          __builtin_amdgcn_sched_barrier(0);
        }
        if (adds) add_columns(h & 1);
      };
      if (ahead) gather(st + 2);                     // ahead of the loads that go by it
      if (has_rows) {
        part(std::integral_constant<int, 0>{});
        if constexpr (kQ == 4) {
          part(std::integral_constant<int, 1>{});
          part(std::integral_constant<int, 2>{});
        }
      }
      if constexpr (!kAllDma) {
        if (more) put(b ^ 1);
      }
      wait_vm<0>();
      if (more) settle(st + 1, b ^ 1);
      __syncthreads();
      if constexpr (!kAllDma) {
        if (ahead) fetch(st + 2);
      }
      if (has_rows && (!mx || filled == kQ)) {
        if (adds) add_columns(1);
        const bool in = inside(st + 2);
        if (more) read_x(b ^ 1, 0);
#pragma unroll
        for (int t = 0; t < NI; ++t) {
          if (more) read_w(b ^ 1, 0, t);
          mul(std::integral_constant<int, 1>{}, t);
          if (in) {
#pragma unroll
            for (int n = t * kIssued / NI; n < (t + 1) * kIssued / NI; ++n) issue_inside(st + 2, b, n);
          } else if (ahead) {
#pragma unroll
            for (int n = t * kIssued / NI; n < (t + 1) * kIssued / NI; ++n) issue_one(st + 2, b, n);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      } else if (ahead) {
        issue(st + 2, b);
      }
    }
  }

  if constexpr (kSums) {
    if (adds && has_rows) {
#pragma unroll
      for (int i = 0; i < MI; ++i) {
        const float sum = col_sum[i] + __shfl_xor(col_sum[i], 32, 64);
        const int64_t c = tl.m0 + wm * 32 * MI + 32 * i + l32;
        if (lh == 0 && c < a.N) a.db[(int64_t)tl.e * a.N + c] = sum;
      }
    }
  }

  // ---- output
  __syncthreads();                                 // every wave is past its reads of the buffers
  if (has_rows) {
    char* stage = smem + wu * 32 * kRowB;
    const float least = PASS == kForward && a.relu ? 0.0f : -INFINITY;
    // all of the wave's part of the output exists and its chunks lie on 16 bytes
    const bool filled = whole && !(PASS == kDx && a.mask) && tl.m0 + (wm + 1) * 32 * MI <= rows &&
                        n0 + (wn + 1) * 32 * NI <= cols;
    // the lane's row and column in the first of the band's rounds
    const int64_t r0 = tl.m0 + wm * 32 * MI + lane / kCh;
    const int c0 = n0 + wn * 32 * NI + lane % kCh * kEl;
    O* const o0 = (O*)a.out + (PASS == kDw ? (int64_t)tl.e * a.N + r0 : tl.s0 + r0) * a.out_stride + c0;
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int t0 = 0; t0 < NI; t0 += kTs) {
#pragma unroll
        for (int t = t0; t < t0 + kTs; ++t)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            float f[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) f[u] = acc[i][t][4 * q + u];
            if constexpr (PASS == kForward) {
#pragma unroll
              for (int u = 0; u < 4; ++u) f[u] = __builtin_elementwise_maximum(f[u], least);   // (NaN stays)
            }
            char* row = stage + l32 * kRowB;
            if constexpr (OUT16) {                 // chunk 4 t + q, half lh
              const int ch = (4 * (t - t0) + q) ^ (l32 & (kCh - 1));
              *reinterpret_cast<uint2*>(row + 16 * ch + 8 * lh) = make_uint2(bf16x2(f[0], f[1]), bf16x2(f[2], f[3]));
            } else {
              const int ch = (8 * (t - t0) + 2 * q + lh) ^ (l32 & (kCh - 1));
              *reinterpret_cast<float4*>(row + 16 * ch) = make_float4(f[0], f[1], f[2], f[3]);
            }
          }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (filled) {                              // no lane looks at what exists
          uint4 u[kCh / 2];
#pragma unroll
          for (int j = 0; j < kCh / 2; ++j) {
            const int rr = j * (64 / kCh) + lane / kCh;
            u[j] = *reinterpret_cast<const uint4*>(stage + rr * kRowB + 16 * (lane % kCh ^ (rr & (kCh - 1))));
          }
#pragma unroll
          for (int j = 0; j < kCh / 2; ++j)
            *reinterpret_cast<uint4*>(o0 + ((32 * i + j * (64 / kCh)) * a.out_stride + 32 * t0)) = u[j];
          __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
          continue;
        }
#pragma unroll
        for (int j = 0; j < kCh / 2; ++j) {        // 64 / kCh rows an instruction
          const int rr = j * (64 / kCh) + lane / kCh, ch = lane % kCh;
          uint4 u = *reinterpret_cast<const uint4*>(stage + rr * kRowB + 16 * (ch ^ (rr & (kCh - 1))));
          const int64_t r = r0 + (32 * i + j * (64 / kCh));
          const int c = c0 + 32 * t0;
          if (r >= rows || c >= cols) continue;
          if constexpr (PASS == kDx && !mx) {
            if (a.mask) {
              const int64_t mr = placed_row(a, a.mask_order, a.mask_rows, tl.s0 + r);
              const char* mp = (const char*)a.mask + (mr < 0 ? 0 : mr) * a.mask_stride + (size_t)c * sizeof(S);
              const uint4 mu =               // (a row outside x: zeros)
                  load_chunk<S>(mp, mr < 0 ? 0 : cols - c, n0 + kWR > cols, cols >= V, (const char*)a.mask);
              S me[V];
              O oe[kEl];
              static_assert(PASS != kDx || V == kEl, "dx has its input's type");
              __builtin_memcpy(me, &mu, 16);
              __builtin_memcpy(oe, &u, 16);
#pragma unroll
              for (int v = 0; v < kEl; ++v)
                if (!(Op<S>::to_f32(me[v]) > 0.0f)) oe[v] = 0;
              __builtin_memcpy(&u, oe, 16);
            }
          }
          O* o = o0 + ((32 * i + j * (64 / kCh)) * a.out_stride + 32 * t0);
          if (whole) {
            *reinterpret_cast<uint4*>(o) = u;
          } else {
            O oe[kEl];
            __builtin_memcpy(oe, &u, 16);
#pragma unroll
            for (int v = 0; v < kEl; ++v)
              if (c + v < cols) o[v] = oe[v];
          }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      }
  }
}

// Few rows a segment: the weights' bytes are the time.  A wave takes 16 columns
// of one expert that has rows and reads their weights once, 16 x 64 bytes a
// load and eight loads ahead, as one operand of a 16-row instruction whose other
// operand is up to 16 rows of x.  SPLIT: the four waves of a workgroup share 16
// columns and split their contraction, and their sums are joined in LDS in the
// waves' order.
template <ExpertType TY, bool OUT16, bool SPLIT>
__global__ __launch_bounds__(256, 4) void k_expert_few(ExpertArgs a) {
  typedef Mm<TY> M;
  typedef typename M::S S;
  constexpr bool mx = TY == kTypeMx4;
  __shared__ f32x4_t part[SPLIT ? 4 : 1][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, lk = lane >> 4;
  int e = (int)blockIdx.y;
  if (a.offsets) {                                   // the blockIdx.y-th expert with rows
    int left = (int)blockIdx.y, found = -1;
    for (int b = 0; b < a.E && found < 0; b += 64) {
      int64_t s0, cnt = 0;
      if (b + lane < a.E) segment(a, b + lane, s0, cnt);
      uint64_t in = __ballot(cnt > 0);
      const int n = __popcll(in);
      if (left < n) {
        for (; left > 0; --left) in &= in - 1;
        found = b + __ffsll((unsigned long long)in) - 1;
      }
      left -= n;
    }
    if (found < 0) return;
    e = __builtin_amdgcn_readfirstlane(found);
  }
  int64_t s0, cnt;
  segment(a, e, s0, cnt);
  const int n0 = (SPLIT ? (int)blockIdx.x : (int)blockIdx.x * 4 + wave) * 16, n = n0 + l16;
  if (!SPLIT && n0 >= a.N) return;
  const int bytes = mx ? (a.K + 127) / 128 * 64 : a.K * (int)sizeof(S);
  const int nst = (bytes + 63) / 64, per = SPLIT ? (nst + 3) / 4 : nst;
  const int st0 = SPLIT ? wave * per : 0, st1 = min(nst, st0 + per);
  const char* wrow = (const char*)a.w + e * a.w_e + (n < a.N ? n : 0) * a.w_n + 16 * lk;
  const char* wsrow = mx ? (const char*)a.ws + e * a.ws_e + (n < a.N ? n : 0) * a.ws_n : nullptr;
  for (int64_t m0 = 0; m0 < cnt; m0 += 16) {
    const int64_t i = m0 + l16;
    const int64_t r = i < cnt ? source_row(a, s0, i) : -1;
    const int64_t xe = a.offsets ? 0 : (int64_t)e;
    const char* xrow = (const char*)a.x + xe * a.x_e + (r < 0 ? 0 : r) * a.x_stride + 16 * lk;
    const char* xsrow = mx ? (const char*)a.xs + xe * a.xs_e + (r < 0 ? 0 : r) * a.xs_stride : nullptr;
    f32x4_t acc = {0.0f, 0.0f, 0.0f, 0.0f};
    // a chunk of step st; whole: the step lies inside the row
    auto load = [&](const char* p, bool have, int st, const void* safe, bool whole) -> uint4 {
      uint4 u;
      if (whole) {
        __builtin_memcpy(&u, p + st * 64, 16);       // (an absent row's pointer is row 0's)
        return have ? u : make_uint4(0, 0, 0, 0);
      }
      const int left = st < st1 ? bytes - st * 64 - 16 * lk : 0;
      if constexpr (mx) {
        return have && left > 0 ? *reinterpret_cast<const uint4*>(p + st * 64) : make_uint4(0, 0, 0, 0);
      } else {
        return load_chunk<S>(p + st * 64, have ? left / (int)sizeof(S) : 0, true, bytes >= 16, (const char*)safe);
      }
    };
    constexpr int U = 8;
    // the scales of U steps, 4 bytes (one a chunk lane) each, the lane's first
    auto scales = [&](const char* p, bool have, int b, uint32_t (&v)[U]) {
#pragma unroll
      for (int u = 0; u < U; u += 4) {
        uint32_t q[4] = {0, 0, 0, 0};
        if (have && b + u + 4 <= st1) {
          __builtin_memcpy(q, __builtin_assume_aligned(p + (b + u) * 4, 4), 16);
        } else if (have) {
#pragma unroll
          for (int d = 0; d < 4; ++d)
            if (b + u + d < st1) q[d] = *reinterpret_cast<const uint32_t*>(p + (b + u + d) * 4);
        }
#pragma unroll
        for (int d = 0; d < 4; ++d) v[u + d] = q[d] >> (8 * lk);
      }
    };
    auto group = [&](int b, auto whole) {
      uint4 fw[U], fx[U];
      uint32_t sw[U], sx[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        fw[u] = load(wrow, n < a.N, b + u, a.w, decltype(whole)::value);
        fx[u] = load(xrow, r >= 0, b + u, a.x, decltype(whole)::value);
        sw[u] = sx[u] = 0;
      }
      if constexpr (mx) {
        scales(wsrow, n < a.N, b, sw);
        scales(xsrow, r >= 0, b, sx);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) acc = M::mma16(fw[u], fx[u], acc, sw[u], sx[u]);
    };
    int b = st0;
    for (; b + U <= st1 && (b + U) * 64 <= bytes; b += U) group(b, std::true_type{});
    for (; b < st1; b += U) group(b, std::false_type{});
    if constexpr (SPLIT) {
      __syncthreads();                               // the last tile's sums have been read
      part[wave][lane] = acc;
      __syncthreads();
      acc = part[0][lane] + part[1][lane] + part[2][lane] + part[3][lane];
    }
    if ((!SPLIT || wave == 0) && i < cnt) {          // lane: row l16, columns n0 + 4 lk + 0 .. 3
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int c = n0 + 4 * lk + u;
        if (c >= a.N) continue;
        float f = acc[u];
        if (a.bias) f += a.bias[(int64_t)e * a.N + c];
        if (a.relu) f = f < 0.0f ? 0.0f : f;         // (NaN stays)
        const int64_t at = (s0 + i) * a.out_stride + c;
        if constexpr (OUT16) ((uint16_t*)a.out)[at] = f32_to_bf16_bits(f);
        else ((float*)a.out)[at] = f;
      }
    }
  }
}

namespace {

// Division of slots, below 2^31, by k > 1: with 2^s >= k the smallest, m =
// floor(2^(31 + s) / k) + 1 exceeds 2^(31 + s) / k by at most 2^s / 2^(31 + s)
// relative, so slot m / 2^(31 + s) exceeds slot / k by less than 1 / k.
ExpertArgs with_divisor(ExpertArgs a) {
  int s = 1;
  while (((int64_t)1 << s) < a.k) ++s;
  a.k_mul = a.k > 1 ? (uint32_t)((1ull << (31 + s)) / (uint32_t)a.k + 1) : 0;
  a.k_shift = s - 1;
  return a;
}

// whether a launch, which counts its work-items in 32 bits, holds so many tiles
template <typename SH>
bool tiles_fit(int64_t tiles) {
  return (tiles + 7) / 8 * 8 * SH::kThreads <= 0xffffffffll;
}

template <typename SH, ExpertType TY, Pass PASS, Load XL, Load WL, bool OUT16>
hipError_t tile_go(const ExpertArgs& a, int64_t tiles, hipStream_t s) {
  if (!tiles_fit<SH>(tiles)) return hipErrorInvalidValue;
  constexpr size_t lds =
      2 * (size_t)(SH::kXBytes + SH::kWBytes + (TY == kTypeMx4 ? SH::kScaleBytes : 0)) + SH::kWR * 4;
  static_assert(lds * SH::WGS <= 160 * 1024, "workgroups of a CU share its LDS");
  auto* fn = k_expert_tile<SH, TY, PASS, XL, WL, OUT16>;
  if (lds > 64 * 1024) {
    const hipError_t err = hipFuncSetAttribute(reinterpret_cast<const void*>(fn),
                                               hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (err != hipSuccess) return err;
  }
  fn<<<(unsigned)((tiles + 7) / 8 * 8), SH::kThreads, lds, s>>>(a);
  return hipGetLastError();
}

// most tiles that the segments can have: one part tile for each expert with rows
template <typename SH>
int64_t most_tiles(const ExpertArgs& a, Pass pass) {
  const int64_t nt = ((pass == kDw ? a.K : a.N) + SH::kWR - 1) / SH::kWR;
  if (pass == kDw) return (int64_t)a.E * ((a.N + SH::kXR - 1) / SH::kXR) * nt;
  if (!a.offsets) return (a.M + SH::kXR - 1) / SH::kXR * a.E * nt;
  return (a.S / SH::kXR + (a.S < a.E ? a.S : a.E)) * nt;
}

// Time of the tiles on 256 CUs in units of a 64 x 64 tile's share of a busy CU:
// rounds of tiles times what a tile takes, `cost` for each 64 x 64 of it, and
// no less than `least` for a round.  Expected tiles count half a part tile for
// each expert with rows.  More tiles than a launch holds take forever.
//
// Both sides of the lines, us for Wide / Mid / Small, forward unless stated:
//   bf16  1024 x 1024 on 1,024 rows 27 / 16 / 10, 2048 x 1024 on 4,096 31 / 26 /
//         37, 64 of 2048 x 1024 on 32,768 slots 169 / 216 / 309 (dx 179 / 209 /
//         292, where Mid is taken), 32 of 1024 x 1024 on 8,192 dw 44 / 48 / 60
//   4 bit 2048 x 1024 on 4,096 rows 17 / 14 / 21, 64 of 2048 x 1024 on 32,768
//         slots 78 / 82 / 138
//   fp32  2048 x 1024 on 2,048 rows 244 / 81 / 82, 64 of 2048 x 1024 on 16,384
//         slots 737 / 657 / 631, dw 661 / 656 / 798
// It misses by most where Wide's one round is half empty: 4096 x 1024 on 4,096
// rows in bf16 38 / 50 / 63 takes Mid.
template <typename SH>
int64_t tile_time(const ExpertArgs& a, Pass pass, int cost, int least) {
  int64_t n = most_tiles<SH>(a, pass);
  if (!tiles_fit<SH>(n)) return INT64_MAX;
  if (pass != kDw && a.offsets) n -= (a.S < a.E ? a.S : a.E) * ((a.N + SH::kWR - 1) / SH::kWR) / 2;
  const int64_t area = SH::kXR / 64 * (SH::kWR / 64), t = (n + 255) / 256 * area * cost;
  return t > least * area ? t : least * area;
}

template <ExpertType TY, Pass PASS, Load XL, Load WL, bool OUT16>
hipError_t tile_shape(const ExpertArgs& a, hipStream_t s) {
  typedef typename Shapes<TY>::Wide Wide;
  typedef typename Shapes<TY>::Mid Mid;
  typedef typename Shapes<TY>::Small Small;
  constexpr bool f = TY == kTypeF32;
  const int64_t w = tile_time<Wide>(a, PASS, 10, 10), m = tile_time<Mid>(a, PASS, f ? 10 : 12, f ? 10 : 20),
                n = tile_time<Small>(a, PASS, f ? 10 : 16, f ? 10 : 40);
  if (w <= m && w <= n) return tile_go<Wide, TY, PASS, XL, WL, OUT16>(a, most_tiles<Wide>(a, PASS), s);
  if (m <= n) return tile_go<Mid, TY, PASS, XL, WL, OUT16>(a, most_tiles<Mid>(a, PASS), s);
  return tile_go<Small, TY, PASS, XL, WL, OUT16>(a, most_tiles<Small>(a, PASS), s);
}

// Loads straight to LDS ask for addresses on dwords and rows of 16 bytes.
bool on_dwords(int64_t row_bytes, const void* p, int64_t a, int64_t b) {
  return ((uintptr_t)p | (uintptr_t)row_bytes | (uintptr_t)a | (uintptr_t)b) % 4 == 0 && row_bytes >= 16;
}
// The contraction is split where 16 columns a wave would leave the chip less
// than eight waves a CU, if each of its parts is a few loads long.  One row for
// each expert of 1,024 columns in bf16, us split / whole: rows of 8 KB 9 / 21 (one
// expert), 14 / 24 (8), 28 / 39 (24), 29 / 42 (32, taken whole), 111 / 127 (128);
// of 2 KB 10 / 13 (24), 20 / 19 (64); of 1 KB 9 / 9 (16), 12 / 9 (24, taken split),
// 23 / 12 (64); of 512 bytes 9 / 9 (16), 11 / 9 (24).
template <ExpertType TY, bool OUT16>
hipError_t few_go(const ExpertArgs& a, int64_t segs, hipStream_t s) {
  const int64_t bands = (a.N + 15) / 16;
  const int64_t bytes = TY == kTypeMx4 ? (a.K + 127) / 128 * 64 : a.K * (int64_t)sizeof(typename Mm<TY>::S);
  if (bands * segs < 2048 && bytes >= 1024)
    k_expert_few<TY, OUT16, true><<<dim3((unsigned)bands, (unsigned)segs), 256, 0, s>>>(a);
  else
    k_expert_few<TY, OUT16, false><<<dim3((unsigned)((bands + 3) / 4), (unsigned)segs), 256, 0, s>>>(a);
  return hipGetLastError();
}

template <ExpertType TY, bool OUT16>
hipError_t forward_out(const ExpertArgs& a, hipStream_t s) {
  // Up to 16 rows a segment on average the weights' bytes bound the product; up
  // to 64, where tiles would leave CUs idle, reading them again for every 16 rows
  // costs less than long contractions on a few CUs (81 rows over 3 experts of
  // 1062 x 2611 in fp32: 32 us, tiles 70).  Both sides, us for few rows / tiles:
  //   4 experts of 1024 x 2048    bf16 16 rows each 12 / 14, 24 12 / 14, 64 28 / 15;
  //                               fp32 16 21 / 45, 64 50 / 46
  //   64 experts of 2048 x 1024   bf16 4 rows each 46 / 42, 16 96 / 43, 24 128 / 45;
  //                               fp32 4 125 / 137, 16 233 / 142; 4 bit 4 20 / 18
  //   256 experts of 512 x 784    bf16 4 rows each 43 / 41, 16 73 / 42; 4 bit 4 18 /
  //                               23, 16 31 / 24
  // With many experts the line lies too high, and rows that all go to one of many
  // pass its weights once for every 16: 1,024 on one of 64 of 2048 x 2048 in bf16
  // 963 / 22.
  const int64_t segs = a.offsets ? (a.S < a.E ? a.S : a.E) : a.E;
  if (segs <= 65535 && (a.S <= segs * 16 || (a.S <= segs * 64 && most_tiles<typename Shapes<TY>::Small>(a, kForward) < 256))) {
    return few_go<TY, OUT16>(a, segs, s);
  }
  if constexpr (TY == kTypeMx4) return tile_shape<TY, kForward, kDma, kDma, OUT16>(a, s);
  const int64_t row = a.K * (int64_t)sizeof(typename Mm<TY>::S);
  if constexpr (TY != kTypeMx4) {
    if (on_dwords(row, a.x, a.x_stride, a.x_e) && on_dwords(row, a.w, a.w_e, a.w_n))
      return tile_shape<TY, kForward, kDma, kDma, OUT16>(a, s);
    return tile_shape<TY, kForward, kGuarded, kGuarded, OUT16>(a, s);
  }
}

template <ExpertType TY>
hipError_t dx_go(const ExpertArgs& a, hipStream_t s) {
  constexpr bool o16 = TY == kTypeBf16;
  const int64_t e = sizeof(typename Mm<TY>::S);
  const bool rows = on_dwords(a.K * e, a.x, a.x_stride, 0);
  if (rows && on_dwords(a.N * e, a.w, a.w_e, a.w_n)) return tile_shape<TY, kDx, kDma, kNatural, o16>(a, s);
  return tile_shape<TY, kDx, kGuarded, kNaturalGuarded, o16>(a, s);
}

}  // namespace

hipError_t launch_expert_forward(const ExpertArgs& args, ExpertType type, bool out_bf16, hipStream_t s) {
  const ExpertArgs a = with_divisor(args);
  switch (type) {
    case kTypeF32: return out_bf16 ? forward_out<kTypeF32, true>(a, s) : forward_out<kTypeF32, false>(a, s);
    case kTypeBf16: return out_bf16 ? forward_out<kTypeBf16, true>(a, s) : forward_out<kTypeBf16, false>(a, s);
    default: return out_bf16 ? forward_out<kTypeMx4, true>(a, s) : forward_out<kTypeMx4, false>(a, s);
  }
}

hipError_t launch_expert_dx(const ExpertArgs& args, ExpertType type, hipStream_t s) {
  const ExpertArgs a = with_divisor(args);
  return type == kTypeF32 ? dx_go<kTypeF32>(a, s) : dx_go<kTypeBf16>(a, s);
}

hipError_t launch_expert_dw(const ExpertArgs& args, ExpertType type, hipStream_t s) {
  const ExpertArgs a = with_divisor(args);
  const int64_t e = type == kTypeF32 ? 4 : 2;
  const bool aligned = on_dwords(a.K * e, a.x, a.x_stride, 0) && on_dwords(a.N * e, a.w, a.w_n, 0);
  if (type == kTypeF32)
    return aligned ? tile_shape<kTypeF32, kDw, kNatural, kNatural, false>(a, s)
                   : tile_shape<kTypeF32, kDw, kNaturalGuarded, kNaturalGuarded, false>(a, s);
  return aligned ? tile_shape<kTypeBf16, kDw, kNatural, kNatural, false>(a, s)
                 : tile_shape<kTypeBf16, kDw, kNaturalGuarded, kNaturalGuarded, false>(a, s);
}

}  // namespace gevo
