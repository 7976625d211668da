// Products of rows with one weight matrix per expert: segment e of the rows
// (sorted by expert, gathered from x; or every row for every expert) times
// W_e^T, with W_e [N][K], and the two products of its gradient.
//
// k_expert_tile computes a 128 x 256 tile of the output.  Operands of every
// type pass through LDS alike, as rows of 64 bytes of contraction a step (16
// fp32, 32 bf16, 128 4-bit values): 16-byte chunks, one a lane and matrix
// instruction.  The order of the contraction inside a chunk is free as long as
// both operands share it, so
//   bf16   a chunk is one operand of a 32x32x16 instruction,
//   fp32   its four values feed four 32x32x2 instructions,
//   4 bit  it is one block of 32 values, whose scale is one byte of the lane's
//          scale operand in a 32x32x64 instruction.
// Four waves of 64 x 128 read 24 KB of operands from LDS for 1,024 matrix
// clocks of a step (96 of the 128 bytes a clock LDS gives; 64 x 64 a wave would
// ask for all of them).  Three buffers of 24 KB hold a step in use and two
// under way, and leave room for two workgroups on a CU.
#include "gevo_internal.h"
#include "gevo_device.h"
#include "gevo_ops.h"

#include <type_traits>

namespace gevo {

namespace {

typedef int i32x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

constexpr int kXR = 128, kWR = 256;              // rows of the two operand tiles
constexpr int kStep = 64;                        // bytes of contraction a step
constexpr int kBufs = 3;
constexpr int kXBytes = kXR * kStep, kWBytes = kWR * kStep;
constexpr int kScaleBytes = (kXR + kWR) * 4;

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

// Chunk c of row r of an operand tile lies at chunk c ^ turn(r) of the row: any
// 8 or 16 consecutive rows then cover the banks once.
__device__ __forceinline__ int turn(int r) { return (r & 4) >> 1 | (((r >> 1) ^ (r >> 3)) & 1); }

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
__device__ __forceinline__ int64_t placed_row(const int32_t* order, int k, int64_t rows, int64_t r) {
  if (order) r = (uint32_t)order[r] / (uint32_t)k;
  return r < rows ? r : -1;
}
__device__ __forceinline__ int64_t source_row(const ExpertArgs& a, int64_t s0, int64_t i) {
  return a.offsets ? placed_row(a.order, a.k, a.xrows, s0 + i) : i;
}

// Workgroup -> tile of a list that runs expert by expert, each expert's tiles
// column tile by column tile with the row tiles fastest.  XCD j (workgroups
// with index j mod 8) gets the j-th eighth of the list, so the tiles that read
// one weight tile run near each other under one L2.  Every wave sums the
// experts' tile counts, 64 at a time.
struct Tile {
  int e, nt;
  int64_t s0, cnt, m0;
};
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
    return (uint32_t)__shfl((int)inc, 63, 64);
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
    const uint32_t per = total / (uint32_t)a.E;
    o.e = (int)(idx / per);
    idx -= (uint32_t)o.e * per;
  } else {
    for (int b = 0;; b += 64) {
      if (b >= a.E) return false;
      uint32_t sum;
      if (a.E > 64 || b > 0) sum = look(b);
      else sum = total;                              // still in the lanes
      if (idx < sum) {
        const uint64_t in = __ballot(idx >= before && idx < before + mine);
        const int l = __ffsll((unsigned long long)in) - 1;
        o.e = b + l;
        idx -= (uint32_t)__shfl((int)before, l, 64);
        break;
      }
      idx -= sum;
    }
  }
  o.e = __builtin_amdgcn_readfirstlane(o.e);
  idx = (uint32_t)__builtin_amdgcn_readfirstlane((int)idx);
  segment(a, o.e, o.s0, o.cnt);
  const uint32_t rt = (uint32_t)((o.cnt + kXR - 1) / kXR);
  o.nt = (int)(idx / rt);
  o.m0 = (int64_t)(idx % rt) * kXR;
  return true;
}

// 16 bytes at p of which the first `valid` elements exist; whole: one load
template <typename S>
__device__ __forceinline__ uint4 load_chunk(const char* p, int valid, bool whole) {
  constexpr int V = 16 / sizeof(S);
  if (valid <= 0) return make_uint4(0, 0, 0, 0);
  if (whole && valid >= V) return *reinterpret_cast<const uint4*>(p);
  S e[V];
#pragma unroll
  for (int i = 0; i < V; ++i) e[i] = i < valid ? reinterpret_cast<const S*>(p)[i] : (S)0;
  uint4 u;
  __builtin_memcpy(&u, e, 16);
  return u;
}

enum Load { kDma, kGuarded, kTransposed };
enum Pass { kForward, kDx, kDw };

}  // namespace

// A tile of a product.  XL, WL: how the operand tiles reach LDS.
//   kDma         16-byte chunks straight to LDS, two steps ahead
//   kGuarded     through registers, element by element where rows are not
//                aligned or the contraction ends inside a chunk
//   kTransposed  the contraction is the operand's outer index: a lane loads a
//                square of 8 x 8 (fp32: 4 x 4) values and turns it in registers
template <ExpertType TY, Pass PASS, Load XL, Load WL, bool OUT16>
__global__ __launch_bounds__(256, 2) void k_expert_tile(ExpertArgs a) {
  typedef Mm<TY> M;
  typedef typename M::S S;
  constexpr int V = 16 / sizeof(S);                  // elements a chunk (not of 4-bit operands)
  constexpr bool mx = TY == kTypeMx4;
  constexpr int kBuf = kXBytes + kWBytes + (mx ? kScaleBytes : 0);
  constexpr bool kAllDma = XL == kDma && WL == kDma;
  constexpr int kIssued = (XL == kDma ? 2 : 0) + (WL == kDma ? 4 : 0) + (mx ? 2 : 0);   // loads to LDS a step and wave
  extern __shared__ __align__(16) char smem[];

  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l32 = lane & 31, lh = lane >> 5;
  const int wu = __builtin_amdgcn_readfirstlane(wave);
  const int wm = wave & 1, wn = wave >> 1;           // 64-row, 128-column band of the wave
  const uint32_t lds0 = lds_addr(smem);

  Tile tl;
  if constexpr (PASS == kDw) {
    // tiles of every expert's [N][K] gradient; x operand: columns of dy, w operand: columns of x
    const int nr = (a.N + kXR - 1) / kXR, nc = (a.K + kWR - 1) / kWR;
    const uint32_t total = (uint32_t)a.E * (uint32_t)(nr * nc), each = (total + 7) / 8, at = blockIdx.x >> 3;
    const uint32_t idx = (blockIdx.x & 7) * each + at;
    if (at >= each || idx >= total) return;
    tl.e = (int)(idx / (uint32_t)(nr * nc));
    const int in = (int)(idx % (uint32_t)(nr * nc));
    tl.nt = in / nr;
    tl.m0 = (int64_t)(in % nr) * kXR;
    segment(a, tl.e, tl.s0, tl.cnt);
  } else {
    if (!find_tile(a, (a.N + kWR - 1) / kWR, tl)) return;
  }
  const int n0 = tl.nt * kWR;
  const int cols = PASS == kDw ? a.K : a.N;          // of the output

  // contraction: elements (steps of kStep bytes), chunks past `bytes` read zeros
  const int64_t clen = PASS == kDw ? tl.cnt : a.K;
  constexpr int kPer = mx ? 2 * kStep : kStep / (int)sizeof(S);   // elements a step
  const int nst = (int)((clen + kPer - 1) / kPer);
  const int bytes = mx ? (int)((a.K + 127) / 128 * 64) : (int)(a.K * (int64_t)sizeof(S));   // (not kDw)

  // ---- chunks in row order: rows 16 j + lane / 4, chunk lane % 4 of LDS
  const int crow16 = lane >> 2, cbyte = 16 * ((lane & 3) ^ turn(crow16));
  const char* xp[2];
  int xlim[2];
  const char* wp[4];
  int wlim[4];
  if constexpr (XL != kTransposed) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int64_t i = tl.m0 + 16 * (2 * wave + j) + crow16;
      int64_t r = i < tl.cnt ? source_row(a, tl.s0, i) : -1;
      xlim[j] = r >= 0 ? bytes : 0;
      if (r < 0) r = 0;
      xp[j] = (const char*)a.x + (a.offsets ? 0 : tl.e * a.x_e) + r * a.x_stride + cbyte;
    }
  }
  if constexpr (WL != kTransposed) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int n = n0 + 16 * (4 * wave + j) + crow16;
      wlim[j] = n < a.N ? bytes : 0;
      wp[j] = (const char*)a.w + tl.e * a.w_e + (n < a.N ? n : 0) * a.w_n + cbyte;
    }
  }
  const char* xsp = nullptr;
  const char* wsp = nullptr;
  if constexpr (mx) {                                // a wave loads 64 rows' scales of each operand, 4 bytes a step
    const int64_t i = tl.m0 + 64 * (wave & 1) + lane;
    const int64_t r = i < tl.cnt ? source_row(a, tl.s0, i) : -1;
    if (r >= 0) xsp = (const char*)a.xs + (a.offsets ? 0 : tl.e * a.xs_e) + r * a.xs_stride;
    const int n = n0 + 64 * wave + lane;
    if (n < a.N) wsp = (const char*)a.ws + tl.e * a.ws_e + n * a.ws_n;
  }
  const char* zero = (const char*)&g_zero_chunk;
  auto issue = [&](int st) {
    const uint32_t buf = lds0 + (uint32_t)(st % kBufs) * kBuf;
    const int at = st * kStep;
    if constexpr (XL == kDma) {
#pragma unroll
      for (int j = 0; j < 2; ++j)
        dma16_at(at + cbyte < xlim[j] ? xp[j] + at : zero, buf + (uint32_t)(2 * wu + j) * 1024u);
    }
    if constexpr (WL == kDma) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        dma16_at(at + cbyte < wlim[j] ? wp[j] + at : zero, buf + kXBytes + (uint32_t)(4 * wu + j) * 1024u);
    }
    if constexpr (mx) {
      dma4_at(xsp ? xsp + st * 4 : zero, buf + kXBytes + kWBytes + (uint32_t)(wu & 1) * 256u);
      dma4_at(wsp ? wsp + st * 4 : zero, buf + kXBytes + kWBytes + kXR * 4 + (uint32_t)wu * 256u);
    }
  };

  // ---- chunks through registers
  uint4 xg[XL == kGuarded ? 2 : 1], wg[WL == kGuarded ? 4 : 1];
  const bool xwhole = ((uintptr_t)a.x | (uintptr_t)a.x_stride) % 16 == 0;
  const bool wwhole = ((uintptr_t)a.w | (uintptr_t)a.w_e | (uintptr_t)a.w_n) % 16 == 0;
  auto fetch = [&](int st) {
    const int at = st * kStep;
    if constexpr (XL == kGuarded) {
#pragma unroll
      for (int j = 0; j < 2; ++j)
        xg[j] = load_chunk<S>(xp[j] + at, (xlim[j] - at - cbyte) / (int)sizeof(S), xwhole);
    }
    if constexpr (WL == kGuarded) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        wg[j] = load_chunk<S>(wp[j] + at, (wlim[j] - at - cbyte) / (int)sizeof(S), wwhole);
    }
  };
  auto put = [&](int st) {
    char* buf = smem + (size_t)(st % kBufs) * kBuf;
    if constexpr (XL == kGuarded) {
#pragma unroll
      for (int j = 0; j < 2; ++j) *reinterpret_cast<uint4*>(buf + (2 * wave + j) * 1024 + lane * 16) = xg[j];
    }
    if constexpr (WL == kGuarded) {
#pragma unroll
      for (int j = 0; j < 4; ++j) *reinterpret_cast<uint4*>(buf + kXBytes + (4 * wave + j) * 1024 + lane * 16) = wg[j];
    }
  };

  // ---- transposed: squares of V contraction rows x V columns.  A square's V
  // chunks are one chunk column of V rows of the tile.  bf16: the w tile's 128
  // squares go to threads 0-127, the x tile's 64 to 128-191; fp32: 256 and 128,
  // two to a thread.
  constexpr bool kTr = XL == kTransposed || WL == kTransposed;
  constexpr int kSq = !kTr ? 0 : (V == 8 ? 1 : (XL == kTransposed ? 2 : 1));
  uint4 sq[kSq ? kSq : 1][V];
  struct Square {
    const char* p;           // contraction row 0, first column
    int64_t stride;          // bytes between contraction rows
    int valid, row, lds;     // columns that exist; first contraction row in a step; place in the buffer
    bool whole, gather, isx;
  } sd[kSq ? kSq : 1];
  float dbs[V];
#pragma unroll
  for (int v = 0; v < V; ++v) dbs[v] = 0.0f;
  if constexpr (kTr) {
#pragma unroll
    for (int q = 0; q < kSq; ++q) {
      Square& d = sd[q];
      constexpr int wsq = kWR / V * 4, xsq = kXR / V * 4;
      const int b = V == 8 ? tid : tid;
      bool isx = V == 8 ? (XL == kTransposed && b >= wsq) : q == 1;
      const int id = V == 8 && isx ? b - wsq : b;
      const bool live = id < (isx ? xsq : wsq) && (isx ? XL == kTransposed : WL == kTransposed);
      const int kc = id & 3, r0 = (id >> 2) * V;     // chunk, first tile row
      d.isx = isx;
      d.row = kc * V;
      d.lds = (isx ? 0 : kXBytes) + r0 * kStep;
      d.gather = false;
      if (PASS == kDx) {                             // w tile: columns n0 + r0 of W_e, contraction over its rows
        const int c = n0 + r0;
        d.valid = a.N - c;
        d.p = (const char*)a.w + tl.e * a.w_e + (size_t)c * sizeof(S);
        d.stride = a.w_n;
        d.whole = wwhole;
      } else if (isx) {                              // dw: columns of dy
        const int c = (int)tl.m0 + r0;
        d.valid = a.N - c;
        d.p = (const char*)a.w + tl.s0 * a.w_n + (size_t)c * sizeof(S);
        d.stride = a.w_n;
        d.whole = ((uintptr_t)a.w | (uintptr_t)a.w_n) % 16 == 0;
      } else {                                       // dw: columns of x, gathered rows
        const int c = n0 + r0;
        d.valid = a.K - c;
        d.p = (const char*)a.x + (size_t)c * sizeof(S);
        d.stride = a.x_stride;
        d.whole = xwhole;
        d.gather = true;
      }
      if (!live) d.valid = 0;
    }
  }
  auto fetch_t = [&](int st) {
    if constexpr (kTr) {
#pragma unroll
      for (int q = 0; q < kSq; ++q) {
        const Square& d = sd[q];
        int64_t row[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const int64_t k = (int64_t)st * kPer + d.row + i;
          row[i] = k < clen && d.valid > 0 ? k : -1;
          if (PASS == kDw && d.gather && row[i] >= 0) row[i] = source_row(a, tl.s0, row[i]);
        }
#pragma unroll
        for (int i = 0; i < V; ++i)
          sq[q][i] = load_chunk<S>(d.p + (row[i] < 0 ? 0 : row[i]) * d.stride, row[i] < 0 ? 0 : d.valid, d.whole);
      }
    }
  };
  auto put_t = [&](int st) {
    if constexpr (kTr) {
      char* buf = smem + (size_t)(st % kBufs) * kBuf;
#pragma unroll
      for (int q = 0; q < kSq; ++q) {
        const Square& d = sd[q];
        const bool live = V == 8 ? tid < (XL == kTransposed ? 192 : 128) : (!d.isx || tid < 128);
        if (!live) continue;
        const int kc = d.row / V, r0 = (d.lds - (d.isx ? 0 : kXBytes)) / kStep;
#pragma unroll
        for (int c = 0; c < V; ++c) {
          uint4 o;
          if constexpr (V == 8) {
            uint32_t w[4];
#pragma unroll
            for (int p = 0; p < 4; ++p) {            // values c of contraction rows 2p, 2p + 1
              const uint32_t lo = (&sq[q][2 * p].x)[c >> 1], hi = (&sq[q][2 * p + 1].x)[c >> 1];
              w[p] = __builtin_amdgcn_perm(hi, lo, c & 1 ? 0x07060302u : 0x05040100u);
            }
            o = make_uint4(w[0], w[1], w[2], w[3]);
          } else {
            o = make_uint4((&sq[q][0].x)[c], (&sq[q][1].x)[c], (&sq[q][2].x)[c], (&sq[q][3].x)[c]);
          }
          *reinterpret_cast<uint4*>(buf + d.lds + c * kStep + 16 * (kc ^ turn(r0 + c))) = o;
          if (PASS == kDw && d.isx && a.db && tl.nt == 0) {
            S e[V];
            __builtin_memcpy(e, &o, 16);
#pragma unroll
            for (int i = 0; i < V; ++i) dbs[c] += Op<S>::to_f32(e[i]);
          }
        }
      }
    }
  };

  f32x16_t acc[2][4];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int t = 0; t < 4; ++t) acc[i][t] = zero16();

  // The tile is accumulated transposed (w operand's rows down): lane l holds
  // row 32 i + l % 32 of the wave's band and, in registers 4 q + r, columns
  // 32 t + 8 q + 4 (l / 32) + r.
  auto compute = [&](int st) {
    const char* buf = smem + (size_t)(st % kBufs) * kBuf;
    const char* xb = buf + (wm * 64 + l32) * kStep;
    const char* wb = buf + kXBytes + (wn * 128 + l32) * kStep;
    const int tr = turn(l32);
    uint32_t sx[2] = {0, 0}, sw[4] = {0, 0, 0, 0};
    if constexpr (mx) {
      const uint32_t* sp = reinterpret_cast<const uint32_t*>(buf + kXBytes + kWBytes);
#pragma unroll
      for (int i = 0; i < 2; ++i) sx[i] = sp[wm * 64 + 32 * i + l32] >> (8 * lh);
#pragma unroll
      for (int t = 0; t < 4; ++t) sw[t] = sp[kXR + wn * 128 + 32 * t + l32] >> (8 * lh);
    }
    auto step = [&](auto sc) {
      constexpr int s = decltype(sc)::value;
      const int co = 16 * ((2 * s + lh) ^ tr);
      uint4 fx[2], fw[4];
#pragma unroll
      for (int i = 0; i < 2; ++i) fx[i] = *reinterpret_cast<const uint4*>(xb + 32 * i * kStep + co);
#pragma unroll
      for (int t = 0; t < 4; ++t) fw[t] = *reinterpret_cast<const uint4*>(wb + 32 * t * kStep + co);
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 2; ++i) acc[i][t] = M::template mma<2 * s>(fw[t], fx[i], acc[i][t], sw[t], sx[i]);
    };
    step(std::integral_constant<int, 0>{});
    step(std::integral_constant<int, 1>{});
  };

  if (nst > 0) {
    issue(0);
    if (nst > 1) issue(1);
    if constexpr (!kAllDma) {
      fetch(0);
      fetch_t(0);
      put(0);
      put_t(0);
    }
    for (int st = 0; st < nst; ++st) {
      if (st + 1 < nst) wait_vm<kIssued>();
      else wait_vm<0>();
      __syncthreads();                               // step st is in LDS; step st - 1's buffer is free
      if (st + 2 < nst) issue(st + 2);
      if constexpr (!kAllDma) {
        if (st + 1 < nst) {
          fetch(st + 1);
          fetch_t(st + 1);
        }
      }
      compute(st);
      if constexpr (!kAllDma) {
        if (st + 1 < nst) {
          put(st + 1);
          put_t(st + 1);
        }
      }
    }
  }

  if constexpr (PASS == kDw) {
    if (a.db && tl.nt == 0) {                        // column sums of dy: the four chunk lanes of a square's rows
#pragma unroll
      for (int v = 0; v < V; ++v) {
        dbs[v] += __shfl_xor(dbs[v], 1, 64);
        dbs[v] += __shfl_xor(dbs[v], 2, 64);
      }
      const int b = V == 8 ? tid - 128 : tid;
      if (b >= 0 && b < kXR / V * 4 && (b & 3) == 0) {
        const int c = (int)tl.m0 + (b >> 2) * V;
#pragma unroll
        for (int v = 0; v < V; ++v)
          if (c + v < a.N) a.db[(int64_t)tl.e * a.N + c + v] = dbs[v];
      }
    }
  }

  // ---- output
  const bool v4 = ((cols | (int)a.out_stride) & 3) == 0 && (uintptr_t)a.out % (OUT16 ? 8 : 16) == 0;
  const int64_t rows = PASS == kDw ? a.N : tl.cnt;
  const float* bias = PASS == kForward && a.bias ? a.bias + (int64_t)tl.e * a.N : nullptr;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int64_t r = tl.m0 + wm * 64 + 32 * i + l32;
    if (r >= rows) continue;
    const int64_t orow = PASS == kDw ? (int64_t)tl.e * a.N + r : tl.s0 + r;
    const S* mrow = nullptr;
    if constexpr (PASS == kDx) {
      if (a.mask) {
        const int64_t mr = placed_row(a.mask_order, a.k, a.mask_rows, tl.s0 + r);
        mrow = (const S*)((const char*)a.mask + (mr < 0 ? 0 : mr) * a.mask_stride);
      }
    }
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int c = n0 + wn * 128 + 32 * t + 8 * q + 4 * lh;
        if (c >= cols) continue;
        float f[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          f[u] = acc[i][t][4 * q + u];
          if (c + u < cols) {
            if (bias) f[u] += bias[c + u];
            if (PASS == kForward && a.relu) f[u] = f[u] > 0.0f || f[u] != f[u] ? f[u] : 0.0f;
            if constexpr (PASS == kDx && !mx) {
              if (mrow && !(Op<S>::to_f32(mrow[c + u]) > 0.0f)) f[u] = 0.0f;
            }
          }
        }
        if constexpr (OUT16) {
          uint16_t* o = (uint16_t*)a.out + orow * a.out_stride + c;
          const uint2 p = make_uint2(bf16x2(f[0], f[1]), bf16x2(f[2], f[3]));
          if (v4) {
            *reinterpret_cast<uint2*>(o) = p;
          } else {
            o[0] = (uint16_t)p.x;
            if (c + 1 < cols) o[1] = (uint16_t)(p.x >> 16);
            if (c + 2 < cols) o[2] = (uint16_t)p.y;
            if (c + 3 < cols) o[3] = (uint16_t)(p.y >> 16);
          }
        } else {
          float* o = (float*)a.out + orow * a.out_stride + c;
          if (v4) {
            *reinterpret_cast<float4*>(o) = make_float4(f[0], f[1], f[2], f[3]);
          } else {
#pragma unroll
            for (int u = 0; u < 4; ++u)
              if (c + u < cols) o[u] = f[u];
          }
        }
      }
  }
}

// Few rows a segment: the weights' bytes are the time.  A workgroup takes 16
// columns of one expert that has rows; its four waves split the contraction,
// each reading its weights once, 16 x 64 bytes a load and eight loads ahead,
// as one operand of a 16-row instruction whose other operand is up to 16 rows
// of x.  The waves' sums are joined in LDS in the waves' order.
template <ExpertType TY, bool VEC, bool OUT16>
__global__ __launch_bounds__(256) void k_expert_few(ExpertArgs a) {
  typedef Mm<TY> M;
  typedef typename M::S S;
  constexpr bool mx = TY == kTypeMx4;
  __shared__ f32x4_t part[4][64];
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
  const int n0 = blockIdx.x * 16, n = n0 + l16;
  const int bytes = mx ? (a.K + 127) / 128 * 64 : a.K * (int)sizeof(S);
  const int nst = (bytes + 63) / 64, per = (nst + 3) / 4, st0 = wave * per, st1 = min(nst, st0 + per);
  const char* wrow = (const char*)a.w + e * a.w_e + (n < a.N ? n : 0) * a.w_n + 16 * lk;
  const char* wsrow = mx ? (const char*)a.ws + e * a.ws_e + (n < a.N ? n : 0) * a.ws_n + lk : nullptr;
  for (int64_t m0 = 0; m0 < cnt; m0 += 16) {
    const int64_t i = m0 + l16;
    const int64_t r = i < cnt ? source_row(a, s0, i) : -1;
    const int64_t xe = a.offsets ? 0 : (int64_t)e;
    const char* xrow = (const char*)a.x + xe * a.x_e + (r < 0 ? 0 : r) * a.x_stride + 16 * lk;
    const char* xsrow = mx ? (const char*)a.xs + xe * a.xs_e + (r < 0 ? 0 : r) * a.xs_stride + lk : nullptr;
    f32x4_t acc = {0.0f, 0.0f, 0.0f, 0.0f};
    auto load = [&](const char* p, bool have, int st) -> uint4 {
      const int left = bytes - st * 64 - 16 * lk;
      if constexpr (VEC || mx) {
        return have && left > 0 ? *reinterpret_cast<const uint4*>(p + st * 64) : make_uint4(0, 0, 0, 0);
      } else {
        return load_chunk<S>(p + st * 64, have ? left / (int)sizeof(S) : 0, false);
      }
    };
    constexpr int U = 8;
    for (int b = st0; b < st1; b += U) {
      uint4 fw[U], fx[U];
      uint32_t sw[U], sx[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const bool in = b + u < st1;
        fw[u] = load(wrow, in && n < a.N, b + u);
        fx[u] = load(xrow, in && r >= 0, b + u);
        sw[u] = sx[u] = 0;
        if constexpr (mx) {
          if (in && n < a.N) sw[u] = (uint8_t)wsrow[(b + u) * 4];
          if (in && r >= 0) sx[u] = (uint8_t)xsrow[(b + u) * 4];
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) acc = M::mma16(fw[u], fx[u], acc, sw[u], sx[u]);
    }
    __syncthreads();                                 // the last tile's sums have been read
    part[wave][lane] = acc;
    __syncthreads();
    if (wave == 0 && r >= 0) {                       // lane: row l16, columns n0 + 4 lk + 0 .. 3
      const f32x4_t sum = part[0][lane] + part[1][lane] + part[2][lane] + part[3][lane];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int c = n0 + 4 * lk + u;
        if (c >= a.N) continue;
        float f = sum[u];
        if (a.bias) f += a.bias[(int64_t)e * a.N + c];
        if (a.relu) f = f > 0.0f || f != f ? f : 0.0f;
        const int64_t at = (s0 + i) * a.out_stride + c;
        if constexpr (OUT16) ((uint16_t*)a.out)[at] = f32_to_bf16_bits(f);
        else ((float*)a.out)[at] = f;
      }
    }
  }
}

namespace {

template <ExpertType TY, Pass PASS, Load XL, Load WL, bool OUT16>
hipError_t tile_go(const ExpertArgs& a, int64_t tiles, hipStream_t s) {
  constexpr size_t lds = kBufs * (size_t)(kXBytes + kWBytes + (TY == kTypeMx4 ? kScaleBytes : 0));
  auto* fn = k_expert_tile<TY, PASS, XL, WL, OUT16>;
  hipError_t err = hipFuncSetAttribute(reinterpret_cast<const void*>(fn), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  if (err != hipSuccess) return err;
  tiles = (tiles + 7) / 8 * 8;
  if (tiles > 0x7ffffff8) return hipErrorInvalidValue;
  fn<<<(unsigned)tiles, 256, lds, s>>>(a);
  return hipGetLastError();
}

// most tiles that the segments can have: one part tile for each expert with rows
int64_t forward_tiles(const ExpertArgs& a) {
  const int64_t nt = (a.N + kWR - 1) / kWR;
  if (!a.offsets) return (a.M + kXR - 1) / kXR * a.E * nt;
  return (a.S / kXR + (a.S < a.E ? a.S : a.E)) * nt;
}

bool aligned16(const void* p, int64_t a, int64_t b, int64_t c) {
  return ((uintptr_t)p | (uintptr_t)a | (uintptr_t)b | (uintptr_t)c) % 16 == 0;
}

template <ExpertType TY, bool OUT16>
hipError_t forward_out(const ExpertArgs& a, hipStream_t s) {
  const bool vec = TY == kTypeMx4 || (aligned16(a.x, a.x_stride, a.x_e, a.K * (int64_t)sizeof(typename Mm<TY>::S)) &&
                                      aligned16(a.w, a.w_e, a.w_n, 0));
  // Up to 16 rows a segment on average the weights' bytes bound the product
  const int64_t segs = a.offsets ? (a.S < a.E ? a.S : a.E) : a.E;
  if (a.S <= segs * 16 && segs <= 65535) {
    const dim3 grid((unsigned)((a.N + 15) / 16), (unsigned)segs);
    if (vec) k_expert_few<TY, true, OUT16><<<grid, 256, 0, s>>>(a);
    else k_expert_few<TY, false, OUT16><<<grid, 256, 0, s>>>(a);
    return hipGetLastError();
  }
  const int64_t tiles = forward_tiles(a);
  if constexpr (TY == kTypeMx4) return tile_go<TY, kForward, kDma, kDma, OUT16>(a, tiles, s);
  else if (vec) return tile_go<TY, kForward, kDma, kDma, OUT16>(a, tiles, s);
  else return tile_go<TY, kForward, kGuarded, kGuarded, OUT16>(a, tiles, s);
}

template <ExpertType TY>
hipError_t dx_go(const ExpertArgs& a, hipStream_t s) {
  constexpr bool o16 = TY == kTypeBf16;
  const int64_t tiles = forward_tiles(a);
  if (aligned16(a.x, a.x_stride, 0, a.K * (int64_t)sizeof(typename Mm<TY>::S)))
    return tile_go<TY, kDx, kDma, kTransposed, o16>(a, tiles, s);
  return tile_go<TY, kDx, kGuarded, kTransposed, o16>(a, tiles, s);
}

}  // namespace

hipError_t launch_expert_forward(const ExpertArgs& a, ExpertType type, bool out_bf16, hipStream_t s) {
  switch (type) {
    case kTypeF32: return out_bf16 ? forward_out<kTypeF32, true>(a, s) : forward_out<kTypeF32, false>(a, s);
    case kTypeBf16: return out_bf16 ? forward_out<kTypeBf16, true>(a, s) : forward_out<kTypeBf16, false>(a, s);
    default: return out_bf16 ? forward_out<kTypeMx4, true>(a, s) : forward_out<kTypeMx4, false>(a, s);
  }
}

hipError_t launch_expert_dx(const ExpertArgs& a, ExpertType type, hipStream_t s) {
  return type == kTypeF32 ? dx_go<kTypeF32>(a, s) : dx_go<kTypeBf16>(a, s);
}

hipError_t launch_expert_dw(const ExpertArgs& a, ExpertType type, hipStream_t s) {
  const int64_t tiles = (int64_t)a.E * ((a.N + kXR - 1) / kXR) * ((a.K + kWR - 1) / kWR);
  if (type == kTypeF32) return tile_go<kTypeF32, kDw, kTransposed, kTransposed, false>(a, tiles, s);
  return tile_go<kTypeBf16, kDw, kTransposed, kTransposed, false>(a, tiles, s);
}

}  // namespace gevo
