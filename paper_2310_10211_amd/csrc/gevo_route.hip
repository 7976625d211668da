// Routing rows to experts: scores and the choice of k experts (k_route), its
// gradient (k_route_bwd), the stable sort of the rows by expert (k_plan_*) and
// the join of the experts' rows with its gradient (k_combine*).
#include "gevo_internal.h"
#include "gevo_device.h"
#include "gevo_ops.h"

#include <math.h>

namespace gevo {

namespace {

template <typename S> __device__ __forceinline__ float to_f(S v);
template <> __device__ __forceinline__ float to_f<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f<uint16_t>(uint16_t v) { return bf16_bits_to_f32(v); }
template <typename S> __device__ __forceinline__ S from_f(float v);
template <> __device__ __forceinline__ float from_f<float>(float v) { return v; }
template <> __device__ __forceinline__ uint16_t from_f<uint16_t>(float v) { return f32_to_bf16_bits(v); }

// exp(x) to about one unit in the last place from the base-2 instruction: x
// log2 e is split into its rounded product and the remainder, whose
// exponential is 1 + ln 2 remainder.  The instruction gives 0 below 2^-126.
__device__ __forceinline__ float exp_split(float x) {
  x = fmaxf(x, -200.0f);
  const float t = x * 1.44269502f;                  // log2 e = 1.44269502 + 1.9259630e-8
  const float r = fmaf(x, 1.9259630e-8f, fmaf(x, 1.44269502f, -t));
  const float e = __builtin_amdgcn_exp2f(t);
  return fmaf(e, r * 0.693147182f, e);
}

// A value rotated by N lanes within each 16.
template <int N>
__device__ __forceinline__ int rotated(int v) {
  return __builtin_amdgcn_update_dpp(0, v, 0x120 + N, 0xf, 0xf, true);
}

// Reductions over the L lanes (16 or 64, aligned) that share a row; f is
// commutative.  32-bit values: rotations within 16 lanes, which cost an
// instruction each, then the four sixteens' values from scalar registers.
template <int L, typename T, typename F>
__device__ __forceinline__ T row_reduce(T v, F f) {
  if constexpr (sizeof(T) == 4) {
    v = f(v, __builtin_bit_cast(T, rotated<8>(__builtin_bit_cast(int, v))));
    v = f(v, __builtin_bit_cast(T, rotated<4>(__builtin_bit_cast(int, v))));
    v = f(v, __builtin_bit_cast(T, rotated<2>(__builtin_bit_cast(int, v))));
    v = f(v, __builtin_bit_cast(T, rotated<1>(__builtin_bit_cast(int, v))));
    if constexpr (L == 64) {
      T q[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        q[i] = __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 16 * i));
      v = f(f(q[0], q[1]), f(q[2], q[3]));
    }
  } else {
#pragma unroll
    for (int m = L / 2; m >= 1; m >>= 1) v = f(v, __shfl_xor(v, m, L));
  }
  return v;
}
template <int L>
__device__ __forceinline__ uint64_t row_ballot(bool p) {
  const uint64_t b = __ballot(p);
  if (L == 64) return b;
  return (b >> ((threadIdx.x & 63) / L * L)) & ((1ull << (L & 63)) - 1);
}

}  // namespace

// A binary32 as an integer that orders like it (no NaN; -0 below 0), and back;
// binary64 keys stay what they are.
__device__ __forceinline__ int ordered(float f) {
  const int i = __builtin_bit_cast(int, f);
  return i ^ ((i >> 31) & 0x7fffffff);
}
__device__ __forceinline__ double ordered(double f) { return f; }
__device__ __forceinline__ float unordered(int i) { return __builtin_bit_cast(float, i ^ ((i >> 31) & 0x7fffffff)); }
__device__ __forceinline__ double unordered(double f) { return f; }

// Row t: scores s = softmax(l) or sigmoid(l), keys l or s + bias, the best
// groups of keys, then the k largest keys among them (descending, ties to the
// lowest index), weights scale s (renormalised over the choice).
//
// L lanes share a row, each holding NE consecutive logits.  A choice is the
// row's largest local maximum and the lowest index that holds it, taken out by
// the lane that has it.  Keys in 32 bits are compared as integers that order
// like them, whose maximum of three is one instruction, with their place in the
// lane in the low bits, which finds and removes a key in three instructions.
// Bound by instructions and their latency: 65,536 rows of 256, 8 groups, 8
// chosen take 50 us, of which their bytes take 14 (60 with logits and biases
// held in registers through the choice, five waves a SIMD where it is six now;
// finding the k-th key by bisection took as long, a row in a whole wave 135).
//
// Two keys nearer than the rounding of 32-bit scores would be ordered by that
// rounding: a row with such a pair among the keys (or groups) that decide its
// choice is done over with 64-bit keys, which a wave does when one of its rows
// asks for it.  Logits as keys need none of this.
template <typename S, int L, int NE>
__global__ __launch_bounds__(256, NE == 16 ? 6 : 1) void k_route(RouteArgs a) {
  constexpr int kRows = 256 / L;
  extern __shared__ __align__(16) char smem[];
  const int lane = threadIdx.x & (L - 1), rw = threadIdx.x / L;
  const int64_t t = (int64_t)blockIdx.x * kRows + rw;
  const bool live = t < a.T;
  const S* lrow = (const S*)a.logits + (live ? t : 0) * a.stride;
  const int e0 = lane * NE;
  const float ninf = -INFINITY;

  // Logits and biases are read again where the rarer paths want them, rather than
  // held through the choice: 16 of each are a third of its registers.
  float l[NE], b[NE];                                // (biases past the row's end: any of its values)
  auto load_logits = [&]() {
    if (a.vec) {                                     // whole rows of aligned chunks
      constexpr int V = 16 / sizeof(S) < NE ? 16 / sizeof(S) : NE;
#pragma unroll
      for (int j = 0; j < NE; j += V) {
        S e[V];
        __builtin_memcpy(e, __builtin_assume_aligned(lrow + e0 + j, V * sizeof(S)), sizeof(e));
#pragma unroll
        for (int v = 0; v < V; ++v) l[j + v] = live ? to_f<S>(e[v]) : ninf;
      }
    } else {
#pragma unroll
      for (int j = 0; j < NE; ++j) l[j] = live && e0 + j < a.E ? to_f<S>(lrow[e0 + j]) : ninf;
    }
  };
  auto load_biases = [&]() {
#pragma unroll
    for (int j = 0; j < NE; ++j) b[j] = 0.0f;
    if (!a.bias) return;
    if (a.vec) {
      __builtin_memcpy(b, a.bias + e0, sizeof(b));
    } else {
#pragma unroll
      for (int j = 0; j < NE; ++j) b[j] = a.bias[e0 + j < a.E ? e0 + j : 0];
    }
  };
  load_logits();
  load_biases();

  bool bad = false;                                  // NaN, or +inf under softmax: no scores
  float m = ninf;
#pragma unroll
  for (int j = 0; j < NE; j += 2) {
    bad |= __builtin_isunordered(l[j], l[j + 1]);
    m = fmaxf(fmaxf(l[j], l[j + 1]), m);
  }
  float bmax = 0.0f;
  if (a.bias) {
#pragma unroll
    for (int j = 0; j < NE; j += 2) {
      bad |= __builtin_isunordered(b[j], b[j + 1]);
      bmax = fmaxf(fmaxf(fabsf(b[j]), fabsf(b[j + 1])), bmax);
    }
    if (__any(bmax == INFINITY)) {                   // the largest finite one
      bmax = 0.0f;
#pragma unroll
      for (int j = 0; j < NE; ++j) bmax = fmaxf(bmax, fabsf(b[j]) < INFINITY ? fabsf(b[j]) : 0.0f);
    }
  }
  m = row_reduce<L>(m, [](float x, float y) { return fmaxf(x, y); });
  bmax = row_reduce<L>(bmax, [](float x, float y) { return fmaxf(x, y); });
  bad = row_ballot<L>(bad || (!a.sigmoid && m == INFINITY)) != 0;

  // the choice with keys of type F; returns whether its order is beyond doubt
  int chosen = -1;                                   // lane j of the row: the j-th choice
  __shared__ int picked[kRows][L];                   // of a row: its choices
  const int gs = a.E / a.groups;
  auto choose = [&](auto zero) -> bool {
    typedef decltype(zero) F;
    typedef decltype(ordered(zero)) K;
    constexpr bool wide = sizeof(F) == 8;
    const F flowest = (F)ninf;
    const K lowest = ordered(flowest);
    auto more = [](K x, K y) { return x > y ? x : y; };
    auto less = [](K x, K y) { return x < y ? x : y; };
    K key[NE];
    F tol = 0, group_tol = 0;                        // of two keys, of two groups' values
    if constexpr (wide) {
      load_logits();
      load_biases();
    }
    if (a.by_logit) {
#pragma unroll
      for (int j = 0; j < NE; ++j) key[j] = ordered((F)l[j] + (F)0);   // (-0 is 0)
    } else {
      F score[NE], sum = 0, top = 1;
      if (a.sigmoid) {
#pragma unroll
        for (int j = 0; j < NE; ++j) {
          if constexpr (wide) score[j] = 1.0 / (1.0 + exp(-(double)l[j]));
          else score[j] = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(l[j] * -1.44269504f));
        }
      } else {
#pragma unroll
        for (int j = 0; j < NE; ++j) {
          if constexpr (wide) score[j] = l[j] == ninf ? 0.0 : exp((double)l[j] - (double)m);
          else score[j] = l[j] == ninf ? 0.0f : __builtin_amdgcn_exp2f((l[j] - m) * 1.44269504f);
          sum += score[j];
        }
        sum = row_reduce<L>(sum, [](F x, F y) { return x + y; });
        top = (F)1 / sum;                            // the row's largest score
#pragma unroll
        for (int j = 0; j < NE; ++j) score[j] *= top;
      }
      // What two keys in 32 bits can be off by together.  exp2's argument is off by
      // 1.4e-7 of |x| at most (x, its product, log2 e), which x s (1 - s) <= 0.23
      // and x e^-x <= 0.37 keep below 5e-8 of a score; its result, the sum with 1
      // and the reciprocal or the product add a step (1.2e-7) each at most.  A
      // softmax's sum carries its terms' errors, 1.4e-7 times their mean x, below
      // ln 2048, and their step, and NE + 6 half steps of its own, in all below
      // 1.2e-6 + 6e-8 (NE + 6), of both scores alike.  The sum with the bias is off
      // by half a step of itself.  A group adds two keys, to half a step of twice
      // their bound.
      if (!wide) {
        const F half = 6e-8f * (top + (F)bmax);
        tol = 2 * ((a.sigmoid ? 5e-7f : 1e-6f + 3e-8f * (NE + 6)) * top + half);
        group_tol = a.group_top == 2 ? 2 * tol + 4 * half : tol;
      }
#pragma unroll
      for (int j = 0; j < NE; ++j) key[j] = ordered(l[j] == ninf ? flowest : score[j] + (F)b[j]);
    }
    bool sure = true;
    if (a.groups > 1) {
      // a group's value, in every lane that holds part of it: from registers where
      // 1, 2, 4 .. whole lanes hold a group, else through LDS (lane g: group g)
      const int per = gs / NE;                       // lanes of a group
      const bool inreg = gs % NE == 0 && (per & (per - 1)) == 0;
      K v1 = lowest, v2 = lowest;                    // its largest keys
      auto take = [&](K x) {
        v2 = more(v2, less(v1, x));
        v1 = more(v1, x);
      };
      const int shift = inreg ? __ffs(per) - 1 : 0;  // lane >> shift: the group whose value the lane holds
      if (inreg) {
#pragma unroll
        for (int j = 0; j < NE; ++j) take(key[j]);
        for (int d = 1; d < per; d <<= 1) {
          const K o1 = __shfl_xor(v1, d, L), o2 = __shfl_xor(v2, d, L);
          take(o1);
          take(o2);
        }
      } else {
        K* ks = reinterpret_cast<K*>(smem) + (size_t)rw * (L * NE);
#pragma unroll
        for (int j = 0; j < NE; ++j) ks[e0 + j] = key[j];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (lane < a.groups)
          for (int i = 0; i < gs; ++i) take(ks[lane * gs + i]);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      }
      const int mine = lane >> shift;
      F v = a.group_top == 2 && v2 > lowest ? unordered(v1) + unordered(v2) : unordered(v1);
      if (mine >= a.groups) v = flowest;
      uint64_t stay = 0;
      F last = flowest;
      for (int i = 0; i <= a.top_groups && i < a.groups; ++i) {
        const F mx = row_reduce<L>(v, [](F x, F y) { return x > y ? x : y; });
        if (i == a.top_groups) {
          if (!(last - mx > group_tol) && last > flowest) sure = false;
          break;
        }
        // lanes and groups ascend together: the first lane has the lowest group
        const uint64_t hold = row_ballot<L>(v == mx);
        const int g = (__ffsll((unsigned long long)hold) - 1) >> shift;
        if (hold) stay |= 1ull << (g & 63);
        last = mx;
        if (mine == g) v = flowest;
      }
      if (inreg) {
        const bool in = (stay >> (mine & 63)) & 1;
#pragma unroll
        for (int j = 0; j < NE; ++j) key[j] = in ? key[j] : lowest;
      } else {
        int g = e0 / gs, left = (g + 1) * gs - e0;
#pragma unroll
        for (int j = 0; j < NE; ++j) {
          if (!((stay >> (g & 63)) & 1)) key[j] = lowest;
          if (--left == 0) { ++g; left = gs; }
        }
      }
    }
    auto largest = [&]() {
      K v = lowest;
#pragma unroll
      for (int j = 0; j < NE; j += 2) v = more(more(key[j], key[j + 1]), v);
      return v;
    };
    picked[rw][lane] = -1;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    K last = lowest;
    if constexpr (wide) {
      K lm = largest();
      for (int i = 0; i < a.k; ++i) {
        const K mx = row_reduce<L>(lm, more);
        const uint64_t hold = row_ballot<L>(lm == mx && mx > lowest);
        const bool owner = lane == __ffsll((unsigned long long)hold) - 1;
        bool left = owner;                           // the first of its keys that is as large goes
        int at = 0;
#pragma unroll
        for (int j = 0; j < NE; ++j) {
          const bool hit = left && key[j] == mx;
          at = hit ? j : at;
          key[j] = hit ? lowest : key[j];
          left = left && !hit;
        }
        lm = largest();
        if (owner) picked[rw][i] = e0 + at;
      }
    } else {
      // A key's low bits hold its place in the lane, the first the largest, so the
      // lane's largest key is one of its own and says which.  Between lanes the
      // rest of the keys is compared, which orders like the keys where it differs:
      // for logits in bf16 it is all there is; other keys that agree in it are in
      // doubt.  (Keys below `lowest` are -inf's.)
      constexpr K low = NE - 1;
      constexpr bool exact = sizeof(S) == 2;
      const F cut = NE * 2.4e-7f;                    // of a key, what its low bits or its like's come to
#pragma unroll
      for (int j = 0; j < NE; ++j) key[j] = (key[j] & ~low) | (low - j);
      K lm = largest();
      const int tries = a.by_logit && exact ? a.k : a.k + 1;   // the first key left out is looked at, too
      for (int i = 0; i < tries; ++i) {
        const K mx = more(row_reduce<L>(lm & ~low, more), lowest);
        if (last > lowest) {
          if (!a.by_logit) {
            const F x = unordered(last);
            if (!(x - unordered(mx) > tol + cut * fabsf(x))) sure = false;
          } else if (!exact && last == mx) {
            sure = false;
          }
        }
        if (i == a.k) break;
        last = mx;
        const uint64_t hold = row_ballot<L>((lm & ~low) == mx && mx > lowest);
        const bool owner = lane == __ffsll((unsigned long long)hold) - 1;
        if (owner) picked[rw][i] = e0 + (int)(low - (lm & low));
        const K out = owner ? lm : 0x7fffffff;       // (no key)
#pragma unroll
        for (int j = 0; j < NE; ++j) key[j] = key[j] == out ? lowest : key[j];
        lm = largest();
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    chosen = picked[rw][lane];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    return sure;
  };
  const bool none = bad || m == ninf;
  const bool sure = choose(0.0f);
  if (__any(live && !none && !sure)) choose(0.0);
  if (none) chosen = -1;

  // weights of the choice: lane j < k holds choice j.  Renormalised scores are
  // formed relative to the largest chosen logit, so that they hold where the
  // scores themselves would underflow.
  const float lc = chosen >= 0 ? to_f<S>(lrow[chosen]) : ninf;
  float w;
  if (a.renorm) {
    const float mc = row_reduce<L>(lc, [](float x, float y) { return fmaxf(x, y); });
    if (a.sigmoid) {
      const float c = fminf(mc, 0.0f);
      w = mc >= 0.0f ? 1.0f / (1.0f + expf(-lc)) : expf(lc - c) / (1.0f + expf(lc));
    } else {
      w = expf(lc - mc);
    }
    if (chosen < 0) w = 0.0f;
    const float sum = row_reduce<L>(w, [](float x, float y) { return x + y; });
    w = w / sum * a.scale;
  } else if (a.sigmoid) {
    w = 1.0f / (1.0f + expf(-lc)) * a.scale;
  } else {
    float sum = 0.0f;
    load_logits();
#pragma unroll
    for (int j = 0; j < NE; ++j) sum += l[j] == ninf ? 0.0f : exp_split(l[j] - m);
    sum = row_reduce<L>(sum, [](float x, float y) { return x + y; });
    w = expf(lc - m) / sum * a.scale;
  }
  if (chosen < 0) w = bad ? NAN : 0.0f;
  if (live && lane < a.k) {
    a.weights[t * a.k + lane] = w;
    a.ids[t * a.k + lane] = chosen;
  }
}

// Gradient of the weights with respect to the logits.  With g the gradient of
// the chosen weights, s their scores, r = s / sum s:
//   softmax:          dl_e = scale s_e ([e chosen] g_e - sum_C s_j g_j), every e
//   softmax, renorm:  dl_j = scale r_j (g_j - sum_C r_i g_i) on the choice
//   sigmoid:          dl_j = scale s_j (1 - s_j) g_j on the choice
//   sigmoid, renorm:  dl_j = scale r_j (1 - s_j) (g_j - sum_C r_i g_i)
// An expert chosen twice by a row gets both terms.  L lanes share a row; the
// row is put together in LDS and written whole.
template <typename S, int L, int NE>
__global__ __launch_bounds__(256) void k_route_bwd(RouteArgs a) {
  constexpr int kRows = 256 / L;
  extern __shared__ __align__(16) char smem[];
  float* row = reinterpret_cast<float*>(smem) + (size_t)(threadIdx.x / L) * (L * NE);
  const int lane = threadIdx.x & (L - 1);
  const int64_t t = (int64_t)blockIdx.x * kRows + threadIdx.x / L;
  const bool live = t < a.T;
  const S* lrow = (const S*)a.logits + (live ? t : 0) * a.stride;
  const float ninf = -INFINITY;
  auto add = [](float x, float y) { return x + y; };
  auto larger = [](float x, float y) { return fmaxf(x, y); };

  int id = live && lane < a.k ? a.ids[t * a.k + lane] : -1;
  if (id < 0 || id >= a.E) id = -1;
  const float g = id >= 0 ? a.dweights[t * a.k + lane] : 0.0f;
  const float lc = id >= 0 ? to_f<S>(lrow[id]) : ninf;
  const bool any = row_ballot<L>(id >= 0) != 0;

  float base[NE];
#pragma unroll
  for (int j = 0; j < NE; ++j) base[j] = 0.0f;
  float mine;                                        // the chosen element's own term
  if (!a.sigmoid && !a.renorm) {
    float l[NE], m = ninf, sum = 0.0f;
#pragma unroll
    for (int j = 0; j < NE; ++j) {
      l[j] = live && lane * NE + j < a.E ? to_f<S>(lrow[lane * NE + j]) : ninf;
      m = fmaxf(m, l[j]);
    }
    m = row_reduce<L>(m, larger);
#pragma unroll
    for (int j = 0; j < NE; ++j) {
      l[j] = l[j] == ninf ? 0.0f : exp_split(l[j] - m);
      sum += l[j];
    }
    sum = row_reduce<L>(sum, add);
    const float s = id >= 0 ? expf(lc - m) / sum : 0.0f;
    const float dot = row_reduce<L>(s * g, add);
    const float c = -a.scale * dot / sum;
    if (any) {
#pragma unroll
      for (int j = 0; j < NE; ++j) base[j] = l[j] * c;
    }
    mine = a.scale * s * g;
  } else if (a.renorm) {
    const float mc = row_reduce<L>(lc, larger);
    float r = 0.0f, rest = 1.0f;                     // rest: 1 - s of a sigmoid
    if (id >= 0) {
      if (a.sigmoid) {
        r = mc >= 0.0f ? 1.0f / (1.0f + expf(-lc)) : expf(lc - mc) / (1.0f + expf(lc));
        rest = 1.0f / (1.0f + expf(lc));
      } else {
        r = expf(lc - mc);
      }
    }
    const float sum = row_reduce<L>(r, add);
    r = id >= 0 ? r / sum : 0.0f;
    const float dot = row_reduce<L>(r * g, add);
    // g_j - sum r_i g_i = sum_i r_i (g_j - g_i): the plain difference
    mine = a.scale * r * rest * (g - dot);
  } else {
    mine = a.scale * g / (1.0f + expf(-lc)) / (1.0f + expf(lc));
  }
  if (id < 0) mine = 0.0f;
#pragma unroll
  for (int j = 0; j < NE; ++j) row[lane * NE + j] = base[j];
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  // the row's terms one after the other, so that an expert chosen twice gets their sum
  for (int j = 0; j < a.k; ++j) {
    if (lane == j && id >= 0) row[id] += mine;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
  if (!live) return;
  S* out = (S*)a.dlogits + t * a.E;
  for (int e = lane; e < a.E; e += L) out[e] = from_f<S>(row[e]);
}

namespace {

// Lanes and logits a lane: 16 lanes where the row and the choice fit them.  Four
// rows to a wave make a maximum over the row four shuffles for the four.
size_t route_lds(const RouteArgs& a, int rows, int L, int NE) {
  const int gs = a.E / a.groups, per = gs / NE;
  return a.groups == 1 || (gs % NE == 0 && (per & (per - 1)) == 0) ? 0 : (size_t)rows * L * NE * 8;
}
template <typename S, bool BWD, int L, int NE>
hipError_t route_go(const RouteArgs& args, hipStream_t s) {
  constexpr int rows = 256 / L, align = NE * sizeof(S) < 16 ? NE * sizeof(S) : 16;
  RouteArgs a = args;
  a.vec = a.E == L * NE && (uintptr_t)a.logits % align == 0 && a.stride * (int64_t)sizeof(S) % align == 0;
  const size_t lds = BWD ? (size_t)rows * L * NE * 4 : route_lds(a, rows, L, NE);
  if constexpr (!BWD && NE == 32) {                  // 64 KB for groups, beside the choices' 1 KB
    if (lds > 0) {
      const hipError_t err = hipFuncSetAttribute(reinterpret_cast<const void*>(k_route<S, L, NE>),
                                                 hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
      if (err != hipSuccess) return err;
    }
  }
  for (int64_t t = 0; t < args.T; t += kLaunchBlocks * rows) {
    a.T = args.T - t < kLaunchBlocks * rows ? args.T - t : kLaunchBlocks * rows;
    a.logits = (const S*)args.logits + t * a.stride;
    a.ids = args.ids + t * a.k;
    const unsigned grid = (unsigned)((a.T + rows - 1) / rows);
    if (BWD) {
      a.dweights = args.dweights + t * a.k;
      a.dlogits = (S*)args.dlogits + t * a.E;
      k_route_bwd<S, L, NE><<<grid, 256, lds, s>>>(a);
    } else {
      a.weights = args.weights + t * a.k;
      k_route<S, L, NE><<<grid, 256, lds, s>>>(a);
    }
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
  }
  return hipSuccess;
}

template <typename S, bool BWD>
hipError_t route_shape(const RouteArgs& a, hipStream_t s) {
  if (a.E > kRouteMaxE || a.k > kRouteMaxK || a.groups > kRouteMaxGroups) return hipErrorInvalidValue;
  if (a.E <= 256 && a.k <= 16 && a.groups <= 16) {
    if (a.E <= 64) return route_go<S, BWD, 16, 4>(a, s);
    if (a.E <= 128) return route_go<S, BWD, 16, 8>(a, s);
    return route_go<S, BWD, 16, 16>(a, s);
  }
  if (a.E <= 256) return route_go<S, BWD, 64, 4>(a, s);
  if (a.E <= 512) return route_go<S, BWD, 64, 8>(a, s);
  if (a.E <= 1024) return route_go<S, BWD, 64, 16>(a, s);
  return route_go<S, BWD, 64, 32>(a, s);
}

}  // namespace

template <typename S> hipError_t launch_route(const RouteArgs& a, hipStream_t s) {
  return route_shape<S, false>(a, s);
}
template <typename S> hipError_t launch_route_backward(const RouteArgs& a, hipStream_t s) {
  return route_shape<S, true>(a, s);
}
template hipError_t launch_route<float>(const RouteArgs&, hipStream_t);
template hipError_t launch_route<uint16_t>(const RouteArgs&, hipStream_t);
template hipError_t launch_route_backward<float>(const RouteArgs&, hipStream_t);
template hipError_t launch_route_backward<uint16_t>(const RouteArgs&, hipStream_t);

// ---------------------------------------------------------------- the plan
// Stable counting sort of the slots by expert.  A workgroup counts its chunk
// of slots per expert (k_plan_count), the counts become each chunk's first
// places (k_plan_scan), and the workgroup places its slots in order
// (k_plan_place): a wave takes 64 slots at a time, finds the lanes with its
// own slot's expert by one ballot per bit of the index, and the earlier ones
// among them are its rank.  Up to kPlanChunk slots the last kernel does it all.
// Integer sums alone, so the order is the same on every run.
namespace {

constexpr int kPlanWaves = 4;
constexpr int kPlanWaveSlots = kPlanChunk / kPlanWaves;

__device__ __forceinline__ int slot_expert(const int32_t* ids, int64_t i, int64_t slots, int E) {
  const int e = i < slots ? ids[i] : -1;
  return e >= 0 && e < E ? e : -1;
}

}  // namespace

__global__ __launch_bounds__(256) void k_plan_count(const int32_t* ids, int64_t slots, int E, uint32_t* counts) {
  extern __shared__ __align__(16) uint32_t cnt[];
  for (int e = threadIdx.x; e < E; e += 256) cnt[e] = 0;
  __syncthreads();
  const int64_t s0 = (int64_t)blockIdx.x * kPlanChunk;
#pragma unroll
  for (int i = 0; i < kPlanChunk / 256; ++i) {
    const int e = slot_expert(ids, s0 + i * 256 + threadIdx.x, slots, E);
    if (e >= 0) atomicAdd(&cnt[e], 1u);
  }
  __syncthreads();
  for (int e = threadIdx.x; e < E; e += 256) counts[(size_t)blockIdx.x * E + e] = cnt[e];
}

// counts [chunks][E] -> exclusive sums over the chunks; total[E].  A workgroup
// takes 64 experts, its 16 waves a range of the chunks each.
__global__ __launch_bounds__(1024) void k_plan_scan(uint32_t* counts, uint32_t* total, int chunks, int E) {
  __shared__ uint32_t part[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, e = blockIdx.x * 64 + lane;
  const int per = (chunks + 15) / 16, c0 = wave * per, c1 = min(chunks, c0 + per);
  uint32_t sum = 0;
  if (e < E) {
#pragma unroll 8
    for (int c = c0; c < c1; ++c) sum += counts[(size_t)c * E + e];
  }
  part[wave][lane] = sum;
  __syncthreads();
  uint32_t at = 0;
  for (int w = 0; w < wave; ++w) at += part[w][lane];
  if (e >= E) return;
  for (int c = c0; c < c1; c += 8) {                 // eight loads at once, then their stores
    uint32_t n[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) n[i] = c + i < c1 ? counts[(size_t)(c + i) * E + e] : 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (c + i < c1) counts[(size_t)(c + i) * E + e] = at;
      at += n[i];
    }
  }
  if (wave == 15) total[e] = at;
}

template <bool ONE>
__global__ __launch_bounds__(256) void k_plan_place(const int32_t* ids, int64_t slots, int E, const uint32_t* first,
                                                    const uint32_t* total, int32_t* order, int32_t* pos,
                                                    int32_t* offsets) {
  extern __shared__ __align__(16) uint32_t cnt[];     // [waves][E], then [E]
  __shared__ uint32_t wsum[kPlanWaves];
  uint32_t* start = cnt + (size_t)kPlanWaves * E;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  for (int i = tid; i < kPlanWaves * E; i += 256) cnt[i] = 0;
  __syncthreads();
  const int64_t s0 = (int64_t)blockIdx.x * kPlanChunk + wave * kPlanWaveSlots;
  int mine[kPlanWaveSlots / 64];
#pragma unroll
  for (int i = 0; i < kPlanWaveSlots / 64; ++i) {
    mine[i] = slot_expert(ids, s0 + i * 64 + lane, slots, E);
    if (mine[i] >= 0) atomicAdd(&cnt[(size_t)wave * E + mine[i]], 1u);
  }
  __syncthreads();
  // exclusive sums of the totals over the experts: thread i takes a run of them
  const int per = (E + 255) / 256, a0 = tid * per, a1 = min(E, a0 + per);
  uint32_t sum = 0;
  for (int e = a0; e < a1; ++e) {
    uint32_t n = 0;
    if (ONE)
      for (int w = 0; w < kPlanWaves; ++w) n += cnt[(size_t)w * E + e];
    else
      n = total[e];
    start[e] = n;
    sum += n;
  }
  uint32_t inc = sum;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t o = __shfl_up(inc, d, 64);
    if (lane >= d) inc += o;
  }
  if (lane == 63) wsum[wave] = inc;
  __syncthreads();
  uint32_t at = inc - sum;
  for (int w = 0; w < wave; ++w) at += wsum[w];
  for (int e = a0; e < a1; ++e) {
    const uint32_t n = start[e];
    if (blockIdx.x == 0) offsets[e] = (int32_t)at;
    uint32_t place = at + (ONE ? 0u : first[(size_t)blockIdx.x * E + e]);
    for (int w = 0; w < kPlanWaves; ++w) {           // each wave's first place
      const uint32_t c = cnt[(size_t)w * E + e];
      cnt[(size_t)w * E + e] = place;
      place += c;
    }
    at += n;
  }
  if (blockIdx.x == 0 && a1 == E && a0 < a1) offsets[E] = (int32_t)at;
  __syncthreads();
  int bits = 1;
  while ((1 << bits) < E) ++bits;
  uint32_t* next = cnt + (size_t)wave * E;
#pragma unroll
  for (int i = 0; i < kPlanWaveSlots / 64; ++i) {
    const int64_t slot = s0 + i * 64 + lane;
    if (s0 + i * 64 >= slots) break;
    const int e = mine[i];
    uint64_t same = __ballot(e >= 0);
    for (int b = 0; b < bits; ++b) {
      const uint64_t set = __ballot((e >> b) & 1);
      same &= ((e >> b) & 1) ? set : ~set;
    }
    const uint64_t earlier = same & ((1ull << lane) - 1);
    const int rank = __popcll(earlier);
    int32_t p = -1;
    if (e >= 0) p = (int32_t)(next[e] + rank);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (e >= 0 && earlier == 0) next[e] += __popcll(same);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (slot < slots) {
      pos[slot] = p;
      if (e >= 0) order[p] = (int32_t)slot;
    }
  }
}

size_t plan_workspace_bytes(int64_t slots, int E) {
  if (slots <= kPlanChunk) return 0;
  const size_t chunks = (size_t)((slots + kPlanChunk - 1) / kPlanChunk);
  return ((chunks + 1) * (size_t)E * 4 + 255) / 256 * 256;
}

hipError_t launch_route_plan(const int32_t* ids, int64_t slots, int E, uint32_t* ws, int32_t* order, int32_t* pos,
                             int32_t* offsets, hipStream_t s) {
  const size_t lds = (size_t)(kPlanWaves + 1) * E * 4;
  if (slots <= kPlanChunk) {
    k_plan_place<true><<<1, 256, lds, s>>>(ids, slots, E, nullptr, nullptr, order, pos, offsets);
    return hipGetLastError();
  }
  const int chunks = (int)((slots + kPlanChunk - 1) / kPlanChunk);
  uint32_t* total = ws + (size_t)chunks * E;
  k_plan_count<<<chunks, 256, (size_t)E * 4, s>>>(ids, slots, E, ws);
  k_plan_scan<<<(E + 63) / 64, 1024, 0, s>>>(ws, total, chunks, E);
  k_plan_place<false><<<chunks, 256, lds, s>>>(ids, slots, E, ws, total, order, pos, offsets);
  return hipGetLastError();
}

// ---------------------------------------------------------------- the join
namespace {

template <typename S, int V> struct Vec;
template <> struct Vec<float, 4> { typedef float4 T; };
template <> struct Vec<uint16_t, 4> { typedef uint2 T; };
template <> struct Vec<uint16_t, 8> { typedef uint4 T; };

// V elements at p, of which `valid` exist.  WHOLE: all of them, aligned; else one
// load or store at any address, or element by element at a row's end.
template <typename S, int V, bool WHOLE>
__device__ __forceinline__ void load_f(const S* p, int valid, float (&f)[V]) {
  S e[V];
  if (WHOLE) {
    typename Vec<S, V>::T v = *reinterpret_cast<const typename Vec<S, V>::T*>(p);
    __builtin_memcpy(e, &v, sizeof(e));
  } else if (valid >= V) {
    __builtin_memcpy(e, p, sizeof(e));
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) e[i] = i < valid ? p[i] : (S)0;
  }
#pragma unroll
  for (int i = 0; i < V; ++i) f[i] = to_f<S>(e[i]);
}
template <typename S, int V, bool WHOLE>
__device__ __forceinline__ void store_f(S* p, int valid, const float (&f)[V]) {
  S e[V];
#pragma unroll
  for (int i = 0; i < V; ++i) e[i] = from_f<S>(f[i]);
  if (WHOLE) {
    typename Vec<S, V>::T v;
    __builtin_memcpy(&v, e, sizeof(v));
    *reinterpret_cast<typename Vec<S, V>::T*>(p) = v;
  } else if (valid >= V) {
    __builtin_memcpy(p, e, sizeof(e));
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i < valid) p[i] = e[i];
  }
}

}  // namespace

// y[t] = sum_j w[t][j] rows[pos[t][j]], summed in j's order in 32 bits and
// rounded once; a slot without a row adds w 0.  A thread takes V columns of a row t.
template <typename S, typename O, int V, bool WHOLE>
__global__ __launch_bounds__(256) void k_combine(CombineArgs a, uint32_t cols, uint32_t total) {
  const uint32_t i = blockIdx.x * 256 + threadIdx.x;
  if (i >= total) return;
  const int64_t t = i / cols;
  const int c = (int)(i - (uint32_t)t * cols) * V;
  float acc[V];
#pragma unroll
  for (int v = 0; v < V; ++v) acc[v] = 0.0f;
  const int32_t* pos = a.pos + t * a.k;
  const float* w = a.weights ? a.weights + t * a.k : nullptr;
#pragma unroll 4
  for (int j = 0; j < a.k; ++j) {
    const int32_t p = (uint32_t)pos[j] < (uint32_t)a.S ? pos[j] : -1;
    const float wj = w ? w[j] : 1.0f;
    float x[V];
    if (p >= 0) {
      load_f<S, V, WHOLE>((const S*)a.rows + (int64_t)p * a.rows_stride + c, a.N - c, x);
    } else {
#pragma unroll
      for (int v = 0; v < V; ++v) x[v] = 0.0f;
    }
#pragma unroll
    for (int v = 0; v < V; ++v) acc[v] = fmaf(wj, x[v], acc[v]);
  }
  store_f<O, V, WHOLE>((O*)a.y + t * a.y_stride + c, a.N - c, acc);
}

// Slot (t, j): drows[pos] = w dy[t], dweights[t][j] = sum_n dy[t][n] rows[pos][n].
// One wave per slot; the slots of a row follow each other, so dy comes from the caches.
template <typename S, int V, bool WHOLE>
__global__ __launch_bounds__(256) void k_combine_bwd(CombineArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t slot = a.slot0 + (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (slot >= a.T * a.k) return;
  const int64_t t = slot / a.k;
  const int32_t p = (uint32_t)a.pos[slot] < (uint32_t)a.S ? a.pos[slot] : -1;
  float dot = 0.0f;
  if (p >= 0) {
    const S* dy = (const S*)a.y + t * a.y_stride;
    const S* row = (const S*)a.rows + (int64_t)p * a.rows_stride;
    S* drow = (S*)a.drows + (int64_t)p * a.N;
    const float w = a.weights ? a.weights[slot] : 1.0f;
#pragma unroll 2
    for (int c = lane * V; c < a.N; c += 64 * V) {
      float d[V], x[V];
      load_f<S, V, WHOLE>(dy + c, a.N - c, d);
      if (a.dweights) {
        load_f<S, V, WHOLE>(row + c, a.N - c, x);
#pragma unroll
        for (int v = 0; v < V; ++v) dot = fmaf(d[v], x[v], dot);
      }
      if (a.drows) {
#pragma unroll
        for (int v = 0; v < V; ++v) x[v] = w * d[v];
        store_f<S, V, WHOLE>(drow + c, a.N - c, x);
      }
    }
  }
  if (!a.dweights) return;
  dot = row_reduce<64>(dot, [](float x, float y) { return x + y; });
  if (lane == 0) a.dweights[slot] = dot;
}

namespace {
bool vec_ok(const void* p, int64_t stride, int N, int V, size_t elt) {
  return N % V == 0 && stride % V == 0 && (uintptr_t)p % (V * elt) == 0;
}
}  // namespace

template <typename S, typename O>
hipError_t launch_combine(const CombineArgs& args, hipStream_t s) {
  CombineArgs a = args;
  const bool whole = vec_ok(a.rows, a.rows_stride, a.N, 4, sizeof(S)) && vec_ok(a.y, a.y_stride, a.N, 4, sizeof(O));
  const uint32_t cols = (uint32_t)(a.N + 3) / 4;
  const int64_t most = kLaunchBlocks * 256 / cols;   // rows of a launch
  for (int64_t t = 0; t < args.T; t += most) {
    a.T = args.T - t < most ? args.T - t : most;
    a.pos = args.pos + t * a.k;
    a.weights = args.weights ? args.weights + t * a.k : nullptr;
    a.y = (O*)args.y + t * a.y_stride;
    const uint32_t total = (uint32_t)(a.T * cols), grid = (total + 255) / 256;
    if (whole) k_combine<S, O, 4, true><<<grid, 256, 0, s>>>(a, cols, total);
    else k_combine<S, O, 4, false><<<grid, 256, 0, s>>>(a, cols, total);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
  }
  return hipSuccess;
}
template hipError_t launch_combine<float, float>(const CombineArgs&, hipStream_t);
template hipError_t launch_combine<float, uint16_t>(const CombineArgs&, hipStream_t);
template hipError_t launch_combine<uint16_t, float>(const CombineArgs&, hipStream_t);
template hipError_t launch_combine<uint16_t, uint16_t>(const CombineArgs&, hipStream_t);

template <typename S>
hipError_t launch_combine_backward(const CombineArgs& args, hipStream_t s) {
  constexpr int V = 16 / sizeof(S);
  CombineArgs a = args;
  const bool vec = vec_ok(a.y, a.y_stride, a.N, V, sizeof(S)) &&
                   (!a.dweights || vec_ok(a.rows, a.rows_stride, a.N, V, sizeof(S))) &&
                   (!a.drows || vec_ok(a.drows, a.N, a.N, V, sizeof(S)));
  const int64_t slots = a.T * a.k;
  for (a.slot0 = 0; a.slot0 < slots; a.slot0 += kLaunchBlocks * 4) {
    const int64_t left = slots - a.slot0;
    const unsigned grid = (unsigned)(left < kLaunchBlocks * 4 ? (left + 3) / 4 : kLaunchBlocks);
    if (vec) k_combine_bwd<S, V, true><<<grid, 256, 0, s>>>(a);
    else k_combine_bwd<S, V, false><<<grid, 256, 0, s>>>(a);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
  }
  return hipSuccess;
}
template hipError_t launch_combine_backward<float>(const CombineArgs&, hipStream_t);
template hipError_t launch_combine_backward<uint16_t>(const CombineArgs&, hipStream_t);

}  // namespace gevo
