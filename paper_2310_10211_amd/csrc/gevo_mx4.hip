// Microscaled 4-bit floating point (OCP MX, E2M1 elements): 32 consecutive
// values of a row share a power-of-two scale.
//   scale  2^X, X = floor(log2 max |v|) - 2, so the largest lies in [4, 8);
//          at least 2^-127; held as X + 127 (255: a value was no finite number)
//   code   sign and index of v / 2^X rounded to nearest even among 0, 0.5, 1,
//          1.5, 2, 3, 4, 6 (beyond 6: 6)
// Rows hold their codes two a byte, the even value low, and are padded with
// zeros to a multiple of 128 values: 64 bytes of codes and 4 of scales, which
// is one contraction step of the products.  Both kernels stream: 4.25 bits a
// value on one side, 16 or 32 on the other.
#include "gevo_internal.h"
#include "gevo_device.h"
#include "gevo_ops.h"

namespace gevo {

namespace {

// gfx950 converts pairs of values with a scale, which it takes from the exponent
// field of a binary32: to E2M1, rounding v / scale to nearest even and
// saturating at 6, and back.  (The tests compare every code and value with the
// definition, ties, halves of the smallest value and the least scale among them.)
template <int B>
__device__ __forceinline__ uint32_t to_e2m1(uint32_t code, float lo, float hi, float scale) {
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, lo, hi, scale, B);   // into byte B of code
}
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
template <int B>
__device__ __forceinline__ void from_e2m1(uint32_t code, float scale, float* v) {
  const f32x2_t p = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, scale, B);
  v[0] = p[0];
  v[1] = p[1];
}
template <int B>
__device__ __forceinline__ void from_e2m1(uint32_t code, float scale, uint16_t* v) {
  const uint32_t p = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, B));
  v[0] = (uint16_t)p;
  v[1] = (uint16_t)(p >> 16);
}

// the larger of a lane's value and another's of its 8: CTRL names the lane
template <int CTRL>
__device__ __forceinline__ uint32_t larger(uint32_t v) {
  return max(v, (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, CTRL, 0xf, 0xf, false));
}

}  // namespace

// A lane holds V consecutive values (16 bytes of them where rows allow it),
// 32 / V lanes a block; a wave takes a row's values 64 V at a time.
template <typename S, bool VEC>
__global__ __launch_bounds__(256) void k_mx4_quantize(Mx4Args a) {
  constexpr int V = 16 / sizeof(S);
  const int lane = threadIdx.x & 63;
  const int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (r >= a.rows) return;
  const S* row = (const S*)a.x + r * a.stride;
  const int seg = (a.Kp + gridDim.y - 1) / gridDim.y;         // a multiple of 128 (see the launcher)
  const int k_end = min(a.Kp, (int)(blockIdx.y + 1) * seg);
  for (int k = (int)blockIdx.y * seg + lane * V; k < k_end; k += 64 * V) {
    float v[V];
    if (VEC && k + V <= a.K) {
      S e[V];
      const uint4 u = *reinterpret_cast<const uint4*>(row + k);
      __builtin_memcpy(e, &u, 16);
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = Op<S>::to_f32(e[i]);
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = k + i < a.K ? Op<S>::to_f32(row[k + i]) : 0.0f;
    }
    // the largest magnitude, as the bits of non-negative numbers order like
    // integers (infinities and NaN above every number)
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
    top = larger<0xb1>(top);                         // lanes 1 0 3 2 of each four
    top = larger<0x4e>(top);                         // lanes 2 3 0 1
    if (V == 4) top = larger<0x141>(top);            // the other four of the eight
    // X + 127 is the exponent field less 2; numbers below 2^-125 take the smallest scale
    const int field = (int)(top >> 23);
    const bool bad = field == 255;
    const int X = max(field - 2, 0) - 127;
    const float scale = __uint_as_float((uint32_t)(X + 127) << 23);
    uint32_t code = to_e2m1<0>(0, v[0], v[1], scale);
    code = to_e2m1<1>(code, v[2], v[3], scale);
    if constexpr (V == 8) {
      code = to_e2m1<2>(code, v[4], v[5], scale);
      code = to_e2m1<3>(code, v[6], v[7], scale);
    }
    if (bad) code = 0;
    uint8_t* c = a.codes + r * (a.Kp / 2) + k / 2;
    if (V == 8) *reinterpret_cast<uint32_t*>(c) = code;
    else *reinterpret_cast<uint16_t*>(c) = (uint16_t)code;
    if ((k & 31) == 0) a.scales[r * (a.Kp / 32) + k / 32] = bad ? 255 : (uint8_t)(X + 127);
  }
}

// Eight values a lane (4 bytes of codes), kDq times: the loads of all go out
// before the first store.  Lane x of the grid takes the chunks x, x + lanes, ..
// of the rows' 8-value chunks in order.
constexpr int kDq = 4;
template <typename S, bool VEC>
__global__ __launch_bounds__(256) void k_mx4_dequantize(Mx4Args a, int64_t total, int chunks) {
  const int64_t lanes = (int64_t)gridDim.x * 256;
  for (int64_t i0 = (int64_t)blockIdx.x * 256 + threadIdx.x; i0 < total; i0 += lanes * kDq) {
    uint32_t code[kDq];
    int sc[kDq], k[kDq];
    int64_t row[kDq];
#pragma unroll
    for (int u = 0; u < kDq; ++u) {
      const int64_t i = i0 + u * lanes;
      code[u] = 0;
      sc[u] = 0;
      row[u] = total <= 0xffffffffll ? (int64_t)((uint32_t)i / (uint32_t)chunks) : i / chunks;
      k[u] = (int)(i - row[u] * chunks) * 8;
      if (i < total && k[u] < a.K) {
        code[u] = *reinterpret_cast<const uint32_t*>(a.codes + row[u] * (a.Kp / 2) + k[u] / 2);
        sc[u] = a.scales[row[u] * (a.Kp / 32) + k[u] / 32];
      }
    }
#pragma unroll
    for (int u = 0; u < kDq; ++u) {
      if (i0 + u * lanes >= total || k[u] >= a.K) continue;
      const float scale = __uint_as_float((uint32_t)sc[u] << 23);
      S e[8];
      from_e2m1<0>(code[u], scale, e);
      from_e2m1<1>(code[u], scale, e + 2);
      from_e2m1<2>(code[u], scale, e + 4);
      from_e2m1<3>(code[u], scale, e + 6);
      if (sc[u] == 255) {
#pragma unroll
        for (int v = 0; v < 8; ++v) e[v] = Op<S>::from_f32(__uint_as_float(0x7fc00000u));
      }
      S* p = (S*)const_cast<void*>(a.x) + row[u] * a.stride + k[u];
      if (VEC && k[u] + 8 <= a.K) {
        uint4 w[sizeof(S) / 2];
        __builtin_memcpy(w, e, sizeof(w));
#pragma unroll
        for (int v = 0; v < (int)sizeof(S) / 2; ++v) reinterpret_cast<uint4*>(p)[v] = w[v];
      } else {
#pragma unroll
        for (int v = 0; v < 8; ++v)
          if (k[u] + v < a.K) p[v] = e[v];
      }
    }
  }
}

namespace {
// a wave per row; rows of more than 4,096 values in segments where there are few rows
dim3 mx4_grid(const Mx4Args& a) {
  int segs = 1;
  while (segs < 16 && a.Kp % (256 * segs) == 0 && a.Kp / segs > 1024 && a.rows * segs < 4096) segs *= 2;
  return dim3((unsigned)((a.rows + 3) / 4), (unsigned)segs);
}
}  // namespace

template <typename S> hipError_t launch_mx4_quantize(const Mx4Args& args, hipStream_t s) {
  Mx4Args a = args;
  const bool vec = (uintptr_t)a.x % 16 == 0 && a.stride * sizeof(S) % 16 == 0;
  for (int64_t r = 0; r < args.rows; r += kLaunchBlocks * 4) {
    a.rows = args.rows - r < kLaunchBlocks * 4 ? args.rows - r : kLaunchBlocks * 4;
    a.x = (const S*)args.x + r * a.stride;
    a.codes = args.codes + r * (a.Kp / 2);
    a.scales = args.scales + r * (a.Kp / 32);
    if (vec) k_mx4_quantize<S, true><<<mx4_grid(a), 256, 0, s>>>(a);
    else k_mx4_quantize<S, false><<<mx4_grid(a), 256, 0, s>>>(a);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
  }
  return hipSuccess;
}
template <typename S> hipError_t launch_mx4_dequantize(const Mx4Args& a, hipStream_t s) {
  const bool vec = (uintptr_t)a.x % 16 == 0 && a.stride * sizeof(S) % 16 == 0;
  const int chunks = (a.K + 7) / 8;
  const int64_t total = a.rows * chunks, wanted = (total + 256 * kDq - 1) / (256 * kDq);
  const unsigned grid = (unsigned)(wanted < 16384 ? wanted : 16384);
  if (vec) k_mx4_dequantize<S, true><<<grid, 256, 0, s>>>(a, total, chunks);
  else k_mx4_dequantize<S, false><<<grid, 256, 0, s>>>(a, total, chunks);
  return hipGetLastError();
}
template hipError_t launch_mx4_quantize<float>(const Mx4Args&, hipStream_t);
template hipError_t launch_mx4_quantize<uint16_t>(const Mx4Args&, hipStream_t);
template hipError_t launch_mx4_dequantize<float>(const Mx4Args&, hipStream_t);
template hipError_t launch_mx4_dequantize<uint16_t>(const Mx4Args&, hipStream_t);

}  // namespace gevo
