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

// sign and index of the E2M1 value nearest to v (already divided by the scale),
// ties to even.  Between 0 and 2 the values are 0.5 apart, to 4 by 1, to 6 by
// 2: a / step is rounded to an integer, whose parity is the index's.
__device__ __forceinline__ uint32_t e2m1(float v) {
  const float a = fabsf(v);
  const float inv = a < 2.0f ? 2.0f : (a < 4.0f ? 1.0f : 0.5f);
  const uint32_t add = a < 2.0f ? 0u : (a < 4.0f ? 2u : 4u);
  const uint32_t i = min((uint32_t)rintf(a * inv) + add, 7u);
  return i | ((__float_as_uint(v) >> 28) & 8u);
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
#pragma unroll
    for (int m = 1; m < 32 / V; m <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, m, 64));
    // X + 127 is the exponent field less 2; numbers below 2^-125 take the smallest scale
    const int field = (int)(top >> 23);
    const bool bad = field == 255;
    const int X = max(field - 2, 0) - 127;
    const float inv = ldexpf(1.0f, -X);
    uint32_t code = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) code |= e2m1(v[i] * inv) << (4 * i);
    if (bad) code = 0;
    uint8_t* c = a.codes + r * (a.Kp / 2) + k / 2;
    if (V == 8) *reinterpret_cast<uint32_t*>(c) = code;
    else *reinterpret_cast<uint16_t*>(c) = (uint16_t)code;
    if ((k & 31) == 0) a.scales[r * (a.Kp / 32) + k / 32] = bad ? 255 : (uint8_t)(X + 127);
  }
}

// Eight values a lane: 4 bytes of codes.
template <typename S, bool VEC>
__global__ __launch_bounds__(256) void k_mx4_dequantize(Mx4Args a) {
  const int lane = threadIdx.x & 63;
  const int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (r >= a.rows) return;
  S* row = (S*)const_cast<void*>(a.x) + r * a.stride;
  const int seg = (a.Kp + gridDim.y - 1) / gridDim.y;
  const int k_end = min(a.K, (int)(blockIdx.y + 1) * seg);
  for (int k = (int)blockIdx.y * seg + lane * 8; k < k_end; k += 512) {
    const uint32_t code = *reinterpret_cast<const uint32_t*>(a.codes + r * (a.Kp / 2) + k / 2);
    const int sc = a.scales[r * (a.Kp / 32) + k / 32];
    const float scale = sc == 255 ? __uint_as_float(0x7fc00000u) : ldexpf(1.0f, sc - 127);
    S e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t q = (code >> (4 * i)) & 15, m = q & 7;
      // index m: exponent m / 2, one mantissa bit; 0 and 0.5 below them
      const float mag = m < 2 ? 0.5f * (float)m : __uint_as_float((126u + (m >> 1)) << 23 | (m & 1) << 22);
      e[i] = Op<S>::from_f32((q & 8 ? -mag : mag) * scale);
    }
    if (VEC && k + 8 <= a.K) {
      uint4 u[sizeof(S) / 2];
      __builtin_memcpy(u, e, sizeof(u));
#pragma unroll
      for (int i = 0; i < (int)sizeof(S) / 2; ++i) reinterpret_cast<uint4*>(row + k)[i] = u[i];
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (k + i < a.K) row[k + i] = e[i];
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

template <typename S> hipError_t launch_mx4_quantize(const Mx4Args& a, hipStream_t s) {
  if ((a.rows + 3) / 4 > 0x7fffffff) return hipErrorInvalidValue;
  const bool vec = (uintptr_t)a.x % 16 == 0 && a.stride * sizeof(S) % 16 == 0;
  if (vec) k_mx4_quantize<S, true><<<mx4_grid(a), 256, 0, s>>>(a);
  else k_mx4_quantize<S, false><<<mx4_grid(a), 256, 0, s>>>(a);
  return hipGetLastError();
}
template <typename S> hipError_t launch_mx4_dequantize(const Mx4Args& a, hipStream_t s) {
  if ((a.rows + 3) / 4 > 0x7fffffff) return hipErrorInvalidValue;
  const bool vec = (uintptr_t)a.x % 16 == 0 && a.stride * sizeof(S) % 16 == 0;
  if (vec) k_mx4_dequantize<S, true><<<mx4_grid(a), 256, 0, s>>>(a);
  else k_mx4_dequantize<S, false><<<mx4_grid(a), 256, 0, s>>>(a);
  return hipGetLastError();
}
template hipError_t launch_mx4_quantize<float>(const Mx4Args&, hipStream_t);
template hipError_t launch_mx4_quantize<uint16_t>(const Mx4Args&, hipStream_t);
template hipError_t launch_mx4_dequantize<float>(const Mx4Args&, hipStream_t);
template hipError_t launch_mx4_dequantize<uint16_t>(const Mx4Args&, hipStream_t);

}  // namespace gevo
