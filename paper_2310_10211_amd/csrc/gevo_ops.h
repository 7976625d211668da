// Internal declarations of the routed and 4-bit operators (gevo_route.hip,
// gevo_mx4.hip, gevo_experts.hip; C-ABI in gevo_ops.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace gevo {

constexpr int kRouteMaxE = 2048;      // experts a row is routed over
constexpr int kRouteMaxK = 64;        // of them chosen for a row
constexpr int kRouteMaxGroups = 64;
constexpr int kPlanChunk = 1024;      // slots a workgroup of the plan kernels sorts
// A launch counts its work-items in 32 bits and drops the rest without an error:
// rows past this many workgroups of 256 go out in further launches.
constexpr int64_t kLaunchBlocks = 1 << 23;

struct RouteArgs {
  const void* logits; int64_t stride;  // [T] rows, elements apart
  const float* bias;                   // [E] (nullable): added for the choice alone
  int64_t T;
  int E, k, groups, top_groups, group_top;
  int sigmoid, renorm, by_logit;       // by_logit: the logits themselves are the keys
  int vec;                             // set by the launcher: rows are aligned and fill the lanes
  float scale;
  float* weights; int32_t* ids;        // [T][k]
  const float* dweights;               // backward: [T][k]
  void* dlogits;                       // backward: [T][E]
};
template <typename S> hipError_t launch_route(const RouteArgs& a, hipStream_t s);
template <typename S> hipError_t launch_route_backward(const RouteArgs& a, hipStream_t s);

size_t plan_workspace_bytes(int64_t slots, int E);
hipError_t launch_route_plan(const int32_t* ids, int64_t slots, int E, uint32_t* ws, int32_t* order, int32_t* pos,
                             int32_t* offsets, hipStream_t s);

struct CombineArgs {
  int64_t T, S;                            // S: sorted rows
  int k, N;
  const void* rows; int64_t rows_stride;   // sorted rows
  const float* weights;                    // [T][k] (nullable: ones)
  const int32_t* pos;                      // [T][k]
  void* y; int64_t y_stride;               // combine: out; backward: the gradient dy
  int64_t slot0;                           // set by the launcher: backward: the launch's first slot
  void* drows; float* dweights;            // backward (either nullable)
};
template <typename S, typename O> hipError_t launch_combine(const CombineArgs& a, hipStream_t s);
template <typename S> hipError_t launch_combine_backward(const CombineArgs& a, hipStream_t s);

struct Mx4Args {
  int64_t rows;
  int K, Kp;                               // Kp: K rounded up to 128
  const void* x; int64_t stride;
  uint8_t* codes; uint8_t* scales;         // [rows][Kp / 2], [rows][Kp / 32]
};
template <typename S> hipError_t launch_mx4_quantize(const Mx4Args& a, hipStream_t s);
template <typename S> hipError_t launch_mx4_dequantize(const Mx4Args& a, hipStream_t s);

// Products of rows with one weight matrix per expert.  Segment e holds the
// sorted rows offsets[e] .. offsets[e + 1), or M rows (dense: offsets null).
struct ExpertArgs {
  int E, N, K;                             // output [row][N], contraction K (elements)
  int64_t S;                               // sorted rows in all (dense: E M)
  int64_t M;                               // dense: rows of a segment
  const int32_t* offsets;                  // [E + 1]
  const int32_t* order;                    // row of x of sorted row s: order[s] / k (null: s; dense: its place)
  int k; int64_t xrows;                    // rows of x (a place beyond them reads zeros)
  uint32_t k_mul; int k_shift;             // set by the launcher: slot / k = slot k_mul / 2^(32 + k_shift)
  const void* x; int64_t x_stride, x_e;    // bytes between rows, and (dense) between segments
  const void* w; int64_t w_e, w_n;         // bytes between experts, between rows of a matrix
  const uint8_t* xs; int64_t xs_stride, xs_e;   // 4-bit operands: scales
  const uint8_t* ws; int64_t ws_e, ws_n;
  const float* bias;                       // [E][N] (nullable)
  int relu;
  const void* mask; int64_t mask_stride;   // dx: rows of the layer's input, bytes apart, whose values <= 0 clear
  const int32_t* mask_order;               // the output (nullable); as order and xrows
  int64_t mask_rows;
  void* out; int64_t out_stride;           // elements between rows
  float* db;                               // dw: [E][N] column sums (nullable)
};
enum ExpertType { kTypeF32 = 0, kTypeBf16 = 1, kTypeMx4 = 2 };
hipError_t launch_expert_forward(const ExpertArgs& a, ExpertType type, bool out_bf16, hipStream_t s);
// dx: x = dy rows [S][K = width of dy], w read transposed (out [S][N = width of x])
hipError_t launch_expert_dx(const ExpertArgs& a, ExpertType type, hipStream_t s);
// dw: x gathered rows [.][K], w = dy sorted rows [S][N]; out [E][N][K] f32
hipError_t launch_expert_dw(const ExpertArgs& a, ExpertType type, hipStream_t s);

}  // namespace gevo
