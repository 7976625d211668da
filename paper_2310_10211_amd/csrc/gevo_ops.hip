// C-ABI of the routed and 4-bit operators (declared in include/gevo.h): checks
// the arguments on the host and enqueues the kernels on the caller's stream.
#include <math.h>

#include "gevo.h"
#include "gevo_internal.h"
#include "gevo_ops.h"

using namespace gevo;

namespace {

constexpr int64_t kMaxSlots = 0x7fffffffll;
constexpr uint32_t kMaxDim = 1u << 20;

bool dtype_ok(gevo_dtype d) { return d == GEVO_F32 || d == GEVO_BF16; }
size_t elt(gevo_dtype d) { return d == GEVO_BF16 ? 2 : 4; }
bool ptr_ok(const void* p, size_t align) { return p && (uintptr_t)p % align == 0; }
bool opt_ok(const void* p, size_t align) { return (uintptr_t)p % align == 0; }

gevo_status done(hipError_t e) {
  if (e == hipSuccess) return GEVO_OK;
  return e == hipErrorInvalidValue ? GEVO_E_UNSUPPORTED : GEVO_E_HIP;
}

gevo_status route_check(const gevo_route_config* c, bool forward) {
  if (!c || c->abi_version != GEVO_ABI_VERSION || !dtype_ok(c->dtype)) return GEVO_E_ARG;
  if (c->score != GEVO_SCORE_SOFTMAX && c->score != GEVO_SCORE_SIGMOID) return GEVO_E_ARG;
  if (c->renorm > 1 || !isfinite(c->scale)) return GEVO_E_ARG;
  if (c->T < 0 || c->E < 1 || c->k < 1 || c->k > c->E || c->logits_stride < (int64_t)c->E) return GEVO_E_SHAPE;
  if (forward) {
    if (c->group_top < 1 || c->group_top > 2) return GEVO_E_ARG;
    if (c->groups < 1 || c->top_groups < 1 || c->top_groups > c->groups || c->E % c->groups) return GEVO_E_SHAPE;
    if (c->groups > GEVO_MAX_GROUPS) return GEVO_E_UNSUPPORTED;
  }
  if (c->E > GEVO_MAX_EXPERTS || c->k > GEVO_MAX_TOP_K || c->T > kMaxSlots / c->k) return GEVO_E_UNSUPPORTED;
  return GEVO_OK;
}

RouteArgs route_args(const gevo_route_config* c) {
  RouteArgs a{};
  a.stride = c->logits_stride;
  a.T = c->T;
  a.E = (int)c->E;
  a.k = (int)c->k;
  a.groups = a.top_groups = a.group_top = 1;
  a.sigmoid = c->score == GEVO_SCORE_SIGMOID;
  a.renorm = (int)c->renorm;
  a.scale = c->scale;
  return a;
}

gevo_status expert_check(const gevo_expert_config* c) {
  if (!c || c->abi_version != GEVO_ABI_VERSION || !dtype_ok(c->dtype) || !dtype_ok(c->out_dtype)) return GEVO_E_ARG;
  if (c->sorted_rows > 1 || c->relu > 1) return GEVO_E_ARG;
  if (c->T < 0 || c->E < 1 || c->k < 1 || c->N < 1 || c->K < 1) return GEVO_E_SHAPE;
  if (c->x_stride < (int64_t)c->K || c->w_stride_n < (int64_t)c->K || c->y_stride < (int64_t)c->N) return GEVO_E_SHAPE;
  if (c->E > GEVO_MAX_EXPERTS || c->N > kMaxDim || c->K > kMaxDim || c->T > kMaxSlots / c->k) return GEVO_E_UNSUPPORTED;
  const int64_t far = (int64_t)1 << 40;            // (products with sizes stay inside 63 bits)
  if (c->x_stride > far || c->w_stride_n > far || c->w_stride_e > ((int64_t)1 << 50) || c->y_stride > far)
    return GEVO_E_UNSUPPORTED;
  if (c->E > 1 && c->w_stride_e < (int64_t)(c->N - 1) * c->w_stride_n + c->K) return GEVO_E_SHAPE;
  return GEVO_OK;
}

ExpertArgs expert_args(const gevo_expert_config* c, const int32_t* order, const int32_t* offsets) {
  ExpertArgs a{};
  a.E = (int)c->E;
  a.N = (int)c->N;
  a.K = (int)c->K;
  a.S = c->T * c->k;
  a.offsets = offsets;
  a.order = c->sorted_rows ? nullptr : order;
  a.k = (int)c->k;
  a.xrows = c->sorted_rows ? a.S : c->T;
  return a;
}

gevo_status combine_check(const gevo_combine_config* c) {
  if (!c || c->abi_version != GEVO_ABI_VERSION || !dtype_ok(c->dtype) || !dtype_ok(c->out_dtype)) return GEVO_E_ARG;
  if (c->T < 0 || c->k < 1 || c->N < 1) return GEVO_E_SHAPE;
  if (c->rows_stride < (int64_t)c->N || c->y_stride < (int64_t)c->N) return GEVO_E_SHAPE;
  const int64_t far = (int64_t)1 << 31;
  if (c->N > kMaxDim || c->T > kMaxSlots / c->k || c->rows_stride > far || c->y_stride > far) return GEVO_E_UNSUPPORTED;
  return GEVO_OK;
}

CombineArgs combine_args(const gevo_combine_config* c, const void* rows, const int32_t* pos, const float* weights) {
  CombineArgs a{};
  a.T = c->T;
  a.S = c->T * c->k;
  a.k = (int)c->k;
  a.N = (int)c->N;
  a.rows = rows;
  a.rows_stride = c->rows_stride;
  a.weights = weights;
  a.pos = pos;
  a.y_stride = c->y_stride;
  return a;
}

gevo_status mx4_check(gevo_dtype dtype, int64_t rows, uint32_t K, const void* x, int64_t stride, const void* codes,
                      const void* scales) {
  if (!dtype_ok(dtype)) return GEVO_E_ARG;
  if (rows < 0 || K < 1 || stride < (int64_t)K) return GEVO_E_SHAPE;
  if (K > kMaxDim || rows > kMaxSlots || stride > (int64_t)1 << 31) return GEVO_E_UNSUPPORTED;
  if (rows > 0 && (!ptr_ok(x, elt(dtype)) || !ptr_ok(codes, 16) || !ptr_ok(scales, 4))) return GEVO_E_ARG;
  return GEVO_OK;
}

}  // namespace

extern "C" {

gevo_status gevo_route(const gevo_route_config* c, const void* logits, const float* bias, float* weights, int32_t* ids,
                       void* stream) {
  const gevo_status st = route_check(c, true);
  if (st != GEVO_OK) return st;
  if (c->T == 0) return GEVO_OK;
  if (!ptr_ok(logits, elt(c->dtype)) || !opt_ok(bias, 4) || !ptr_ok(weights, 4) || !ptr_ok(ids, 4)) return GEVO_E_ARG;
  RouteArgs a = route_args(c);
  a.logits = logits;
  a.bias = bias;
  a.groups = (int)c->groups;
  a.top_groups = (int)c->top_groups;
  a.group_top = (int)c->group_top;
  a.by_logit = !bias && (c->group_top == 1 || c->groups == 1);
  a.weights = weights;
  a.ids = ids;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  return done(c->dtype == GEVO_BF16 ? launch_route<uint16_t>(a, s) : launch_route<float>(a, s));
}

gevo_status gevo_route_backward(const gevo_route_config* c, const void* logits, const int32_t* ids,
                                const float* dweights, void* dlogits, void* stream) {
  const gevo_status st = route_check(c, false);
  if (st != GEVO_OK) return st;
  if (c->T == 0) return GEVO_OK;
  if (!ptr_ok(logits, elt(c->dtype)) || !ptr_ok(ids, 4) || !ptr_ok(dweights, 4) || !ptr_ok(dlogits, elt(c->dtype)))
    return GEVO_E_ARG;
  RouteArgs a = route_args(c);
  a.logits = logits;
  a.ids = const_cast<int32_t*>(ids);
  a.dweights = dweights;
  a.dlogits = dlogits;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  return done(c->dtype == GEVO_BF16 ? launch_route_backward<uint16_t>(a, s) : launch_route_backward<float>(a, s));
}

gevo_status gevo_route_plan_bytes(int64_t slots, uint32_t E, size_t* bytes) {
  if (!bytes) return GEVO_E_ARG;
  if (slots < 0 || E < 1) return GEVO_E_SHAPE;
  if (slots > kMaxSlots || E > GEVO_MAX_EXPERTS) return GEVO_E_UNSUPPORTED;
  *bytes = plan_workspace_bytes(slots, (int)E);
  return GEVO_OK;
}

gevo_status gevo_route_plan(int64_t slots, uint32_t E, const int32_t* ids, void* ws, size_t ws_bytes, int32_t* order,
                            int32_t* pos, int32_t* offsets, void* stream) {
  size_t need = 0;
  const gevo_status st = gevo_route_plan_bytes(slots, E, &need);
  if (st != GEVO_OK) return st;
  if (!ptr_ok(offsets, 4)) return GEVO_E_ARG;
  if (slots > 0 && (!ptr_ok(ids, 4) || !ptr_ok(order, 4) || !ptr_ok(pos, 4))) return GEVO_E_ARG;
  if (need > 0 && (!ptr_ok(ws, 4) || ws_bytes < need)) return GEVO_E_WORKSPACE;
  return done(launch_route_plan(ids, slots, (int)E, static_cast<uint32_t*>(ws), order, pos, offsets,
                                static_cast<hipStream_t>(stream)));
}

gevo_status gevo_expert_forward(const gevo_expert_config* c, const void* x, const void* w, const float* bias,
                                const int32_t* order, const int32_t* offsets, void* out, void* stream) {
  const gevo_status st = expert_check(c);
  if (st != GEVO_OK) return st;
  if (c->T == 0) return GEVO_OK;
  const size_t e = elt(c->dtype);
  if (!ptr_ok(x, e) || !ptr_ok(w, e) || !opt_ok(bias, 4) || !ptr_ok(offsets, 4) || !ptr_ok(out, elt(c->out_dtype)))
    return GEVO_E_ARG;
  if (!c->sorted_rows && !ptr_ok(order, 4)) return GEVO_E_ARG;
  ExpertArgs a = expert_args(c, order, offsets);
  a.x = x;
  a.x_stride = c->x_stride * (int64_t)e;
  a.w = w;
  a.w_e = c->w_stride_e * (int64_t)e;
  a.w_n = c->w_stride_n * (int64_t)e;
  a.bias = bias;
  a.relu = (int)c->relu;
  a.out = out;
  a.out_stride = c->y_stride;
  return done(launch_expert_forward(a, c->dtype == GEVO_BF16 ? kTypeBf16 : kTypeF32, c->out_dtype == GEVO_BF16,
                                    static_cast<hipStream_t>(stream)));
}

gevo_status gevo_expert_backward(const gevo_expert_config* c, const void* dy, const void* x, const void* w,
                                 const int32_t* order, const int32_t* offsets, void* dx, float* dw, float* db,
                                 void* stream) {
  const gevo_status st = expert_check(c);
  if (st != GEVO_OK) return st;
  const size_t e = elt(c->dtype);
  const bool rows = c->T > 0;
  if (!ptr_ok(offsets, 4) || (rows && !ptr_ok(dy, e))) return GEVO_E_ARG;
  if (!opt_ok(dx, e) || !opt_ok(dw, 4) || !opt_ok(db, 4)) return GEVO_E_ARG;
  if (dx && !ptr_ok(w, e)) return GEVO_E_ARG;
  if (rows && (dw || (dx && c->relu)) && !ptr_ok(x, e)) return GEVO_E_ARG;
  if (rows && !c->sorted_rows && !ptr_ok(order, 4)) return GEVO_E_ARG;
  if (db && !dw) return GEVO_E_ARG;                // its sums are formed beside dw's
  const ExpertType type = c->dtype == GEVO_BF16 ? kTypeBf16 : kTypeF32;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (dx && rows) {                                // rows of dy times W_e: contraction N, output columns K
    ExpertArgs a = expert_args(c, order, offsets);
    a.N = (int)c->K;
    a.K = (int)c->N;
    a.mask_order = a.order;
    a.mask_rows = a.xrows;
    a.order = nullptr;
    a.xrows = a.S;
    a.x = dy;
    a.x_stride = c->y_stride * (int64_t)e;
    a.w = w;
    a.w_e = c->w_stride_e * (int64_t)e;
    a.w_n = c->w_stride_n * (int64_t)e;
    a.mask = c->relu ? x : nullptr;
    a.mask_stride = c->x_stride * (int64_t)e;
    a.out = dx;
    a.out_stride = c->K;
    const gevo_status r = done(launch_expert_dx(a, type, s));
    if (r != GEVO_OK) return r;
  }
  if (dw) {
    ExpertArgs a = expert_args(c, order, offsets);
    a.x = x;
    a.x_stride = c->x_stride * (int64_t)e;
    a.w = dy;
    a.w_n = c->y_stride * (int64_t)e;
    a.out = dw;
    a.out_stride = c->K;
    a.db = db;
    return done(launch_expert_dw(a, type, s));
  }
  return GEVO_OK;
}

gevo_status gevo_expert_combine(const gevo_combine_config* c, const void* rows, const int32_t* pos,
                                const float* weights, void* y, void* stream) {
  const gevo_status st = combine_check(c);
  if (st != GEVO_OK) return st;
  if (c->T == 0) return GEVO_OK;
  if (!ptr_ok(rows, elt(c->dtype)) || !ptr_ok(pos, 4) || !opt_ok(weights, 4) || !ptr_ok(y, elt(c->out_dtype)))
    return GEVO_E_ARG;
  CombineArgs a = combine_args(c, rows, pos, weights);
  a.y = y;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (c->dtype == GEVO_BF16)
    return done(c->out_dtype == GEVO_BF16 ? launch_combine<uint16_t, uint16_t>(a, s) : launch_combine<uint16_t, float>(a, s));
  return done(c->out_dtype == GEVO_BF16 ? launch_combine<float, uint16_t>(a, s) : launch_combine<float, float>(a, s));
}

gevo_status gevo_expert_combine_backward(const gevo_combine_config* c, const void* dy, const void* rows,
                                         const int32_t* pos, const float* weights, void* drows, float* dweights,
                                         void* stream) {
  const gevo_status st = combine_check(c);
  if (st != GEVO_OK) return st;
  if (c->T == 0 || (!drows && !dweights)) return GEVO_OK;
  const size_t e = elt(c->dtype);
  if (!ptr_ok(dy, e) || !ptr_ok(pos, 4) || !opt_ok(weights, 4) || !opt_ok(drows, e) || !opt_ok(dweights, 4))
    return GEVO_E_ARG;
  if (dweights && !ptr_ok(rows, e)) return GEVO_E_ARG;
  CombineArgs a = combine_args(c, rows, pos, weights);
  a.y = const_cast<void*>(dy);
  a.drows = drows;
  a.dweights = dweights;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  return done(c->dtype == GEVO_BF16 ? launch_combine_backward<uint16_t>(a, s) : launch_combine_backward<float>(a, s));
}

gevo_status gevo_mx4_quantize(gevo_dtype dtype, int64_t rows, uint32_t K, const void* x, int64_t stride, uint8_t* codes,
                              uint8_t* scales, void* stream) {
  const gevo_status st = mx4_check(dtype, rows, K, x, stride, codes, scales);
  if (st != GEVO_OK || rows == 0) return st;
  const Mx4Args a{rows, (int)K, round_up((int)K, 128), x, stride, codes, scales};
  const hipStream_t s = static_cast<hipStream_t>(stream);
  return done(dtype == GEVO_BF16 ? launch_mx4_quantize<uint16_t>(a, s) : launch_mx4_quantize<float>(a, s));
}

gevo_status gevo_mx4_dequantize(gevo_dtype dtype, int64_t rows, uint32_t K, const uint8_t* codes, const uint8_t* scales,
                                void* x, int64_t stride, void* stream) {
  const gevo_status st = mx4_check(dtype, rows, K, x, stride, codes, scales);
  if (st != GEVO_OK || rows == 0) return st;
  const Mx4Args a{rows, (int)K, round_up((int)K, 128), x, stride, const_cast<uint8_t*>(codes),
                  const_cast<uint8_t*>(scales)};
  const hipStream_t s = static_cast<hipStream_t>(stream);
  return done(dtype == GEVO_BF16 ? launch_mx4_dequantize<uint16_t>(a, s) : launch_mx4_dequantize<float>(a, s));
}

gevo_status gevo_mx4_matmul(const gevo_mx4_config* c, const uint8_t* a_codes, const uint8_t* a_scales,
                            const uint8_t* b_codes, const uint8_t* b_scales, const float* bias, const int32_t* order,
                            const int32_t* offsets, void* out, void* stream) {
  if (!c || c->abi_version != GEVO_ABI_VERSION || !dtype_ok(c->out_dtype)) return GEVO_E_ARG;
  if (c->a_each > 1 || c->relu > 1 || c->sorted_rows > 1) return GEVO_E_ARG;
  if (c->M < 0 || c->P < 1 || c->N < 1 || c->K < 1) return GEVO_E_SHAPE;
  if (offsets && (c->k < 1 || c->a_each)) return GEVO_E_SHAPE;
  if (c->N > kMaxDim || c->K > kMaxDim || c->M > kMaxSlots / (offsets ? c->k : c->P)) return GEVO_E_UNSUPPORTED;
  if (offsets && c->P > GEVO_MAX_EXPERTS) return GEVO_E_UNSUPPORTED;
  if (c->M == 0) return GEVO_OK;
  if (!ptr_ok(a_codes, 16) || !ptr_ok(a_scales, 4) || !ptr_ok(b_codes, 16) || !ptr_ok(b_scales, 4)) return GEVO_E_ARG;
  if (!opt_ok(bias, 4) || !opt_ok(offsets, 4) || !ptr_ok(out, elt(c->out_dtype))) return GEVO_E_ARG;
  if (offsets && !c->sorted_rows && !ptr_ok(order, 4)) return GEVO_E_ARG;
  ExpertArgs a{};
  a.E = (int)c->P;
  a.N = (int)c->N;
  a.K = (int)c->K;
  a.M = c->M;
  a.S = c->M * (offsets ? c->k : c->P);
  a.offsets = offsets;
  a.order = c->sorted_rows ? nullptr : order;
  a.k = (int)c->k;
  a.xrows = offsets && c->sorted_rows ? a.S : c->M;
  const int64_t row = round_up((int)c->K, 128) / 2;
  a.x = a_codes;
  a.x_stride = row;
  a.xs = a_scales;
  a.xs_stride = row / 16;
  if (c->a_each) {
    a.x_e = c->M * row;
    a.xs_e = c->M * (row / 16);
  }
  a.w = b_codes;
  a.w_n = row;
  a.w_e = c->N * row;
  a.ws = b_scales;
  a.ws_n = row / 16;
  a.ws_e = c->N * (row / 16);
  a.bias = bias;
  a.relu = (int)c->relu;
  a.out = out;
  a.out_stride = c->N;
  return done(launch_expert_forward(a, kTypeMx4, c->out_dtype == GEVO_BF16, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
