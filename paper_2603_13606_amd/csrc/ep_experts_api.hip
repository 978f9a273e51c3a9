// C-ABI entry points of the gate, the experts' products and the layer of few tokens: checks of the
// arguments and their translation into kernel arguments.  Host code only.
#include <algorithm>
#include <cmath>

#include "ep_check.h"
#include "ep_experts.h"
#include "ep_internal.h"

using namespace ep;

namespace {

constexpr int64_t kMaxExtent = 1 << 22;      // rows' lengths and strides, elements: a tile's offsets stay below 2^31 bytes
constexpr int64_t kMaxRows = 0x7fffff00LL;   // of a window or a tensor: rounded up to blocks of 256 they are counted in 32 bits
constexpr int64_t kMaxLayerExtent = 1 << 17; // of the layer: its grid stays below 2^32 work-items
constexpr int64_t kMaxLayerRows = 1 << 30;   // elements between the layer's products: 32-bit byte offsets
constexpr int kMaxGroups = 64;

bool float_or_bf16(const ep_tensor_t* t) { return t->dtype == EP_DTYPE_F32 || t->dtype == EP_DTYPE_BF16; }

// A 2-D tensor whose number of rows is its own.
bool check_rows(const ep_tensor_t* t, int dtype, int64_t cols) {
    return t && t->ndim == 2 && t->shape[0] >= 0 && check_2d(t, dtype, t->shape[0], cols, true);
}

ep_result_t check_route(const ep_route_config_t* cfg, const ep_tensor_t* logits, const ep_tensor_t* idx, const ep_tensor_t* w) {
    if (!cfg || cfg->size != sizeof(ep_route_config_t)) return EP_ERR_INVALID_ARG;
    if (cfg->score != EP_SCORE_SOFTMAX && cfg->score != EP_SCORE_SIGMOID) return EP_ERR_INVALID_ARG;
    if (cfg->renormalise != 0 && cfg->renormalise != 1) return EP_ERR_INVALID_ARG;
    if (!std::isfinite(cfg->scale)) return EP_ERR_INVALID_ARG;
    if (!logits || logits->ndim != 2 || !float_or_bf16(logits) || !idx || idx->ndim != 2) return EP_ERR_INVALID_ARG;
    const int64_t T = logits->shape[0], E = logits->shape[1], K = idx->shape[1];
    if (E < 1 || E > kMaxExperts || K < 1 || K > kMaxTopK || T < 0 || T > (1 << 28) / K) return EP_ERR_INVALID_ARG;
    if (!check_rows(logits, logits->dtype, E) || !check_2d(idx, EP_DTYPE_I32, T, K, true) || !check_2d(w, EP_DTYPE_F32, T, K, true))
        return EP_ERR_INVALID_ARG;
    if (cfg->num_groups < 1 || cfg->num_groups > kMaxGroups || E % cfg->num_groups || cfg->groups_kept < 1 ||
        cfg->groups_kept > cfg->num_groups)
        return EP_ERR_INVALID_ARG;
    return EP_SUCCESS;
}

ep_result_t check_product_config(const ep_product_config_t* c) {
    if (!c || c->size != sizeof(ep_product_config_t)) return EP_ERR_INVALID_ARG;
    if (c->activation < EP_ACT_NONE || c->activation > EP_ACT_GELU) return EP_ERR_INVALID_ARG;
    if ((c->gated != 0 && c->gated != 1) || (c->accumulate != 0 && c->accumulate != 1) || c->first_expert < 0) return EP_ERR_INVALID_ARG;
    return EP_SUCCESS;
}

// Whether no two rows of a 3-D tensor share elements: what is written has to be.
bool apart(const ep_tensor_t* t) {
    const int64_t a = t->shape[0], b = t->shape[1], k = t->shape[2], sa = t->stride[0], sb = t->stride[1];
    if (a <= 1 || b < 1) return true;
    return sa >= (b - 1) * sb + k || (sa >= k && sb >= (a - 1) * sa + k);
}

// bf16 (or f32 where allowed) [L, n, k] with rows on 16-byte boundaries.
bool check_weights(const ep_tensor_t* t, bool f32_too = false) {
    if (!t || t->ndim != 3 || !(t->dtype == EP_DTYPE_BF16 || (f32_too && t->dtype == EP_DTYPE_F32))) return false;
    if (t->shape[0] < 1 || t->shape[0] > kMaxExperts || !t->data || !aligned16(t->data)) return false;
    if (t->shape[1] < 8 || t->shape[1] % 8 || t->shape[1] > kMaxExtent || t->shape[2] < 8 || t->shape[2] % 8 || t->shape[2] > kMaxExtent)
        return false;
    if (t->stride[2] != 1 || t->stride[1] < t->shape[2] || t->stride[1] % 8 || t->stride[1] >= kMaxExtent) return false;
    if (t->dtype == EP_DTYPE_F32 && t->stride[1] >= kMaxExtent / 2) return false;
    return t->stride[0] % 8 == 0 && t->stride[0] >= 0;
}

// [L, n] f32 or bf16, rows on 16-byte boundaries.
bool check_bias(const ep_tensor_t* t, int64_t L, int64_t n) {
    return t && float_or_bf16(t) && check_2d(t, t->dtype, L, n, true) && aligned16(t->data) && t->stride[0] % 8 == 0;
}

// The row windows of one call: where they lie on the device, and what every row tensor has to look like.
struct Rows {
    Windows win;
    int64_t tensor_experts = 0;  // padded: leading extent of the row tensors
    int64_t slots = 0;           // padded: rows per expert, once known
    int first = 0;               // padded: the expert of the tensors that the first weights belong to
    bool padded = false;
    int32_t* status = nullptr;
};

// From a handle, or from ROW_OFFSET (2-D rows only) and ROW_COUNT.
ep_result_t find_windows(ep_handle_t h, const ep_product_config_t* cfg, const ep_tensor_t* in, int n, int64_t L, const ep_tensor_t* rows,
                         Rows* r) {
    const ep_tensor_t* off = find_tag(in, n, EP_TAG_ROW_OFFSET);
    const ep_tensor_t* cnt = find_tag(in, n, EP_TAG_ROW_COUNT);
    if (!rows) return EP_ERR_INVALID_ARG;
    r->win.L = (int)L;
    if (h) {
        HandleRows hr;
        if (off || cnt) return EP_ERR_INVALID_ARG;
        handle_rows(h, &hr);
        if (cfg->first_expert + L > hr.experts) return EP_ERR_INVALID_ARG;
        r->padded = hr.padded;
        r->tensor_experts = hr.experts;
        r->slots = hr.slots;
        r->first = cfg->first_expert;
        r->win.offset = hr.padded ? nullptr : hr.offset + cfg->first_expert;
        r->win.count = hr.kept + cfg->first_expert;
        r->status = hr.status;
    } else {
        if (cfg->first_expert != 0) return EP_ERR_INVALID_ARG;
        r->padded = rows->ndim == 3;
        if (!check_1d(cnt, EP_DTYPE_I32, L) || !cnt->data || (off != nullptr) == r->padded) return EP_ERR_INVALID_ARG;
        if (off && (!check_1d(off, EP_DTYPE_I32, L) || !off->data)) return EP_ERR_INVALID_ARG;
        r->tensor_experts = L;
        r->slots = r->padded ? rows->shape[1] : 0;
        r->win.offset = off ? (const int32_t*)off->data : nullptr;
        r->win.count = (const int32_t*)cnt->data;
    }
    r->win.cap = r->padded ? r->slots : kMaxRows;
    return EP_SUCCESS;
}

// A tensor of bf16 rows of `cols` elements in the windows of the call; the shortest tensor bounds the rows.
bool row_tensor(const ep_tensor_t* t, int64_t cols, Rows* r, RowsDesc* d, bool written = false) {
    if (!t || t->dtype != EP_DTYPE_BF16 || !aligned16(t->data)) return false;
    const int inner = r->padded ? 2 : 1;
    if (t->ndim != inner + 1 || t->shape[inner] != cols || t->stride[inner] != 1) return false;
    const int64_t row = t->stride[inner - 1];
    if (row < cols || row % 8 || row >= kMaxExtent) return false;
    if (r->padded) {
        if (t->shape[0] != r->tensor_experts || t->shape[1] != r->slots || t->shape[1] < 0 || t->shape[1] > kMaxRows) return false;
        if (t->stride[0] < 0 || t->stride[0] % 8) return false;
        if ((!t->data && t->shape[1] > 0) || (written && !apart(t))) return false;
        d->expert_stride = t->stride[0];
        d->base = (uint16_t*)t->data + r->first * t->stride[0];
    } else {
        if (t->shape[0] < 0 || t->shape[0] > kMaxRows || (!t->data && t->shape[0] > 0)) return false;
        d->expert_stride = 0;
        d->base = (uint16_t*)t->data;
        r->win.cap = std::min(r->win.cap, t->shape[0]);
    }
    d->row_stride = row;
    return true;
}

ep_result_t done(hipError_t e) { return e == hipSuccess ? EP_SUCCESS : EP_ERR_HIP; }

}  // namespace

extern "C" {

ep_result_t ep_route(const ep_route_config_t* cfg, const ep_tensor_t* inputs, int32_t num_inputs, const ep_tensor_t* outputs,
                     int32_t num_outputs, ep_stream_t stream) {
    if (!inputs || !outputs || num_inputs < 1 || num_outputs < 1) return EP_ERR_INVALID_ARG;
    const ep_tensor_t* logits = find_tag(inputs, num_inputs, EP_TAG_LOGITS);
    const ep_tensor_t* bias = find_tag(inputs, num_inputs, EP_TAG_SELECT_BIAS);
    const ep_tensor_t* idx = find_tag(outputs, num_outputs, EP_TAG_TOPK_IDX);
    const ep_tensor_t* w = find_tag(outputs, num_outputs, EP_TAG_TOPK_WEIGHTS);
    if (ep_result_t r = check_route(cfg, logits, idx, w); r != EP_SUCCESS) return r;
    if (bias && (!check_1d(bias, EP_DTYPE_F32, logits->shape[1]) || !bias->data)) return EP_ERR_INVALID_ARG;
    RouteArgs a = {};
    a.logits = logits->data; a.logits_stride = logits->stride[0]; a.logits_bf16 = logits->dtype == EP_DTYPE_BF16;
    a.bias = bias ? (const float*)bias->data : nullptr;
    a.topk_idx = (int32_t*)idx->data; a.idx_stride = idx->stride[0];
    a.topk_w = (float*)w->data; a.w_stride = w->stride[0];
    a.T = (int)logits->shape[0]; a.E = (int)logits->shape[1]; a.K = (int)idx->shape[1];
    a.score = cfg->score; a.renormalise = cfg->renormalise; a.groups = cfg->num_groups; a.kept = cfg->groups_kept;
    a.scale = cfg->scale;
    return done(launch_route(a, (hipStream_t)stream));
}

ep_result_t ep_route_backward(const ep_route_config_t* cfg, const ep_tensor_t* inputs, int32_t num_inputs, const ep_tensor_t* outputs,
                              int32_t num_outputs, ep_stream_t stream) {
    if (!inputs || !outputs || num_inputs < 1 || num_outputs < 1) return EP_ERR_INVALID_ARG;
    const ep_tensor_t* logits = find_tag(inputs, num_inputs, EP_TAG_LOGITS);
    const ep_tensor_t* idx = find_tag(inputs, num_inputs, EP_TAG_TOPK_IDX);
    const ep_tensor_t* gw = find_tag(inputs, num_inputs, EP_TAG_TOPK_WEIGHTS);
    const ep_tensor_t* gl = find_tag(outputs, num_outputs, EP_TAG_LOGITS);
    if (ep_result_t r = check_route(cfg, logits, idx, gw); r != EP_SUCCESS) return r;
    if (!check_2d(gl, logits->dtype, logits->shape[0], logits->shape[1], true)) return EP_ERR_INVALID_ARG;
    RouteBackwardArgs a = {};
    a.logits = logits->data; a.logits_stride = logits->stride[0]; a.logits_bf16 = logits->dtype == EP_DTYPE_BF16;
    a.topk_idx = (const int32_t*)idx->data; a.idx_stride = idx->stride[0];
    a.grad_w = (const float*)gw->data; a.gw_stride = gw->stride[0];
    a.grad_logits = gl->data; a.gl_stride = gl->stride[0];
    a.T = (int)logits->shape[0]; a.E = (int)logits->shape[1]; a.K = (int)idx->shape[1];
    a.score = cfg->score; a.renormalise = cfg->renormalise;
    a.scale = cfg->scale;
    return done(launch_route_backward(a, (hipStream_t)stream));
}

ep_result_t ep_expert_product(ep_handle_t handle, const ep_product_config_t* cfg, const ep_tensor_t* inputs, int32_t num_inputs,
                              const ep_tensor_t* outputs, int32_t num_outputs, ep_stream_t stream) {
    if (!inputs || !outputs || num_inputs < 1 || num_outputs < 1) return EP_ERR_INVALID_ARG;
    if (ep_result_t r = check_product_config(cfg); r != EP_SUCCESS) return r;
    const ep_tensor_t* x = find_tag(inputs, num_inputs, EP_TAG_TOKENS);
    const ep_tensor_t* w = find_tag(inputs, num_inputs, EP_TAG_EXPERT_WEIGHTS);
    const ep_tensor_t* b = find_tag(inputs, num_inputs, EP_TAG_EXPERT_BIAS);
    const ep_tensor_t* res = find_tag(inputs, num_inputs, EP_TAG_RESIDUAL);
    const ep_tensor_t* out = find_tag(outputs, num_outputs, EP_TAG_TOKENS);
    const ep_tensor_t* pre = find_tag(outputs, num_outputs, EP_TAG_PREACT);
    if (cfg->accumulate || !check_weights(w)) return EP_ERR_INVALID_ARG;
    const int64_t L = w->shape[0], N = w->shape[1], Kd = w->shape[2], No = cfg->gated ? N / 2 : N;
    if (No % 8) return EP_ERR_INVALID_ARG;
    // the up rows of a gated tile are addressed from its gate rows with 32-bit byte offsets
    if (cfg->gated && N * w->stride[1] >= (int64_t(1) << 30)) return EP_ERR_UNSUPPORTED;
    if (b && !check_bias(b, L, N)) return EP_ERR_INVALID_ARG;
    Rows r;
    if (ep_result_t e = find_windows(handle, cfg, inputs, num_inputs, L, x, &r); e != EP_SUCCESS) return e;
    ProductArgs a = {};
    if (!row_tensor(x, Kd, &r, &a.x) || !row_tensor(out, No, &r, &a.out, true) || (pre && !row_tensor(pre, N, &r, &a.pre, true)) ||
        (res && !row_tensor(res, No, &r, &a.res)))
        return EP_ERR_INVALID_ARG;
    a.win = r.win; a.status = r.status;
    a.w = (const uint16_t*)w->data; a.w_expert = w->stride[0]; a.w_row = w->stride[1];
    a.bias = b ? b->data : nullptr; a.bias_stride = b ? b->stride[0] : 0; a.bias_f32 = b && b->dtype == EP_DTYPE_F32;
    a.N = (int)N; a.No = (int)No; a.Kd = (int)Kd; a.act = cfg->activation; a.gated = cfg->gated;
    if (handle) handle_used(handle, (hipStream_t)stream);
    return done(launch_product(a, (hipStream_t)stream));
}

ep_result_t ep_expert_product_backward(ep_handle_t handle, const ep_product_config_t* cfg, const ep_tensor_t* inputs, int32_t num_inputs,
                                       const ep_tensor_t* outputs, int32_t num_outputs, ep_stream_t stream) {
    if (!inputs || !outputs || num_inputs < 1 || num_outputs < 1) return EP_ERR_INVALID_ARG;
    if (ep_result_t r = check_product_config(cfg); r != EP_SUCCESS) return r;
    const ep_tensor_t* go = find_tag(inputs, num_inputs, EP_TAG_EXPERT_TOKENS);
    const ep_tensor_t* pre = find_tag(inputs, num_inputs, EP_TAG_PREACT);
    const ep_tensor_t* x = find_tag(inputs, num_inputs, EP_TAG_TOKENS);
    const ep_tensor_t* w = find_tag(inputs, num_inputs, EP_TAG_EXPERT_WEIGHTS);
    const ep_tensor_t* gp = find_tag(outputs, num_outputs, EP_TAG_PREACT);
    const ep_tensor_t* gx = find_tag(outputs, num_outputs, EP_TAG_TOKENS);
    const ep_tensor_t* gw = find_tag(outputs, num_outputs, EP_TAG_EXPERT_WEIGHTS);
    const ep_tensor_t* gb = find_tag(outputs, num_outputs, EP_TAG_EXPERT_BIAS);
    const bool elementwise = cfg->activation != EP_ACT_NONE || cfg->gated;
    if ((gx && !w) || (!w && !gw) || (gw && !x) || (gb && !gw)) return EP_ERR_INVALID_ARG;
    if (elementwise != (pre != nullptr) || elementwise != (gp != nullptr)) return EP_ERR_INVALID_ARG;
    if ((w && !check_weights(w)) || (gw && !(check_weights(gw, true) && apart(gw)))) return EP_ERR_INVALID_ARG;
    if (w && gw)
        for (int i = 0; i < 3; ++i)
            if (w->shape[i] != gw->shape[i]) return EP_ERR_INVALID_ARG;
    const ep_tensor_t* shape = w ? w : gw;
    const int64_t L = shape->shape[0], N = shape->shape[1], Kd = shape->shape[2], No = cfg->gated ? N / 2 : N;
    if (No % 8) return EP_ERR_INVALID_ARG;
    if (gb && (gb->dtype != gw->dtype || !check_2d(gb, gb->dtype, L, N, true))) return EP_ERR_INVALID_ARG;
    Rows r;
    if (ep_result_t e = find_windows(handle, cfg, inputs, num_inputs, L, go, &r); e != EP_SUCCESS) return e;
    ActBackwardArgs act = {};
    GradRowsArgs rows = {};
    GradWeightsArgs weights = {};
    RowsDesc xd = {}, gxd = {};
    if (!row_tensor(go, No, &r, &act.grad_out)) return EP_ERR_INVALID_ARG;
    RowsDesc grad_pre = act.grad_out;
    if (elementwise) {
        if (!row_tensor(pre, N, &r, &act.pre) || !row_tensor(gp, N, &r, &act.grad_pre, true)) return EP_ERR_INVALID_ARG;
        grad_pre = act.grad_pre;
    }
    if ((gw && !row_tensor(x, Kd, &r, &xd)) || (gx && !row_tensor(gx, Kd, &r, &gxd, true))) return EP_ERR_INVALID_ARG;
    if (handle) handle_used(handle, (hipStream_t)stream);
    if (elementwise) {
        act.win = r.win; act.N = (int)N; act.No = (int)No; act.act = cfg->activation; act.gated = cfg->gated;
        if (launch_act_backward(act, (hipStream_t)stream) != hipSuccess) return EP_ERR_HIP;
    }
    if (gx) {
        rows.win = r.win; rows.grad_pre = grad_pre; rows.grad_x = gxd;
        rows.w = (const uint16_t*)w->data; rows.w_expert = w->stride[0]; rows.w_row = w->stride[1];
        rows.N = (int)N; rows.Kd = (int)Kd;
    }
    if (gw) {
        weights.win = r.win; weights.grad_pre = grad_pre; weights.x = xd;
        weights.grad_w = gw->data; weights.gw_expert = gw->stride[0]; weights.gw_row = gw->stride[1];
        weights.gw_f32 = gw->dtype == EP_DTYPE_F32;
        weights.grad_b = gb ? gb->data : nullptr; weights.gb_stride = gb ? gb->stride[0] : 0;
        weights.N = (int)N; weights.Kd = (int)Kd; weights.accumulate = cfg->accumulate;
    }
    return gx || gw ? done(launch_gradients(gx ? &rows : nullptr, gw ? &weights : nullptr, (hipStream_t)stream)) : EP_SUCCESS;
}

ep_result_t ep_expert_layer_plan(int64_t num_tokens, int32_t top_k, int32_t num_experts, int32_t hidden, int32_t inner,
                                 ep_expert_layer_plan_t* plan) {
    if (!plan || num_tokens < 0 || num_tokens > kLayerMaxTokens || top_k < 1 || top_k > kMaxTopK || num_experts < 1 ||
        num_experts > kMaxExperts || hidden < 8 || hidden % 8 || hidden > kMaxLayerExtent || inner < 8 || inner % 8 ||
        inner > kMaxLayerExtent)
        return EP_ERR_INVALID_ARG;
    if (num_tokens * top_k * inner >= kMaxLayerRows) return EP_ERR_UNSUPPORTED;
    LayerPlan p;
    plan_layer((int)num_tokens, top_k, num_experts, hidden, inner, &p);
    plan->workspace_bytes = p.total;
    plan->slots = p.slots;
    plan->reserved = 0;
    return EP_SUCCESS;
}

ep_result_t ep_expert_layer(const ep_product_config_t* cfg, const ep_tensor_t* inputs, int32_t num_inputs, const ep_tensor_t* outputs,
                            int32_t num_outputs, ep_stream_t stream) {
    if (!inputs || !outputs || num_inputs < 1 || num_outputs < 1) return EP_ERR_INVALID_ARG;
    if (ep_result_t r = check_product_config(cfg); r != EP_SUCCESS) return r;
    const ep_tensor_t* x = find_tag(inputs, num_inputs, EP_TAG_TOKENS);
    const ep_tensor_t* idx = find_tag(inputs, num_inputs, EP_TAG_TOPK_IDX);
    const ep_tensor_t* w = find_tag(inputs, num_inputs, EP_TAG_TOPK_WEIGHTS);
    const ep_tensor_t* up = find_tag(inputs, num_inputs, EP_TAG_EXPERT_WEIGHTS);
    const ep_tensor_t* down = find_tag(inputs, num_inputs, EP_TAG_DOWN_WEIGHTS);
    const ep_tensor_t* bu = find_tag(inputs, num_inputs, EP_TAG_EXPERT_BIAS);
    const ep_tensor_t* bd = find_tag(inputs, num_inputs, EP_TAG_DOWN_BIAS);
    const ep_tensor_t* res = find_tag(inputs, num_inputs, EP_TAG_RESIDUAL);
    const ep_tensor_t* out = find_tag(outputs, num_outputs, EP_TAG_TOKENS);
    const ep_tensor_t* ws = find_tag(outputs, num_outputs, EP_TAG_WORKSPACE);
    if (cfg->accumulate || !check_weights(up) || !check_weights(down) || !x || x->ndim != 2 || !idx || idx->ndim != 2) return EP_ERR_INVALID_ARG;
    const int64_t T = x->shape[0], K = idx->shape[1], L = up->shape[0], H = up->shape[2], N = up->shape[1], I = cfg->gated ? N / 2 : N;
    if (T > kLayerMaxTokens) return EP_ERR_UNSUPPORTED;
    if (T < 0 || K < 1 || K > kMaxTopK || I % 8 || H > kMaxLayerExtent || I > kMaxLayerExtent) return EP_ERR_INVALID_ARG;
    if (T * K * I >= kMaxLayerRows) return EP_ERR_UNSUPPORTED;
    if (down->shape[0] != L || down->shape[1] != H || down->shape[2] != I) return EP_ERR_INVALID_ARG;
    auto token_rows = [&](const ep_tensor_t* t) {
        return check_2d(t, EP_DTYPE_BF16, T, H, true) && t->stride[0] % 8 == 0 && t->stride[0] < kMaxExtent && aligned16(t->data);
    };
    if (!token_rows(x) || !token_rows(out) || (res && !token_rows(res))) return EP_ERR_INVALID_ARG;
    if (!check_2d(idx, EP_DTYPE_I32, T, K, true) || (w && !check_2d(w, EP_DTYPE_F32, T, K, true))) return EP_ERR_INVALID_ARG;
    if ((bu && !check_bias(bu, L, N)) || (bd && !check_bias(bd, L, H))) return EP_ERR_INVALID_ARG;
    LayerPlan plan;
    plan_layer((int)T, (int)K, (int)L, (int)H, (int)I, &plan);
    if (T > 0 && (!check_1d(ws, EP_DTYPE_U8, plan.total) || !aligned16(ws->data))) return EP_ERR_INVALID_ARG;
    LayerArgs a = {};
    a.x = (const uint16_t*)x->data; a.x_stride = x->stride[0];
    a.topk_idx = (const int32_t*)idx->data; a.idx_stride = idx->stride[0];
    a.topk_w = w ? (const float*)w->data : nullptr; a.w_stride = w ? w->stride[0] : 0;
    a.w_up = (const uint16_t*)up->data; a.up_expert = up->stride[0]; a.up_row = up->stride[1];
    a.w_down = (const uint16_t*)down->data; a.down_expert = down->stride[0]; a.down_row = down->stride[1];
    a.b_up = bu ? bu->data : nullptr; a.b_up_stride = bu ? bu->stride[0] : 0; a.b_up_f32 = bu && bu->dtype == EP_DTYPE_F32;
    a.b_down = bd ? bd->data : nullptr; a.b_down_stride = bd ? bd->stride[0] : 0; a.b_down_f32 = bd && bd->dtype == EP_DTYPE_F32;
    a.res = res ? (const uint16_t*)res->data : nullptr; a.res_stride = res ? res->stride[0] : 0;
    a.out = (uint16_t*)out->data; a.out_stride = out->stride[0];
    a.workspace = ws ? (uint8_t*)ws->data : nullptr;
    a.T = (int)T; a.K = (int)K; a.L = (int)L; a.H = (int)H; a.inner = (int)I; a.first = cfg->first_expert;
    a.act = cfg->activation; a.gated = cfg->gated;
    return done(launch_layer(a, (hipStream_t)stream));
}

}  // extern "C"
