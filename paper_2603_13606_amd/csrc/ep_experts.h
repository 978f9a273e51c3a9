// The gate, the experts' products and the layer of few tokens: argument structs, launch functions
// and the device helpers that their kernels share.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ep.h"

namespace ep {

// ---- gate ---------------------------------------------------------------------------------

struct RouteArgs {
    const void* logits;     // [T, E] f32 or bf16
    int64_t logits_stride;
    int logits_bf16;
    const float* bias;      // [E] or nullptr: added to the scores for the selection only
    int32_t* topk_idx;      // [T, K]
    int64_t idx_stride;
    float* topk_w;          // [T, K]
    int64_t w_stride;
    int T, E, K;
    int score, renormalise, groups, kept;
    float scale;
};

struct RouteBackwardArgs {
    const void* logits;     // [T, E]
    int64_t logits_stride;
    int logits_bf16;        // of logits and grad_logits
    const int32_t* topk_idx;
    int64_t idx_stride;
    const float* grad_w;    // [T, K]
    int64_t gw_stride;
    void* grad_logits;      // [T, E]
    int64_t gl_stride;
    int T, E, K;
    int score, renormalise;
    float scale;
};

hipError_t launch_route(const RouteArgs& a, hipStream_t s);
hipError_t launch_route_backward(const RouteBackwardArgs& a, hipStream_t s);

// ---- experts' products ----------------------------------------------------------------------

// A matrix of token rows in expert windows: row r of expert e at base + e * expert_stride + (first + r) * row_stride
// elements, first = offset[e] for concatenated windows (expert_stride 0) and 0 for padded ones.
struct RowsDesc {
    uint16_t* base;
    int64_t expert_stride, row_stride;
};

struct Windows {
    const int32_t* offset;  // [L] first row of each expert, nullptr for padded windows
    const int32_t* count;   // [L] rows of each expert
    int64_t cap;            // concatenated: rows of the shortest tensor; padded: rows per expert
    int L;
};

struct ProductArgs {
    Windows win;
    RowsDesc x, out, pre, res;   // pre.base, res.base may be nullptr
    const uint16_t* w;           // [L, N, Kd]
    int64_t w_expert, w_row;
    const void* bias;            // [L, N] or nullptr
    int64_t bias_stride;
    int bias_f32;
    int N, No, Kd;               // N = No, or 2 * No when gated
    int act, gated;
    int32_t* status;             // status word of a handle, or nullptr
};

// Gradient of the pre-activation from that of the output (elementwise).
struct ActBackwardArgs {
    Windows win;
    RowsDesc grad_out, pre, grad_pre;
    int N, No, act, gated;
};

// grad_x = grad_pre W
struct GradRowsArgs {
    Windows win;
    RowsDesc grad_pre, grad_x;
    const uint16_t* w;
    int64_t w_expert, w_row;
    int N, Kd;
};

// grad_w (+)= grad_pre^T x, grad_b (+)= column sums of grad_pre
struct GradWeightsArgs {
    Windows win;
    RowsDesc grad_pre, x;
    void* grad_w;                // [L, N, Kd] f32 or bf16
    int64_t gw_expert, gw_row;
    int gw_f32;
    void* grad_b;                // [L, N] or nullptr, of the same type
    int64_t gb_stride;
    int N, Kd, accumulate;
};

hipError_t launch_product(const ProductArgs& a, hipStream_t s);
hipError_t launch_act_backward(const ActBackwardArgs& a, hipStream_t s);
// Either may be nullptr; both have the same windows and grad_pre.
hipError_t launch_gradients(const GradRowsArgs* rows, const GradWeightsArgs* weights, hipStream_t s);

// ---- the layer of few tokens ------------------------------------------------------------------

constexpr int kLayerMaxTokens = 128;

struct LayerArgs {
    const uint16_t* x;
    int64_t x_stride;
    const int32_t* topk_idx;
    int64_t idx_stride;
    const float* topk_w;         // or nullptr: unit weights
    int64_t w_stride;
    const uint16_t *w_up, *w_down;  // [L, N, H], [L, H, inner]
    int64_t up_expert, up_row, down_expert, down_row;
    const void *b_up, *b_down;   // [L, N], [L, H] or nullptr
    int64_t b_up_stride, b_down_stride;
    int b_up_f32, b_down_f32;
    const uint16_t* res;         // [T, H] or nullptr
    int64_t res_stride;
    uint16_t* out;
    int64_t out_stride;
    uint8_t* workspace;
    int T, K, L, H, inner, first, act, gated;
};

// Where the parts of the layer's workspace lie (bytes from its start).
struct LayerPlan {
    int64_t mid, total;          // the sorted entries come first, then the rows between the products
    int slots;                   // experts that can be named: min(L, T * K)
    int up_parts;                // shares of a named expert's rows in the first launch, a workgroup each
    int token_parts;             // shares of its tokens, too
    int token_step;              // tokens per pass over the weights
};
void plan_layer(int T, int K, int L, int H, int inner, LayerPlan* p);
hipError_t launch_layer(const LayerArgs& a, hipStream_t s);

// Compute units of the current device, asked once per device.
int compute_units();

// ---- device helpers ----------------------------------------------------------------------------

__device__ __forceinline__ float bf16_f32(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));

// Two float32 -> two bfloat16, low and high half: round to nearest even.
__device__ __forceinline__ uint32_t pack2_bf16(float lo, float hi) {
    const f32x2_t v = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2_t));
}

// Activations in float32.  The exponential is the part's own: its argument is rounded, which makes a relative error of up to 1e-5
// where the result is smallest, far below the rounding of the result to bf16 (2e-3 to 4e-3 of it).
__device__ __forceinline__ float sigmoid_f32(float v) { return __builtin_amdgcn_rcpf(1.0f + __expf(-v)); }

// (1 + erf(v / sqrt 2)) / 2 without a branch, from e^(v^2 / 2) erfc(|v| / sqrt 2): a polynomial in t = 1 / (1 + 0.37 |v| / sqrt 2) whose
// coefficients make its largest RELATIVE error over |v| <= 13.3 smallest (a linear programme, with the value 1 at v = 0): 7e-7.
// gelu(v) is proportional to it for negative v, so an error relative to erf would show there: 1.5e-7 of erf is 0.4 % of gelu(-6).
__device__ __forceinline__ float normal_cdf(float v) {
    const float t = __builtin_amdgcn_rcpf(fmaf(0.26162951f, fabsf(v), 1.0f));
    float p = fmaf(-0.1428908550f, t, 0.4367967860f);
    p = fmaf(p, t, -0.1879631269f);
    p = fmaf(p, t, 0.3184649016f);
    p = fmaf(p, t, 0.1522594205f);
    p = fmaf(p, t, 0.2149588644f);
    p = fmaf(p, t, 0.2083740092f) * t;
    const float tail = 0.5f * p * __expf(-0.5f * v * v);
    return v < 0.0f ? tail : 1.0f - tail;
}

__device__ __forceinline__ float activate(int act, float v) {
    if (act == EP_ACT_SILU) return v * sigmoid_f32(v);
    if (act == EP_ACT_GELU) return v * normal_cdf(v);
    return v;
}

// Value and derivative of the activation.
__device__ __forceinline__ float activate_grad(int act, float v, float* value) {
    if (act == EP_ACT_SILU) {
        const float s = sigmoid_f32(v);
        *value = v * s;
        return s * (1.0f + v * (1.0f - s));
    }
    if (act == EP_ACT_GELU) {
        const float p = normal_cdf(v);
        *value = v * p;
        return p + v * (0.39894228040143268f * __expf(-0.5f * v * v));
    }
    *value = v;
    return 1.0f;
}

}  // namespace ep
