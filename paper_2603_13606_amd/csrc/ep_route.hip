// The gate: logits to the top-k experts of a token and their gate weights, forward and backward.
//
//   s = softmax(l) over the routable experts, or sigmoid(l);  the K largest s + bias, descending, ties to the
//   lowest id;  w_k = scale * s[idx_k] / (sum over the selected, if renormalised)
//
// One wavefront per token; lane l holds the experts l, l + 64, ...  Softmax and sigmoid grow with the logit, so
// without a bias and without groups the order of the scores is that of the logits, which is exact: the key of an
// expert is its logit as an ordered integer.  With a bias or groups the key is a sum of computed numbers; it is
// taken in 64 bits, so that two experts change places only where their scores agree to 1e-16.  The K rounds of the
// selection each take the wave's maximum of the lanes' best keys (six DPP steps in registers, no LDS), then the
// lowest id that has it.  Memory is read once; below some thousand tokens a launch is latency.
// Measured in a graph, 256 experts, top-8: 128 tokens 4.1 us, 4096 tokens 6.0, with a bias 10.0, with bias and groups 12.3 (the
// exponentials in 64 bits 1.3 of it).
#include <algorithm>

#include "ep_experts.h"
#include "ep_internal.h"

namespace ep {

namespace {

constexpr int kRouteWaves = 4;       // wavefronts (tokens) per workgroup
constexpr int kRouteMaxGrid = 16384;  // workgroups; further tokens go round

template <class F>
__device__ __forceinline__ uint32_t wave_reduce(uint32_t v, uint32_t none, F f) {
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp((int)none, (int)v, 0x111, 0xf, 0xf, false));  // row_shr:1
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp((int)none, (int)v, 0x112, 0xf, 0xf, false));
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp((int)none, (int)v, 0x114, 0xf, 0xf, false));
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp((int)none, (int)v, 0x118, 0xf, 0xf, false));
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp((int)none, (int)v, 0x142, 0xf, 0xf, false));  // last lane of each row to the next
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp((int)none, (int)v, 0x143, 0xf, 0xf, false));  // lane 31 to the upper half
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}

__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
    return wave_reduce(v, 0u, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}
__device__ __forceinline__ uint32_t wave_min(uint32_t v) {
    return wave_reduce(v, 0xffffffffu, [](uint32_t a, uint32_t b) { return a < b ? a : b; });
}
__device__ __forceinline__ float wave_sum(float v) {
    return __uint_as_float(wave_reduce(__float_as_uint(v), 0u, [](uint32_t a, uint32_t b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }));
}
__device__ __forceinline__ double wave_sum64(double v) {
    for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
    return v;
}

// Integers in the order of the numbers; never 0 for a finite number, so 0 is "none".
__device__ __forceinline__ uint32_t ordered(float v) {
    const uint32_t u = __float_as_uint(v);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t u) { return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u); }
__device__ __forceinline__ uint64_t ordered64(double v) {
    const uint64_t u = (uint64_t)__double_as_longlong(v);
    return u >> 63 ? ~u : u | 0x8000000000000000ull;
}

// A logit as the gate takes it: NaN and -inf mean "not routable" (returned as -inf), +inf the largest finite
// number, and both zeros are the same zero.
__device__ __forceinline__ float load_logit(const void* p, int64_t i, int is_bf16) {
    float v = is_bf16 ? bf16_f32(((const uint16_t*)p)[i]) : ((const float*)p)[i];
    if (!(v > -__builtin_inff())) return -__builtin_inff();
    return fminf(v, 3.402823466e38f) + 0.0f;
}

__device__ __forceinline__ float sigmoid_exact(float l) { return 1.0f / (1.0f + expf(-l)); }

// Renormalised sigmoid scores relative to e^top, `top` the largest selected logit: for tokens whose scores add up to less than
// kFaint, where single ones are lost below the range of float32 (logits under -87), or all of them.  Of at most 64 scores with a
// larger sum the largest is 2^-16 or more, and what is lost beside it is less than 2^-110 of it.  As in 64 bits, a score below
// 2^-1022 (a logit under -708.39) is 0.
constexpr float kFaint = 0x1p-10f, kNoScore = -708.39f;
static_assert(kMaxTopK <= 64, "scores that add up to kFaint");
__device__ __forceinline__ float faint_score(float l, float top) { return l < kNoScore ? 0.0f : expf(l - top) / (1.0f + expf(l)); }

// SCORES: selection by scores in 64 bits (bias or groups); otherwise by logits.
template <int NPL, bool SCORES>
__global__ __launch_bounds__(64 * kRouteWaves) void route_kernel(const RouteArgs a) {
    __shared__ double group_keys[SCORES ? kRouteWaves * 64 * NPL : 1];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int64_t t = (int64_t)blockIdx.x * kRouteWaves + wave; t < a.T; t += (int64_t)gridDim.x * kRouteWaves) {
        float l[NPL];
#pragma unroll
        for (int i = 0; i < NPL; ++i) {
            const int e = lane + 64 * i;
            l[i] = e < a.E ? load_logit(a.logits, t * a.logits_stride + e, a.logits_bf16) : -__builtin_inff();
        }
        float top = 0.0f;   // the largest logit, where the softmax over all experts is wanted
        if (a.score == EP_SCORE_SOFTMAX && (SCORES || !a.renormalise)) {
            top = l[0];
#pragma unroll
            for (int i = 1; i < NPL; ++i) top = fmaxf(top, l[i]);
            top = unordered(wave_max(top > -__builtin_inff() ? ordered(top) : 0u));
        }
        uint32_t hi[NPL], lo[SCORES ? NPL : 1];
        if constexpr (!SCORES) {
#pragma unroll
            for (int i = 0; i < NPL; ++i) hi[i] = l[i] > -__builtin_inff() ? ordered(l[i]) : 0u;
        } else {
            double s[NPL];
            double sum = 0.0;
#pragma unroll
            for (int i = 0; i < NPL; ++i) {
                const bool there = l[i] > -__builtin_inff();
                if (a.score == EP_SCORE_SIGMOID) {
                    s[i] = there ? 1.0 / (1.0 + exp(-(double)l[i])) : 0.0;
                } else {
                    s[i] = there ? exp((double)l[i] - (double)top) : 0.0;
                    sum += s[i];
                }
            }
            if (a.score != EP_SCORE_SIGMOID) {
                sum = wave_sum64(sum);
#pragma unroll
                for (int i = 0; i < NPL; ++i) s[i] = sum > 0.0 ? s[i] / sum : 0.0;
            }
#pragma unroll
            for (int i = 0; i < NPL; ++i) {
                const int e = lane + 64 * i;
                const float b = a.bias && e < a.E ? a.bias[e] : 0.0f;
                double key = l[i] > -__builtin_inff() ? s[i] + (double)b : -__builtin_inf();
                if (!(key > -__builtin_inf())) key = -__builtin_inf();  // a bias of NaN or -inf takes the expert out
                s[i] = key + 0.0;
            }
            if (a.groups > 1) {
                double* keys = group_keys + wave * 64 * NPL;
#pragma unroll
                for (int i = 0; i < NPL; ++i) keys[lane + 64 * i] = s[i];
                __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
                __builtin_amdgcn_wave_barrier();
                // `sub` lanes per group find its two largest keys; lane g then holds the worth of group g
                const int size = a.E / a.groups;
                int sub = 1;
                while (sub * 2 * a.groups <= 64) sub *= 2;
                const int g = lane / sub;
                double first = -__builtin_inf(), second = -__builtin_inf();
                if (g < a.groups)
                    for (int m = lane % sub; m < size; m += sub) {
                        const double v = keys[g * size + m];
                        if (v > first) { second = first; first = v; }
                        else if (v > second) second = v;
                    }
                for (int d = 1; d < sub; d <<= 1) {
                    const double f = __shfl_xor(first, d), n = __shfl_xor(second, d);
                    if (f > first) { second = fmax(first, n); first = f; }
                    else second = fmax(second, f);
                }
                double worth = first + (second > -__builtin_inf() ? second : 0.0);
                worth = __shfl(worth, min(lane, a.groups - 1) * sub);
                int rank = 0;
                for (int j = 0; j < a.groups; ++j) {
                    const uint64_t u = (uint64_t)__double_as_longlong(worth);
                    const double w = __longlong_as_double((long long)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(u >> 32), j) << 32 |
                                                                      (uint32_t)__builtin_amdgcn_readlane((int)u, j)));
                    rank += w > worth || (w == worth && j < lane);
                }
                const uint64_t kept = __ballot(lane < a.groups && rank < a.kept);
#pragma unroll
                for (int i = 0; i < NPL; ++i) {
                    const int e = lane + 64 * i;
                    if (e < a.E && !(kept >> (e / size) & 1)) s[i] = -__builtin_inf();
                }
                __builtin_amdgcn_wave_barrier();  // the next token's keys come behind these reads
            }
#pragma unroll
            for (int i = 0; i < NPL; ++i) {
                const uint64_t u = s[i] > -__builtin_inf() ? ordered64(s[i]) : 0ull;
                hi[i] = (uint32_t)(u >> 32);
                lo[i] = (uint32_t)u;
            }
        }

        // Up to four experts per lane are put in order once (neighbours change places, so equal ones stay as they are), and
        // the lane's best is the first; more are searched in every round.
        constexpr bool SORTED = NPL <= 4;
        int at[NPL];   // place j: expert lane + 64 * at[j]
#pragma unroll
        for (int i = 0; i < NPL; ++i) at[i] = i;
        if constexpr (SORTED) {
#pragma unroll
            for (int n = NPL - 1; n > 0; --n)
#pragma unroll
                for (int i = 0; i < n; ++i) {
                    const bool swap = SCORES ? hi[i + 1] > hi[i] || (hi[i + 1] == hi[i] && lo[i + 1] > lo[i]) : hi[i + 1] > hi[i];
                    auto exchange = [swap](auto& x, auto& y) {
                        const auto z = x;
                        x = swap ? y : x;
                        y = swap ? z : y;
                    };
                    exchange(hi[i], hi[i + 1]);
                    if (SCORES) exchange(lo[i], lo[i + 1]);
                    exchange(at[i], at[i + 1]);
                }
        }
        int my_idx = -1;        // lane k: the k-th expert
        float my_l = -__builtin_inff();
        for (int k = 0; k < a.K; ++k) {
            uint32_t bh = hi[0], bl = SCORES ? lo[0] : 0u;
            int bi = at[0];
            if constexpr (!SORTED) {
#pragma unroll
                for (int i = 1; i < NPL; ++i)
                    if (SCORES ? hi[i] > bh || (hi[i] == bh && lo[i] > bl) : hi[i] > bh) {
                        bh = hi[i];
                        if (SCORES) bl = lo[i];
                        bi = i;
                    }
            }
            const uint32_t mh = wave_max(bh);
            if (mh == 0) break;  // nothing routable is left
            bool mine = bh == mh;
            uint64_t who = __ballot(mine);
            if (who & (who - 1)) {  // a tie between lanes: the larger low word, then the lowest id
                if (SCORES) {
                    const uint32_t ml = wave_max(mine ? bl : 0u);
                    mine = mine && bl == ml;
                }
                const uint32_t e = wave_min(mine ? lane + 64 * bi : 0xffffffffu);
                mine = mine && lane + 64 * bi == (int)e;
                who = __ballot(mine);
            }
            const int from = __builtin_ctzll(who);
            const int i = __builtin_amdgcn_readlane(bi, from);
            float logit;
            if constexpr (SCORES) {
                logit = l[0];
#pragma unroll
                for (int j = 1; j < NPL; ++j) logit = i == j ? l[j] : logit;
                logit = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(logit), from));
            } else {
                logit = unordered(mh);
            }
            if (lane == k) { my_idx = from + 64 * i; my_l = logit; }
            if constexpr (SORTED) {
#pragma unroll
                for (int j = 0; j < NPL; ++j) {
                    hi[j] = mine ? (j + 1 < NPL ? hi[(j + 1) % NPL] : 0u) : hi[j];
                    if (SCORES) lo[j] = mine ? (j + 1 < NPL ? lo[(j + 1) % NPL] : 0u) : lo[j];
                    at[j] = mine && j + 1 < NPL ? at[(j + 1) % NPL] : at[j];
                }
            } else {
#pragma unroll
                for (int j = 0; j < NPL; ++j)
                    if (mine && i == j) {
                        hi[j] = 0;
                        if (SCORES) lo[j] = 0;
                    }
            }
        }

        float w;
        if (a.score == EP_SCORE_SIGMOID) {
            w = my_idx >= 0 ? sigmoid_exact(my_l) : 0.0f;
        } else {
            // renormalised: only the selected count, taken relative to their largest
            float m = top;
            if (a.renormalise) m = unordered(wave_max(my_idx >= 0 ? ordered(my_l) : 0u));
            w = my_idx >= 0 ? expf(my_l - m) : 0.0f;
            if (!a.renormalise) {
                float sum = 0.0f;
#pragma unroll
                for (int i = 0; i < NPL; ++i) sum += l[i] > -__builtin_inff() ? expf(l[i] - top) : 0.0f;
                sum = wave_sum(sum);
                w = my_idx >= 0 ? w / sum : 0.0f;
            }
        }
        if (a.renormalise) {
            float sum = wave_sum(w);
            if (a.score == EP_SCORE_SIGMOID && sum < kFaint) {
                const float most = unordered(wave_max(my_idx >= 0 ? ordered(my_l) : 0u));
                w = my_idx >= 0 ? faint_score(my_l, most) : 0.0f;
                sum = wave_sum(w);
            }
            w = sum > 0.0f ? w / sum : 0.0f;
        }
        if (lane < a.K) {
            a.topk_idx[t * a.idx_stride + lane] = my_idx;
            a.topk_w[t * a.w_stride + lane] = w * a.scale;
        }
    }
}

template <int NPL>
__global__ __launch_bounds__(64 * kRouteWaves) void route_backward_kernel(const RouteBackwardArgs a) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int64_t t = (int64_t)blockIdx.x * kRouteWaves + wave; t < a.T; t += (int64_t)gridDim.x * kRouteWaves) {
        // lane k: entry k
        int e = lane < a.K ? a.topk_idx[t * a.idx_stride + lane] : -1;
        if (e < 0 || e >= a.E) e = -1;
        const float g = e >= 0 ? a.grad_w[t * a.gw_stride + lane] * a.scale : 0.0f;
        const float le = e >= 0 ? load_logit(a.logits, t * a.logits_stride + e, a.logits_bf16) : -__builtin_inff();
        const bool there = le > -__builtin_inff();
        float p[NPL];  // scores of the lane's experts, where every expert has a gradient
        float s, d;    // entry k: its score, and the gradient of the score
        const bool dense = a.score == EP_SCORE_SOFTMAX && !a.renormalise;
        float dot = 0.0f;
        if (dense) {
            float top = -__builtin_inff(), sum = 0.0f;
#pragma unroll
            for (int i = 0; i < NPL; ++i) {
                const int c = lane + 64 * i;
                p[i] = c < a.E ? load_logit(a.logits, t * a.logits_stride + c, a.logits_bf16) : -__builtin_inff();
                top = fmaxf(top, p[i]);
            }
            top = unordered(wave_max(top > -__builtin_inff() ? ordered(top) : 0u));
#pragma unroll
            for (int i = 0; i < NPL; ++i) {
                p[i] = p[i] > -__builtin_inff() ? expf(p[i] - top) : 0.0f;
                sum += p[i];
            }
            sum = wave_sum(sum);
            const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
#pragma unroll
            for (int i = 0; i < NPL; ++i) p[i] *= inv;
            s = there ? expf(le - top) * inv : 0.0f;
            dot = wave_sum(there ? g * s : 0.0f);  // dl_e = p_e (sum of g over the entries of e - dot)
            d = there ? g : 0.0f;
        } else if (a.score == EP_SCORE_SOFTMAX) {
            const float m = unordered(wave_max(there ? ordered(le) : 0u));
            s = there ? expf(le - m) : 0.0f;
            const float sum = wave_sum(s);
            s = sum > 0.0f ? s / sum : 0.0f;
            const float mean = wave_sum(there ? g * s : 0.0f);
            d = there ? s * (g - mean) : 0.0f;      // gradient of the logit
        } else {
            s = there ? sigmoid_exact(le) : 0.0f;
            const float rest = there ? 1.0f / (1.0f + expf(le)) : 0.0f;  // 1 - s without cancellation
            d = there ? g * s * rest : 0.0f;
            if (a.renormalise) {
                // From the weights, as above: the scores may be so small that the gradient of a weight over their sum overflows, where
                // that of the logit does not.  Of one entry, whose weight is 1 whatever its logit, exactly nothing is left.
                float q = s, sum = wave_sum(s);
                if (sum < kFaint) {
                    const float most = unordered(wave_max(there ? ordered(le) : 0u));
                    q = there ? faint_score(le, most) : 0.0f;
                    sum = wave_sum(q);
                }
                q = sum > 0.0f ? q / sum : 0.0f;
                const float mean = wave_sum(there ? g * q : 0.0f);
                d = there ? (g - mean) * q * rest : 0.0f;
            }
        }
        float out[NPL];
#pragma unroll
        for (int i = 0; i < NPL; ++i) out[i] = dense ? -dot : 0.0f;
        for (int k = 0; k < a.K; ++k) {
            const int ek = __builtin_amdgcn_readlane(e, k);
            const float dk = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(d), k));
            if (ek < 0) continue;
#pragma unroll
            for (int i = 0; i < NPL; ++i)
                if (ek == lane + 64 * i) out[i] += dk;
        }
#pragma unroll
        for (int i = 0; i < NPL; ++i) {
            const int c = lane + 64 * i;
            if (c >= a.E) continue;
            const float v = dense ? out[i] * p[i] : out[i];
            const int64_t at = t * a.gl_stride + c;
            if (a.logits_bf16) ((uint16_t*)a.grad_logits)[at] = (uint16_t)pack2_bf16(v, 0.0f);
            else ((float*)a.grad_logits)[at] = v;
        }
    }
}

template <class F>
void by_lanes(int E, F f) {  // experts per lane
    const int n = (E + 63) / 64;
    if (n <= 1) f(std::integral_constant<int, 1>());
    else if (n <= 2) f(std::integral_constant<int, 2>());
    else if (n <= 4) f(std::integral_constant<int, 4>());
    else if (n <= 8) f(std::integral_constant<int, 8>());
    else f(std::integral_constant<int, 16>());
}

dim3 route_grid(int T) { return dim3((uint32_t)std::min((T + kRouteWaves - 1) / kRouteWaves, kRouteMaxGrid)); }

}  // namespace

hipError_t launch_route(const RouteArgs& a, hipStream_t s) {
    if (a.T == 0) return hipSuccess;
    by_lanes(a.E, [&](auto n) {
        if (a.bias || a.groups > 1) hipLaunchKernelGGL((route_kernel<n.value, true>), route_grid(a.T), dim3(64 * kRouteWaves), 0, s, a);
        else hipLaunchKernelGGL((route_kernel<n.value, false>), route_grid(a.T), dim3(64 * kRouteWaves), 0, s, a);
    });
    return hipGetLastError();
}

hipError_t launch_route_backward(const RouteBackwardArgs& a, hipStream_t s) {
    if (a.T == 0) return hipSuccess;
    by_lanes(a.E, [&](auto n) {
        hipLaunchKernelGGL((route_backward_kernel<n.value>), route_grid(a.T), dim3(64 * kRouteWaves), 0, s, a);
    });
    return hipGetLastError();
}

}  // namespace ep
