// The whole expert layer for a few tokens, without windows, in two launches.
//
//   out[t] = res[t] + sum_k w[t,k] (W2_e act(W1_e x[t] + b1_e) + b2_e),  e = topk_idx[t,k], local experts only
//
// What bounds it is reading the weights of the experts that are named, once.  Both kernels therefore stream
// weight rows from memory into registers as the left operand of MFMA 16x16x32, 16 rows at a time, the tokens
// that name the expert (up to 16 per instruction) being the right operand:
//   up    a workgroup per (named expert, 16 rows of the inner dimension): the contraction over H is split over
//         its wavefronts and joined through LDS in wave order; bias, activation and gate weight are applied in
//         float32, and one row per (token, expert) goes to the workspace in bf16.
//   down  a workgroup per 16 columns of the output: its wavefronts share out the (expert, part of the inner
//         dimension) pairs evenly, each adds up its own part of the output for all tokens in LDS, and the
//         parts are joined in wave order.  No atomics: results do not depend on timing.
// An expert works on its own tokens only, so what its weights hold (an infinity, a NaN) reaches no others.
#include <algorithm>

#include "ep_experts.h"
#include "ep_internal.h"

namespace ep {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kUpWaves = 4, kDownWaves = 8;
constexpr int kRows = 16;     // weight rows per workgroup
constexpr int kBlock = 64;    // contraction indices per step of a wavefront: whole 128-byte lines of 16 rows

// members of slot s: {expert, n, then n pairs {token, row of the workspace}}; one slot per named expert
__host__ __device__ constexpr int member_words(int T) { return 2 + 2 * T; }

__device__ __forceinline__ float load_bias(const void* b, int64_t i, int is_f32) {
    return is_f32 ? ((const float*)b)[i] : bf16_f32(((const uint16_t*)b)[i]);
}

// The id that entry (t, k) names among the local experts, or -1.
__device__ __forceinline__ int local_id(const LayerArgs& a, int t, int k) {
    const int64_t e = (int64_t)a.topk_idx[t * a.idx_stride + k] - a.first;
    return e >= 0 && e < a.L ? (int)e : -1;
}

__device__ __forceinline__ bf16x8 load8(const uint16_t* p, bool there) {
    u32x4 v = {0, 0, 0, 0};
    if (there) v = *(const u32x4*)p;
    return __builtin_bit_cast(bf16x8, v);
}

// acc[g][jt] += 16 weight rows (of each of G matrices) x the tokens of JT groups of 16, over the blocks
// [b0, b1) with the given stride of the contraction.
template <int G, int JT>
__device__ __forceinline__ void multiply(f32x4 (&acc)[G][8], const uint16_t* const (&w)[G], const uint16_t* const (&x)[8],
                                         const bool (&there)[8], int b0, int b1, int stride, int K, int lane) {
    for (int b = b0; b < b1; b += stride) {
        bf16x8 wf[G][2], xf[JT][2];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int k = b * kBlock + s * 32 + (lane >> 4) * 8;
            const bool in = k < K;
#pragma unroll
            for (int g = 0; g < G; ++g) wf[g][s] = load8(w[g] + k, in);
#pragma unroll
            for (int jt = 0; jt < JT; ++jt) xf[jt][s] = load8(x[jt] + k, in && there[jt]);
        }
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
                for (int jt = 0; jt < JT; ++jt)
                    acc[g][jt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[g][s], xf[jt][s], acc[g][jt], 0, 0, 0);
    }
}

template <int G>
__device__ __forceinline__ void multiply_groups(int n, f32x4 (&acc)[G][8], const uint16_t* const (&w)[G], const uint16_t* const (&x)[8],
                                                const bool (&there)[8], int b0, int b1, int stride, int K, int lane) {
    if (n <= 16) multiply<G, 1>(acc, w, x, there, b0, b1, stride, K, lane);
    else if (n <= 32) multiply<G, 2>(acc, w, x, there, b0, b1, stride, K, lane);
    else if (n <= 64) multiply<G, 4>(acc, w, x, there, b0, b1, stride, K, lane);
    else multiply<G, 8>(acc, w, x, there, b0, b1, stride, K, lane);
}

template <int G>
__global__ __launch_bounds__(64 * kUpWaves) void layer_up_kernel(const LayerArgs a, const LayerPlan plan, int slices) {
    __shared__ uint32_t named[kMaxExperts / 32];
    __shared__ int s_n[2];
    __shared__ int s_token[kLayerMaxTokens], s_row[kLayerMaxTokens];
    __shared__ float s_gate[kLayerMaxTokens];
    __shared__ float part[kUpWaves][G][16 * 16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int slot = blockIdx.x / slices, slice = blockIdx.x % slices;

    // the slot-th of the experts that any token names
    if (threadIdx.x < kMaxExperts / 32) named[threadIdx.x] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < a.T * a.K; i += 64 * kUpWaves) {
        const int e = local_id(a, i / a.K, i % a.K);
        if (e >= 0) atomicOr(&named[e >> 5], 1u << (e & 31));
    }
    __syncthreads();
    const uint32_t word = lane < kMaxExperts / 32 ? named[lane] : 0u;
    int upto = __popc(word);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int v = __shfl_up(upto, d);
        if (lane >= d) upto += v;
    }
    int* members = (int*)(a.workspace + plan.members);
    const int total = __shfl(upto, 63);
    if (blockIdx.x == 0 && threadIdx.x == 0) *(int*)a.workspace = total;
    if (slot >= total) return;
    const uint64_t before = __ballot(upto <= slot);
    const int at = __builtin_popcountll(before);  // the word that holds it: the counts only grow
    uint32_t bits = (uint32_t)__builtin_amdgcn_readlane((int)word, at);
    for (int skip = slot - (__shfl(upto, at) - __popc(bits)); skip > 0; --skip) bits &= bits - 1;
    const int e = __builtin_amdgcn_readfirstlane(at * 32 + __builtin_ctz(bits));

    // the tokens that name it: gate weights of all their entries that do, and the workspace row of the first
    bool has = false;
    float gate = 0.0f;
    int row = 0;
    if ((int)threadIdx.x < a.T) {
        const int t = threadIdx.x;
        for (int k = 0; k < a.K; ++k)
            if (local_id(a, t, k) == e) {
                if (!has) row = t * a.K + k;
                has = true;
                gate += a.topk_w ? a.topk_w[t * a.w_stride + k] : 1.0f;
            }
    }
    const uint64_t who = __ballot(has);
    if (wave < 2 && lane == 0) s_n[wave] = __builtin_popcountll(who);
    __syncthreads();
    const int n = s_n[0] + s_n[1];
    if (has) {
        const int pos = (wave == 1 ? s_n[0] : 0) + __builtin_popcountll(who & ((1ull << lane) - 1));
        s_token[pos] = threadIdx.x;
        s_row[pos] = row;
        s_gate[pos] = gate;
    }
    __syncthreads();
    if (slice == 0) {
        int* m = members + slot * member_words(a.T);
        if (threadIdx.x == 0) { m[0] = e; m[1] = n; }
        if ((int)threadIdx.x < n) { m[2 + 2 * threadIdx.x] = s_token[threadIdx.x]; m[3 + 2 * threadIdx.x] = s_row[threadIdx.x]; }
    }

    const int i0 = slice * kRows;
    const int i = min(i0 + (lane & 15), a.inner - 1);
    const uint16_t* w[G];
#pragma unroll
    for (int g = 0; g < G; ++g) w[g] = a.w_up + e * a.up_expert + (int64_t)(i + g * a.inner) * a.up_row;
    const uint16_t* x[8];
    bool there[8];
#pragma unroll
    for (int jt = 0; jt < 8; ++jt) {
        const int pos = jt * 16 + (lane & 15);
        there[jt] = pos < n;
        x[jt] = a.x + (there[jt] ? s_token[pos] : 0) * a.x_stride;
    }
    f32x4 acc[G][8];
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
        for (int jt = 0; jt < 8; ++jt) acc[g][jt] = f32x4{0, 0, 0, 0};
    multiply_groups<G>(n, acc, w, x, there, wave, (a.H + kBlock - 1) / kBlock, kUpWaves, a.H, lane);

    uint16_t* mid = (uint16_t*)(a.workspace + plan.mid);
#pragma unroll
    for (int jt = 0; jt < 8; ++jt) {
        if (jt * 16 >= n) break;
#pragma unroll
        for (int g = 0; g < G; ++g)
            *(f32x4*)&part[wave][g][(lane & 15) * 16 + (lane >> 4) * 4] = acc[g][jt];
        __syncthreads();
        const int pos = jt * 16 + (threadIdx.x >> 4), ii = i0 + (threadIdx.x & 15);
        if (pos < n && ii < a.inner) {
            float v[G];
#pragma unroll
            for (int g = 0; g < G; ++g) {
                v[g] = a.b_up ? load_bias(a.b_up, e * a.b_up_stride + ii + g * a.inner, a.b_up_f32) : 0.0f;
#pragma unroll
                for (int q = 0; q < kUpWaves; ++q) v[g] += part[q][g][threadIdx.x];
            }
            float h = activate(a.act, v[0]);
            if (G == 2) h *= v[G - 1];
            // the gate weight goes in before the rounding to bf16: one rounding of the product of both
            mid[(int64_t)s_row[pos] * a.inner + ii] = (uint16_t)pack2_bf16(h * s_gate[pos], 0.0f);
        }
        __syncthreads();
    }
}

__global__ __launch_bounds__(64 * kDownWaves) void layer_down_kernel(const LayerArgs a, const LayerPlan plan) {
    extern __shared__ __attribute__((aligned(16))) float sums[];  // [waves][T][16]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int h0 = blockIdx.x * kRows;
    const int total = __builtin_amdgcn_readfirstlane(*(const int*)a.workspace);
    const int* members = (const int*)(a.workspace + plan.members);
    const uint16_t* mid = (const uint16_t*)(a.workspace + plan.mid);
    float* mine = sums + wave * a.T * 16;
    for (int i = lane; i < a.T * 16; i += 64) mine[i] = 0.0f;

    const int blocks = (a.inner + kBlock - 1) / kBlock;
    const int64_t items = (int64_t)total * blocks;
    int64_t q = items * wave / kDownWaves;
    const int64_t end = items * (wave + 1) / kDownWaves;
    const int h = min(h0 + (lane & 15), a.H - 1);
    while (q < end) {
        const int slot = (int)(q / blocks), b0 = (int)(q - (int64_t)slot * blocks);
        const int b1 = (int)min((int64_t)blocks, b0 + (end - q));
        const int* m = members + slot * member_words(a.T);
        const int e = __builtin_amdgcn_readfirstlane(m[0]), n = __builtin_amdgcn_readfirstlane(m[1]);
        const uint16_t* w[1] = {a.w_down + e * a.down_expert + (int64_t)h * a.down_row};
        const uint16_t* x[8];
        bool there[8];
        int token[8];
#pragma unroll
        for (int jt = 0; jt < 8; ++jt) {
            const int pos = jt * 16 + (lane & 15);
            there[jt] = pos < n;
            token[jt] = there[jt] ? m[2 + 2 * pos] : 0;
            x[jt] = mid + (int64_t)(there[jt] ? m[3 + 2 * pos] : 0) * a.inner;
        }
        f32x4 acc[1][8];
#pragma unroll
        for (int jt = 0; jt < 8; ++jt) acc[0][jt] = f32x4{0, 0, 0, 0};
        multiply_groups<1>(n, acc, w, x, there, b0, b1, 1, a.inner, lane);
#pragma unroll
        for (int jt = 0; jt < 8; ++jt)
            if (there[jt]) {
                f32x4* to = (f32x4*)(mine + token[jt] * 16 + (lane >> 4) * 4);
                *to = *to + acc[0][jt];
            }
        q += b1 - b0;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < a.T * 16; i += 64 * kDownWaves) {
        const int t = i >> 4, c = h0 + (i & 15);
        if (c >= a.H) continue;
        float v = 0.0f;
        for (int p = 0; p < kDownWaves; ++p) v += sums[p * a.T * 16 + i];
        if (a.b_down)
            for (int k = 0; k < a.K; ++k) {
                const int e = local_id(a, t, k);
                if (e >= 0) v += (a.topk_w ? a.topk_w[t * a.w_stride + k] : 1.0f) * load_bias(a.b_down, e * a.b_down_stride + c, a.b_down_f32);
            }
        if (a.res) v += bf16_f32(a.res[t * a.res_stride + c]);
        a.out[t * a.out_stride + c] = (uint16_t)pack2_bf16(v, 0.0f);
    }
}

int64_t up256(int64_t v) { return (v + 255) / 256 * 256; }

}  // namespace

void plan_layer(int T, int K, int L, int H, int inner, LayerPlan* p) {
    p->slots = (int)std::min<int64_t>(L, (int64_t)T * K);
    p->members = 256;  // the number of named experts comes first
    p->mid = p->members + up256((int64_t)p->slots * member_words(T) * 4);
    p->total = p->mid + up256((int64_t)T * K * inner * 2);
}

hipError_t launch_layer(const LayerArgs& a, hipStream_t s) {
    if (a.T == 0) return hipSuccess;
    LayerPlan plan;
    plan_layer(a.T, a.K, a.L, a.H, a.inner, &plan);
    const int slices = (a.inner + kRows - 1) / kRows;
    const dim3 grid((uint32_t)(plan.slots * slices));
    if (a.gated) hipLaunchKernelGGL(layer_up_kernel<2>, grid, dim3(64 * kUpWaves), 0, s, a, plan, slices);
    else hipLaunchKernelGGL(layer_up_kernel<1>, grid, dim3(64 * kUpWaves), 0, s, a, plan, slices);
    const size_t lds = (size_t)kDownWaves * a.T * 16 * sizeof(float);
    hipLaunchKernelGGL(layer_down_kernel, dim3((uint32_t)((a.H + kRows - 1) / kRows)), dim3(64 * kDownWaves), lds, s, a, plan);
    return hipGetLastError();
}

}  // namespace ep
