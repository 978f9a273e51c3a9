// The whole expert layer for a few tokens, without windows, in two launches.
//
//   out[t] = res[t] + sum_k w[t,k] (W2_e act(W1_e x[t] + b1_e) + b2_e),  e = topk_idx[t,k], local experts only
//
// What bounds it is reading the weights of the experts that are named, once.  Both kernels therefore stream
// weight rows from memory into registers as the left operand of MFMA 16x16x32, 16 rows at a time and several
// blocks ahead, the tokens that name the expert (up to 16 per instruction) being the right operand:
//   up    a workgroup per (named expert, some runs of 16 rows of the inner dimension): the contraction over H is split
//         over its wavefronts and joined through LDS in wave order; bias, activation and gate weight are applied in
//         float32, and one row per (token, expert) goes to the workspace in bf16, as between two products on windows.
//         (As two bf16 parts, which keep 16 bits: the result's error falls from 2.4e-3 to the 1.7e-3 of its own rounding, but
//         every workgroup of the second launch reads the rows twice: one token of 64 experts below 116 -> 122 us, 128 of 128 experts
//         703 -> 780, 128 tokens that all name the same 8 experts 610 -> 857.)  One more workgroup sorts the routed entries by
//         expert for the second launch.
//   down  a workgroup per 16 columns of the output: its wavefronts share out the (expert, part of the inner
//         dimension) pairs evenly, each adds up its own part of the output for all tokens in LDS, and the
//         parts are joined in wave order.  No atomics on values: results do not depend on timing.
// Measured: one token of 64 experts, top-8, 7168 and 2 x 2048: up 72 us (6.5 TB/s), down 43 (5.4, 448 workgroups on 256
// compute units); 128 tokens of 128 experts, 4096 and 2 x 1408, every expert named: 495 and 242 (6.0), one behind the other 702 (6.3).
// An expert works on its own tokens only, so what its weights hold (an infinity, a NaN) reaches no others.
#include <algorithm>

#include "ep_experts.h"
#include "ep_internal.h"

namespace ep {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kUpWaves = 4, kDownWaves = 8;
constexpr int kUpDepth = 4, kDownDepth = 4;   // blocks of weights on their way per wavefront
constexpr int kRows = 16;     // weight rows per run
constexpr int kBlock = 64;    // contraction indices per step of a wavefront: whole 128-byte lines of 16 rows
constexpr int kGroups = 4;    // groups of 16 tokens per pass over the weights
constexpr uint32_t kNowhere = 0x80000000u;  // offset of a lane that has nothing to load: reads zeros

// The routed entries by expert, as the second launch wants them (in the workspace): the number of named experts, their
// ids and where their entries start (one more than there are experts), then the entries: t * K + k, which is the row between
// the products.  A token that names an expert twice has one entry.  All of them are below 2^16: 128 tokens of 64 entries.
struct Sorted {
    uint16_t *count, *expert, *start, *entry;
};
static_assert(kLayerMaxTokens * kMaxTopK < 1 << 16 && kMaxExperts < 1 << 16, "16 bits");
__host__ __device__ constexpr int64_t sorted_words(int slots, int entries) { return (2 + 2 * slots + entries + 1) / 2; }   // of 32 bits
__host__ __device__ inline Sorted sorted_at(uint8_t* base, int slots) {
    uint16_t* p = (uint16_t*)base;
    return {p, p + 1, p + 1 + slots, p + 2 + 2 * slots};
}

__device__ __forceinline__ float load_bias(const void* b, int64_t i, int is_f32) {
    return is_f32 ? ((const float*)b)[i] : bf16_f32(((const uint16_t*)b)[i]);
}

// The id that entry (t, k) names among the local experts, or -1.
__device__ __forceinline__ int local_id(const LayerArgs& a, int t, int k) {
    const int64_t e = (int64_t)a.topk_idx[t * a.idx_stride + k] - a.first;
    return e >= 0 && e < a.L ? (int)e : -1;
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(const void* p) {
    return __builtin_amdgcn_make_buffer_rsrc((void*)p, 0, 0x7fffffff, 0x00027000);
}

__device__ __forceinline__ bf16x8 load8(__amdgpu_buffer_rsrc_t r, uint32_t off) {
    return __builtin_bit_cast(bf16x8, __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, 0));
}

// The weights of a block (16 rows of 128 bytes per matrix) go to LDS without passing through registers: the eight lanes of
// a row load a whole line in one instruction, which is what lets the non-temporal hint pay (a plain sweep over rows, TB/s:
// whole lines with the hint 7.0 to 7.3, without 6.2 to 6.5; half lines, as the matrix instruction wants its operand, 6.2
// without and 5.5 to 6.0 with it).  The unit u of row r lies at u ^ (r & 7): a fragment read touches all banks.  Each
// wavefront has a ring of its own, no barriers.
constexpr int kWeightBlock = kRows * kBlock * 2;
constexpr int kNonTemporal = 2;   // cache policy bit of a buffer load: for weights whose rows start on lines

typedef __attribute__((address_space(3))) void* lds_ptr;

// acc[g][jt] += 16 weight rows (of each of G matrices) x the tokens of JT groups of 16, over the blocks b0, b0 + stride, ..
// below b1 of the contraction (K indices in all), DEPTH of them on their way at any time.  wo: the lane's offset in the first
// and in the second eight weight rows, its unit included; xo: its token's row in each group, kNowhere if there is none.
template <int G, int JT, int DEPTH, int ROWS, bool NT>
__device__ __forceinline__ void multiply(f32x4 (&acc)[G][kGroups], const __amdgpu_buffer_rsrc_t (&w)[G], const uint32_t (&wo)[2],
                                         __amdgpu_buffer_rsrc_t x, const uint32_t (&xo)[kGroups], char* ring, int b0, int b1, int stride, int K, int lane) {
    constexpr int kHalves = ROWS / 8, kLoads = kHalves * G + 2 * JT;   // per block
    bf16x8 xf[DEPTH][JT][2];
    const int wk = ((lane & 7) ^ (lane >> 3)) * 8, xk = (lane >> 4) * 8;
    auto load = [&](int d, int b) {
        const int left = b < b1 ? K - b * kBlock : 0;
        const uint32_t out = wk < left ? 0 : kNowhere;   // an offset with this bit is beyond the buffer's end
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
            for (int s = 0; s < kHalves; ++s)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(w[g], (lds_ptr)(ring + (d * G + g) * kWeightBlock + s * 1024), 16,
                                                         (wo[s] + b * (kBlock * 2)) | out, 0, 0, NT ? kNonTemporal : 0);
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const uint32_t gone = s * 32 + xk < left ? 0 : kNowhere;
#pragma unroll
            for (int jt = 0; jt < JT; ++jt) xf[d][jt][s] = load8(x, (xo[jt] + (b * kBlock + s * 32 + xk) * 2) | gone);
        }
    };
    const char* mine = ring + (lane & 15) * 128;
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) load(d, b0 + d * stride);
    for (int b = b0; b < b1; b += DEPTH * stride) {
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"((DEPTH - 1) * kLoads) : "memory");
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    const bf16x8 wf = *(const bf16x8*)(mine + (d * G + g) * kWeightBlock + (((s * 4 + (lane >> 4)) ^ (lane & 7)) << 4));
#pragma unroll
                    for (int jt = 0; jt < JT; ++jt)
                        acc[g][jt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf, xf[d][jt][s], acc[g][jt], 0, 0, 0);
                }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the block has been read before its place is loaded again
            __builtin_amdgcn_sched_barrier(0);
            load(d, b + (DEPTH + d) * stride);
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // nothing writes to the ring any more
}

// The same for up to 16 tokens and several runs of `blocks` blocks one after the other, without a pause between them: items
// [q0, q1) count blocks, item q is block q % blocks of run q / blocks.  open(run, w, wo, xo) points at a run's weights and
// rows, close(run, acc) takes its sums (of what lies in [q0, q1)).
template <int G, int DEPTH, int ROWS, bool NT, class Open, class Close>
__device__ __forceinline__ void stream(int64_t q0, int64_t q1, int blocks, __amdgpu_buffer_rsrc_t x, char* ring, int K, int lane, Open open, Close close) {
    constexpr int kHalves = ROWS / 8, kLoads = kHalves * G + 2;
    if (q0 >= q1) return;
    __amdgpu_buffer_rsrc_t w[G];
    uint32_t wo[2], xo;
    bf16x8 xf[DEPTH][2];
    const int wk = ((lane & 7) ^ (lane >> 3)) * 8, xk = (lane >> 4) * 8;
    int run = (int)(q0 / blocks), b = (int)(q0 - (int64_t)run * blocks);   // of the item to multiply next
    int run_ahead = run, b_ahead = b;                                      // and to load next
    int to_load = (int)(q1 - q0);
    open(run, w, wo, xo);
    auto load = [&](int d) {
        if (b_ahead == blocks && to_load > 0) {
            b_ahead = 0;
            open(++run_ahead, w, wo, xo);
        }
        const int left = to_load > 0 ? K - b_ahead * kBlock : 0;
        const uint32_t out = wk < left ? 0 : kNowhere;   // an offset with this bit is beyond the buffer's end
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
            for (int s = 0; s < kHalves; ++s)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(w[g], (lds_ptr)(ring + (d * G + g) * kWeightBlock + s * 1024), 16,
                                                         (wo[s] + b_ahead * (kBlock * 2)) | out, 0, 0, NT ? kNonTemporal : 0);
#pragma unroll
        for (int s = 0; s < 2; ++s)
            xf[d][s] = load8(x, (xo + (b_ahead * kBlock + s * 32 + xk) * 2) | (s * 32 + xk < left ? 0 : kNowhere));
        ++b_ahead;
        --to_load;
    };
    const char* mine = ring + (lane & 15) * 128;
    f32x4 acc[G];
#pragma unroll
    for (int g = 0; g < G; ++g) acc[g] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) load(d);
    // Whole rounds, the last one filled up with loads and products of nothing: a way out in between would join the way back to
    // the top, and the compiler would then wait there for all loads in every round.
    for (int left = (int)(q1 - q0); left > 0;) {
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"((DEPTH - 1) * kLoads) : "memory");
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    const bf16x8 wf = *(const bf16x8*)(mine + (d * G + g) * kWeightBlock + (((s * 4 + (lane >> 4)) ^ (lane & 7)) << 4));
                    acc[g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf, xf[d][s], acc[g], 0, 0, 0);
                }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the block has been read before its place is loaded again
            __builtin_amdgcn_sched_barrier(0);
            load(d);
            --left;
            if (left >= 0 && (++b == blocks || left == 0)) {
                close(run, acc);
#pragma unroll
                for (int g = 0; g < G; ++g) acc[g] = f32x4{0, 0, 0, 0};
                ++run;
                b = 0;
            }
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // nothing writes to the ring any more
}

// The same where the rows of weights do not start on lines.  Loaded as they are wanted, each line would come in two parts, at
// two times (20 tokens of 64 experts, 3512 and 2 x 1208: 396 us; by lines 299).  So the lines themselves are loaded, each once: chunk c of a row is its
// c-th line, and a block of 64 indices lies in chunks b and b + 1, from unit `shift` of the row on.  Items [q0, q1) as
// above; weights(run, g) points at the first of a run's rows, of which rows(run) exist, `stride` elements apart; row(run) is the
// lane's token row.
template <int G, int DEPTH, int ROWS, class Weights, class Rows, class Row, class Close>
__device__ __forceinline__ void stream_lines(int64_t q0, int64_t q1, int blocks, int64_t stride, __amdgpu_buffer_rsrc_t x, char* ring, int K, int lane,
                                             Weights weights, Rows rows, Row row, Close close) {
    constexpr int kHalves = ROWS / 8, kLoads = kHalves * G + 2;
    if (q0 >= q1) return;
    const int unit = (lane & 7) ^ (lane >> 3), xk = (lane >> 4) * 8;
    struct Place {          // a chunk: those of a run's part [from, to) are from, .., to
        int run, chunk, from, to, rest;   // rest: blocks of later runs
    };
    auto first = [&](int run, int from, int rest) {
        const int to = min(blocks, from + rest);
        return Place{run, from, from, to, rest - (to - from)};
    };
    Place in = first((int)(q0 / blocks), (int)(q0 % blocks), (int)(q1 - q0)), out = in;   // to load next, to multiply next
    __amdgpu_buffer_rsrc_t w[G];
    uint32_t wo[G][kHalves], xo;
    int shift[G][kHalves];          // units before the row's first in its first line
    auto open = [&] {
        const int there = rows(in.run);
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const uintptr_t p = (uintptr_t)weights(in.run, g);
            const uint32_t phase = (uint32_t)p & 127;
            w[g] = buffer((const void*)(p - phase));
#pragma unroll
            for (int s = 0; s < kHalves; ++s) {
                const int r = s * 8 + (lane >> 3);
                const uint32_t off = (uint32_t)(r * stride * 2) + phase;
                wo[g][s] = r < there ? (off & ~127u) + unit * 16 : kNowhere;
                shift[g][s] = (off & 127) >> 4;
            }
        }
        xo = row(in.run);
    };
    uint32_t at[G][2];   // the lane's unit of a fragment in its chunk, and whether that is the second one
    bool next[G][2];
    auto aim = [&] {
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const int r = lane & 15;
            const uint32_t off = (uint32_t)(r * stride * 2) + ((uint32_t)(uintptr_t)weights(out.run, g) & 127);
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const int u = s * 4 + (lane >> 4) + (int)((off & 127) >> 4);
                at[g][s] = g * kWeightBlock + r * 128 + (((u & 7) ^ (r & 7)) << 4);
                next[g][s] = u > 7;
            }
        }
    };
    bf16x8 xf[DEPTH][2];
    int to_load = (int)(q1 - q0) + (int)((q1 - 1) / blocks - q0 / blocks) + 1;
    auto load = [&](int d) {
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
            for (int s = 0; s < kHalves; ++s) {
                const bool there = to_load > 0 && (uint32_t)(in.chunk * 8 + unit - shift[g][s]) < (uint32_t)K / 8;
                __builtin_amdgcn_raw_ptr_buffer_load_lds(w[g], (lds_ptr)(ring + (d * G + g) * kWeightBlock + s * 1024), 16,
                                                         (wo[g][s] + in.chunk * 128) | (there ? 0 : kNowhere), 0, 0, kNonTemporal);
            }
        const int block = in.chunk - 1, left = to_load > 0 && in.chunk > in.from ? K - block * kBlock : 0;
#pragma unroll
        for (int s = 0; s < 2; ++s)
            xf[d][s] = load8(x, (xo + (uint32_t)(block * kBlock + s * 32 + xk) * 2) | (s * 32 + xk < left ? 0 : kNowhere));
        --to_load;
        if (in.chunk++ == in.to && to_load > 0) {
            in = first(in.run + 1, 0, in.rest);
            open();
        }
    };
    f32x4 acc[G];
#pragma unroll
    for (int g = 0; g < G; ++g) acc[g] = f32x4{0, 0, 0, 0};
    int left = to_load;
    open();
    aim();
#pragma unroll
    for (int d = 0; d < DEPTH - 1; ++d) load(d);
    while (left > 0) {   // whole rounds, as above
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            constexpr int kSlot = G * kWeightBlock;
            const int before = (d + DEPTH - 1) % DEPTH;
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"((DEPTH - 2) * kLoads) : "memory");
            __builtin_amdgcn_sched_barrier(0);
            if (left > 0 && out.chunk > out.from) {
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int g = 0; g < G; ++g) {
                        const bf16x8 wf = *(const bf16x8*)(ring + at[g][s] + (next[g][s] ? d : before) * kSlot);
                        acc[g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf, xf[d][s], acc[g], 0, 0, 0);
                    }
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // both chunks have been read before the earlier one's place is loaded again
            __builtin_amdgcn_sched_barrier(0);
            load(before);
            if (--left >= 0 && out.chunk++ == out.to) {
                close(out.run, acc);
#pragma unroll
                for (int g = 0; g < G; ++g) acc[g] = f32x4{0, 0, 0, 0};
                out = first(out.run + 1, 0, out.rest);
                if (left > 0) aim();
            }
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // nothing writes to the ring any more
}

// By the number of tokens: the more groups, the fewer blocks of them fit the registers.
template <int G, int DEPTH, int ROWS, bool NT>
__device__ __forceinline__ void multiply_groups(int n, f32x4 (&acc)[G][kGroups], const __amdgpu_buffer_rsrc_t (&w)[G], const uint32_t (&wo)[2],
                                                __amdgpu_buffer_rsrc_t x, const uint32_t (&xo)[kGroups], char* ring, int b0, int b1, int stride, int K, int lane) {
    if (n <= 16) multiply<G, 1, DEPTH, ROWS, NT>(acc, w, wo, x, xo, ring, b0, b1, stride, K, lane);
    else if (n <= 32) multiply<G, 2, 3, ROWS, NT>(acc, w, wo, x, xo, ring, b0, b1, stride, K, lane);
    else multiply<G, 4, 2, ROWS, NT>(acc, w, wo, x, xo, ring, b0, b1, stride, K, lane);
}

// The lane's offsets in the two halves of 16 weight rows `stride` elements apart, of which `rows` exist.
__device__ __forceinline__ void weight_offsets(uint32_t (&wo)[2], int64_t stride, int rows, int lane) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        const int r = s * 8 + (lane >> 3);
        wo[s] = r < rows ? (uint32_t)(r * stride * 2) + (((lane & 7) ^ (lane >> 3)) << 4) : kNowhere;
    }
}

// The routed entries sorted by expert, by one workgroup, from their local ids.  The order of an expert's entries is
// arbitrary: each token's column is a sum of its own.
__device__ __forceinline__ void sort_entries(const LayerArgs& a, const LayerPlan& plan, const int16_t* ids, int* fill) {
    const Sorted out = sorted_at(a.workspace, plan.slots);
    for (int e = threadIdx.x; e < kMaxExperts; e += 64 * kUpWaves) fill[e] = 0;
    __syncthreads();
    auto entry_id = [&](int i) {   // -1 for the second entry of a token that names the same expert, too
        const int e = ids[i];
        for (int q = i - i % a.K; q < i && e >= 0; ++q)
            if (ids[q] == e) return -1;
        return e;
    };
    for (int i = threadIdx.x; i < a.T * a.K; i += 64 * kUpWaves) {
        const int e = entry_id(i);
        if (e >= 0) atomicAdd(&fill[e], 1);
    }
    __syncthreads();
    if (threadIdx.x < 64) {
        constexpr int kPer = kMaxExperts / 64;
        const int lane = threadIdx.x, e0 = lane * kPer;
        int n[kPer], sum = 0, named = 0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            n[i] = fill[e0 + i];
            sum += n[i];
            named += n[i] > 0;
        }
        int s1 = sum, n1 = named;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int v = __shfl_up(s1, d), u = __shfl_up(n1, d);
            if (lane >= d) { s1 += v; n1 += u; }
        }
        int at = s1 - sum, slot = n1 - named;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            fill[e0 + i] = at;
            if (n[i] > 0) {
                out.expert[slot] = (uint16_t)(e0 + i);
                out.start[slot] = (uint16_t)at;
                ++slot;
                at += n[i];
            }
        }
        if (lane == 63) {
            *out.count = (uint16_t)n1;
            out.start[n1] = (uint16_t)s1;
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < a.T * a.K; i += 64 * kUpWaves) {
        const int e = entry_id(i);
        if (e >= 0) out.entry[atomicAdd(&fill[e], 1)] = (uint16_t)i;
    }
}

// SPLIT: wavefronts that share the contraction of a run of rows, 4 or 1.
template <int G, int SPLIT, bool NT>
__global__ __launch_bounds__(64 * kUpWaves, 2) void layer_up_kernel(const LayerArgs a, const LayerPlan plan) {
    // each wavefront's ring of weights; afterwards its part of the sums, or the sort's counters
    __shared__ __attribute__((aligned(1024))) char rings[kUpWaves][kUpDepth * G * kWeightBlock];
    __shared__ uint32_t named[kMaxExperts / 32];
    __shared__ int s_n[2];
    __shared__ int s_token[kLayerMaxTokens], s_row[kLayerMaxTokens];
    __shared__ float s_gate[kLayerMaxTokens];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int16_t* ids = (int16_t*)rings;   // local ids of all entries, until the weights come
    static_assert(sizeof(rings) >= 2 * kLayerMaxTokens * kMaxTopK + 4 * kMaxExperts, "ids and the sort's counters");
    if (threadIdx.x < kMaxExperts / 32) named[threadIdx.x] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < a.T * a.K; i += 64 * kUpWaves) {
        const int e = local_id(a, i / a.K, i % a.K);
        ids[i] = (int16_t)e;
        if (e >= 0) atomicOr(&named[e >> 5], 1u << (e & 31));
    }
    __syncthreads();
    if (blockIdx.x == 0) {
        sort_entries(a, plan, ids, (int*)(ids + kLayerMaxTokens * kMaxTopK));
        return;
    }
    // the shares of an expert's tokens on the same XCD, whose L2 they have the weights from
    const int units = plan.slots * plan.up_parts, pitch8 = (units + 7) & ~7;
    const int unit = (blockIdx.x - 1) % pitch8, token_part = (blockIdx.x - 1) / pitch8;
    if (unit >= units) return;
    const int slot = unit / plan.up_parts, part = unit % plan.up_parts;

    // the slot-th of the experts that any token names
    const uint32_t word = lane < kMaxExperts / 32 ? named[lane] : 0u;
    int upto = __popc(word);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int v = __shfl_up(upto, d);
        if (lane >= d) upto += v;
    }
    if (slot >= __shfl(upto, 63)) return;
    const int at = __builtin_popcountll(__ballot(upto <= slot));  // the word that holds it: the counts only grow
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
            if (ids[t * a.K + k] == e) {
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
    __syncthreads();   // the ids have been read, too: weights may take their place

    const auto x = buffer(a.x);
    uint16_t* mid = (uint16_t*)(a.workspace + plan.mid);
    const int blocks = (a.H + kBlock - 1) / kBlock;
    const int slices = (a.inner + kRows - 1) / kRows;
    // Four sums of one token (position pos of the list), rows i0 + 4 (lane / 16) on, to the workspace.  The gate weight goes
    // in before the rounding to bf16: one rounding of the product of both.
    auto finish = [&](int i0, int pos, const f32x4 (&sum)[G]) {
        const int ii = i0 + (lane >> 4) * 4;
        if (pos >= n || ii >= a.inner) return;
        float h[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            float v[G];
#pragma unroll
            for (int g = 0; g < G; ++g) v[g] = sum[g][r] + (a.b_up ? load_bias(a.b_up, e * a.b_up_stride + ii + r + g * a.inner, a.b_up_f32) : 0.0f);
            h[r] = activate(a.act, v[0]);
            if (G == 2) h[r] *= v[G - 1];
            h[r] *= s_gate[pos];
        }
        *(uint2*)(mid + (int64_t)s_row[pos] * a.inner + ii) = make_uint2(pack2_bf16(h[0], h[1]), pack2_bf16(h[2], h[3]));
    };
    auto weights_of = [&](int i0, __amdgpu_buffer_rsrc_t (&w)[G]) {
#pragma unroll
        for (int g = 0; g < G; ++g) w[g] = buffer(a.w_up + e * a.up_expert + (int64_t)(i0 + g * a.inner) * a.up_row);
    };
    constexpr int kRuns = kUpWaves / SPLIT;   // of rows, next to each other
    const int first = part * kRuns + wave / SPLIT, pitch = plan.up_parts * kRuns;
    auto slice_weights = [&](int slice, int g) { return a.w_up + e * a.up_expert + (int64_t)(slice * kRows + g * a.inner) * a.up_row; };
    if (SPLIT == 1 && n <= 16) {
        const int mine = first < slices ? (slices - first + pitch - 1) / pitch : 0;
        const uint32_t xo = (lane & 15) < n ? (uint32_t)(s_token[lane & 15] * a.x_stride * 2) : kNowhere;
        auto close = [&](int run, const f32x4 (&acc)[G]) { finish((first + run * pitch) * kRows, lane & 15, acc); };
        if constexpr (NT)
            stream<G, kUpDepth, kRows, NT>(0, (int64_t)mine * blocks, blocks, x, rings[wave], a.H, lane,
                [&](int run, __amdgpu_buffer_rsrc_t (&w)[G], uint32_t (&wo)[2], uint32_t& row) {
                    const int i0 = (first + run * pitch) * kRows;
                    weights_of(i0, w);
                    weight_offsets(wo, a.up_row, a.inner - i0, lane);
                    row = xo;
                }, close);
        else
            stream_lines<G, kUpDepth, kRows>(0, (int64_t)mine * blocks, blocks, a.up_row, x, rings[wave], a.H, lane,
                [&](int run, int g) { return slice_weights(first + run * pitch, g); }, [&](int run) { return a.inner - (first + run * pitch) * kRows; },
                [&](int) { return xo; }, close);
        return;
    }
    for (int slice = first; slice - wave / SPLIT < slices; slice += pitch) {
        if (SPLIT == 1 && slice >= slices) break;
        const int i0 = slice * kRows;
        uint32_t wo[2];
        weight_offsets(wo, a.up_row, a.inner - i0, lane);
        __amdgpu_buffer_rsrc_t w[G];
        weights_of(i0, w);
        for (int p0 = token_part * plan.token_step; p0 < n; p0 += plan.token_parts * plan.token_step) {
            const int p1 = min(n, p0 + plan.token_step);
            uint32_t xo[kGroups];
            f32x4 acc[G][kGroups];
#pragma unroll
            for (int jt = 0; jt < kGroups; ++jt) {
                const int pos = p0 + jt * 16 + (lane & 15);
                xo[jt] = pos < p1 ? (uint32_t)(s_token[pos] * a.x_stride * 2) : kNowhere;
#pragma unroll
                for (int g = 0; g < G; ++g) acc[g][jt] = f32x4{0, 0, 0, 0};
            }
            multiply_groups<G, kUpDepth, kRows, NT>(p1 - p0, acc, w, wo, x, xo, rings[wave], wave % SPLIT, blocks, SPLIT, a.H, lane);
#pragma unroll
            for (int jt = 0; jt < kGroups; ++jt) {
                if (p0 + jt * 16 >= p1) break;
                f32x4 sum[G];
#pragma unroll
                for (int g = 0; g < G; ++g) sum[g] = acc[g][jt];
                if constexpr (SPLIT > 1) {   // wavefront 0 adds the others' parts to its own, in order
#pragma unroll
                    for (int g = 0; g < G; ++g) *(f32x4*)((float*)rings[wave] + (g * 64 + lane) * 4) = sum[g];
                    __syncthreads();
                    if (wave == 0) {
#pragma unroll
                        for (int g = 0; g < G; ++g)
#pragma unroll
                            for (int q = 1; q < SPLIT; ++q) sum[g] += *(const f32x4*)((const float*)rings[q] + (g * 64 + lane) * 4);
                        finish(i0, p0 + jt * 16 + (lane & 15), sum);
                    }
                    __syncthreads();
                } else {
                    finish(i0, p0 + jt * 16 + (lane & 15), sum);
                }
            }
        }
    }
}

// ROWS: columns of the output per workgroup, 16 or 8 (the other half of each instruction idle).
template <int ROWS, bool NT>
__global__ __launch_bounds__(64 * kDownWaves, 2) void layer_down_kernel(const LayerArgs a, const LayerPlan plan) {
    // each wavefront's ring of weights, its part of the output [T][16], then the sorted entries
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    float* sums = (float*)(lds + kDownWaves * kDownDepth * kWeightBlock);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int h0 = blockIdx.x * ROWS;
    uint32_t* words = (uint32_t*)(sums + kDownWaves * a.T * 16);
    for (int i = threadIdx.x; i < (int)sorted_words(plan.slots, a.T * a.K); i += 64 * kDownWaves) words[i] = ((const uint32_t*)a.workspace)[i];
    for (int i = threadIdx.x; i < kDownWaves * a.T * 16; i += 64 * kDownWaves) sums[i] = 0.0f;
    __syncthreads();
    const Sorted table = sorted_at((uint8_t*)words, plan.slots);
    auto token_of = [&](uint32_t entry) { return entry / (uint32_t)a.K; };
    float* mine = sums + wave * a.T * 16;

    const auto x = buffer(a.workspace + plan.mid);
    const int blocks = (a.inner + kBlock - 1) / kBlock;
    const int64_t items = (int64_t)*table.count * blocks;
    int64_t q = items * wave / kDownWaves;
    const int64_t end = items * (wave + 1) / kDownWaves;
    char* ring = lds + wave * (kDownDepth * kWeightBlock);
    uint32_t wo[2];
    weight_offsets(wo, a.down_row, min(ROWS, a.H - h0), lane);
    int most = 0;   // entries of one expert
    for (int i = lane; i < *table.count; i += 64) most = max(most, (int)table.start[i + 1] - (int)table.start[i]);
    if (!__any(most > 16)) {
        auto expert_of = [&](int slot) { return __builtin_amdgcn_readfirstlane(table.expert[slot]); };
        auto row_of = [&](int slot) {
            const int pos = table.start[slot] + (lane & 15);
            return pos < table.start[slot + 1] ? (uint32_t)table.entry[pos] * (uint32_t)a.inner * 2 : kNowhere;
        };
        auto close = [&](int slot, const f32x4 (&acc)[1]) {
            const int pos = table.start[slot] + (lane & 15);
            if (pos < table.start[slot + 1] && (lane >> 4) * 4 < ROWS) {
                f32x4* to = (f32x4*)(mine + token_of(table.entry[pos]) * 16 + (lane >> 4) * 4);
                *to = *to + acc[0];
            }
        };
        auto weights = [&](int slot, int) { return a.w_down + expert_of(slot) * a.down_expert + (int64_t)h0 * a.down_row; };
        // eight columns: few workgroups, for which the time of one counts (344 columns 9.3 against 12.9 us by lines)
        if constexpr (NT || ROWS == 8)
            stream<1, kDownDepth, ROWS, NT>(q, end, blocks, x, ring, a.inner, lane,
                [&](int slot, __amdgpu_buffer_rsrc_t (&w)[1], uint32_t (&to)[2], uint32_t& row) {
                    to[0] = wo[0];
                    to[1] = wo[1];
                    w[0] = buffer(weights(slot, 0));
                    row = row_of(slot);
                }, close);
        else
            stream_lines<1, kDownDepth, ROWS>(q, end, blocks, a.down_row, x, ring, a.inner, lane, weights, [&](int) { return min(ROWS, a.H - h0); }, row_of, close);
        q = end;
    }
    while (q < end) {
        const int slot = (int)(q / blocks), b0 = (int)(q - (int64_t)slot * blocks);
        const int b1 = (int)min((int64_t)blocks, b0 + (end - q));
        const int e = __builtin_amdgcn_readfirstlane(table.expert[slot]), first = __builtin_amdgcn_readfirstlane(table.start[slot]);
        const int n = __builtin_amdgcn_readfirstlane(table.start[slot + 1]) - first;
        const __amdgpu_buffer_rsrc_t w[1] = {buffer(a.w_down + e * a.down_expert + (int64_t)h0 * a.down_row)};
        for (int p0 = 0; p0 < n; p0 += kGroups * 16) {
            uint32_t xo[kGroups];
            f32x4 acc[1][kGroups];
#pragma unroll
            for (int jt = 0; jt < kGroups; ++jt) {
                const int pos = p0 + jt * 16 + (lane & 15);
                xo[jt] = pos < n ? (uint32_t)table.entry[first + pos] * (uint32_t)a.inner * 2 : kNowhere;
                acc[0][jt] = f32x4{0, 0, 0, 0};
            }
            multiply_groups<1, kDownDepth, ROWS, NT>(n - p0, acc, w, wo, x, xo, ring, b0, b1, 1, a.inner, lane);
#pragma unroll
            for (int jt = 0; jt < kGroups; ++jt) {
                const int pos = p0 + jt * 16 + (lane & 15);
                if (pos < n && (lane >> 4) * 4 < ROWS) {
                    f32x4* to = (f32x4*)(mine + token_of(table.entry[first + pos]) * 16 + (lane >> 4) * 4);
                    *to = *to + acc[0][jt];
                }
            }
        }
        q += b1 - b0;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < a.T * 16; i += 64 * kDownWaves) {
        const int t = i >> 4, c = h0 + (i & 15);
        if ((i & 15) >= ROWS || c >= a.H) continue;
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

int64_t down_lds(int T, int K, int slots) {
    return kDownWaves * (kDownDepth * kWeightBlock + (int64_t)T * 16 * 4) + sorted_words(slots, T * K) * 4;
}

}  // namespace

void plan_layer(int T, int K, int L, int H, int inner, LayerPlan* p) {
    p->slots = (int)std::min<int64_t>(L, (int64_t)T * K);
    p->mid = up256(sorted_words(p->slots, T * K) * 4);
    p->total = p->mid + up256((int64_t)T * K * inner * 2);
    p->up_parts = p->token_parts = p->token_step = 0;
}

hipError_t launch_layer(const LayerArgs& a, hipStream_t s) {
    if (a.T == 0) return hipSuccess;
    LayerPlan plan;
    plan_layer(a.T, a.K, a.L, a.H, a.inner, &plan);
    const int cus = compute_units();
    // Whole lines of weights: rows that start on lines.  A line that two blocks share would be fetched twice.
    auto lines = [](const void* p, int64_t expert, int64_t row) { return (uintptr_t)p % 128 == 0 && expert % 64 == 0 && row % 64 == 0; };
    // up: two workgroups share a compute unit.  Where there are runs of rows for half of their wavefronts, each takes runs of its
    // own and no sums are joined (13 tokens of 40 experts, 2888 into 2 x 504: 34 us; with runs shared 47.8), for all of them
    // where an expert has many tokens (64 of 8 experts, 2048 into 2 x 1024: 56.9 and 38.9); beyond that it takes several,
    // which spares the search for its expert's tokens.
    const int slices = (a.inner + kRows - 1) / kRows;
    const bool many = a.T * a.K > 16 * plan.slots;
    const bool split = (int64_t)plan.slots * slices < (many ? 2 : 1) * kUpWaves * (int64_t)cus;
    const int runs = split ? slices : (slices + kUpWaves - 1) / kUpWaves;
    plan.up_parts = std::clamp((4 * cus + plan.slots - 1) / plan.slots, 1, runs);
    // Where that leaves compute units idle, the tokens of an expert are shared out too: its weights then come from the L2
    // (104 tokens of one expert, 4912 into 136: 35.4 us in 9 workgroups, 10.4 in 63).
    const int groups = (a.T + 15) / 16;
    const int shares = split ? std::clamp(2 * cus / (plan.slots * plan.up_parts), 1, groups) : 1;
    plan.token_step = 16 * std::min(kGroups, (groups + shares - 1) / shares);
    plan.token_parts = std::min(shares, (a.T + plan.token_step - 1) / plan.token_step);
    const dim3 grid((uint32_t)((plan.slots * plan.up_parts + 7) / 8 * 8 * plan.token_parts + 1)), block(64 * kUpWaves);
    auto up = [&](auto g, auto n) {
        constexpr int G = decltype(g)::value, S = decltype(n)::value;
        if (lines(a.w_up, a.up_expert, a.up_row) && (!a.gated || a.inner * a.up_row % 64 == 0)) hipLaunchKernelGGL((layer_up_kernel<G, S, true>), grid, block, 0, s, a, plan);
        else hipLaunchKernelGGL((layer_up_kernel<G, S, false>), grid, block, 0, s, a, plan);
    };
    using one = std::integral_constant<int, 1>;
    using two = std::integral_constant<int, 2>;
    using four = std::integral_constant<int, 4>;
    if (a.gated) split ? up(two(), four()) : up(two(), one());
    else split ? up(one(), four()) : up(one(), one());
    // down: 8 columns per workgroup where all of those run at once (2048 columns on 256 compute units 4.7 us, with 16 5.1; 2888
    // columns 42 us, with 16 37.5)
    const bool narrow = (a.H + 7) / 8 <= cus;
    const dim3 columns((uint32_t)(narrow ? (a.H + 7) / 8 : (a.H + 15) / 16));
    const size_t lds = (size_t)down_lds(a.T, a.K, plan.slots);
    auto down = [&](auto rows) {
        constexpr int ROWS = decltype(rows)::value;
        if (lines(a.w_down, a.down_expert, a.down_row)) hipLaunchKernelGGL((layer_down_kernel<ROWS, true>), columns, dim3(64 * kDownWaves), lds, s, a, plan);
        else hipLaunchKernelGGL((layer_down_kernel<ROWS, false>), columns, dim3(64 * kDownWaves), lds, s, a, plan);
    };
    if (narrow) down(std::integral_constant<int, 8>());
    else down(std::integral_constant<int, 16>());
    return hipGetLastError();
}

}  // namespace ep
