// The experts' products: rows in expert windows times that expert's weights, forward and backward.
//
//   forward    out[r, :]  = act(x[r, :] W_e^T + b_e) (+ res[r, :])            W_e [N, Kd]
//   gradients  grad_x     = grad_pre W_e
//              grad_W_e   = grad_pre_e^T x_e,  grad_b_e = column sums of grad_pre_e
//
// All three are one tiled kernel over MFMA 16x16x32 with float32 accumulators.  The matrix instruction
// leaves each lane four consecutive rows of one column of its result, so the operand that runs along the
// contiguous axis of the output (P) is given as its left one and the other (Q) as its right one: a lane
// then owns four neighbouring values of an output row.  An operand whose contraction index is contiguous
// in memory is read from LDS 16 bytes per lane; one whose contraction index is the row (the weights of
// grad_x, both operands of grad_W) goes through the transposing LDS read.
//
// Measured: forward, 32768 rows of 8 experts, 7168 into 2 x 2048: 1.37 to 1.42 PFLOP/s, matrix units busy 82 to 85 % at the
// 1.6 GHz that the power limit leaves; both gradients of 16384 rows of 8, 4096 and 2 x 1408: 1.13 PFLOP/s, 61 % at 1.9 GHz; 128 rows
// each of 8, 7168 into 2 x 2048: 95 us, of which reading the weights takes 69.
#include <algorithm>
#include <atomic>

#include "ep_experts.h"
#include "ep_internal.h"

namespace ep {

namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void* lds_ptr;

constexpr int kSmall = 64;                    // indices of a small tile along P and along Q
constexpr int kBK = 64;                       // contraction indices per LDS tile
constexpr uint32_t kNowhere = 0x80000000u;    // offset of a lane that has nothing there: beyond the buffer's end, reads zeros

enum { FORWARD = 0, GRAD_ROWS = 1, GRAD_WEIGHTS = 2 };

// What the three kernels have in common.
struct Product {
    Windows win;
    const uint16_t *p, *q;
    int64_t p_expert, p_row, q_expert, q_row;
    uint16_t* out;
    int64_t out_expert, out_row;
    int I, J, Kc;        // extents along P, along Q (grad_W) and of the contraction (not grad_W)
    // forward
    int p_lines;         // rows of the weights start on 128-byte lines
    int act, gated;
    const void* bias;
    int64_t bias_stride;
    int bias_f32;
    uint16_t *pre, *res;
    int64_t pre_expert, pre_row, res_expert, res_row;
    int32_t* status;
    // grad_W
    int out_f32, accumulate;
    void* grad_b;
    int64_t gb_stride;
};

// Rows of expert e, cut to what the tensors hold, and the first of them.
__device__ __forceinline__ int window_rows(const Windows& w, int e, int64_t* first) {
    int64_t at = w.offset ? w.offset[e] : 0;
    int64_t n = w.count[e];
    if (n < 0 || at < 0 || at >= w.cap) n = 0;
    else if (n > w.cap - at) n = w.cap - at;
    *first = n > 0 ? at : 0;
    return (int)n;
}

// The windows of a call in LDS: first row and rows of each expert.  Its rows go in blocks of `rows`, or in one short block if
// half of that is enough for all of them (the short end of a longer window is a block like the others: it goes next to
// them, while the weights are in the L2; apart from them it would read the weights again, 668 against 711 us at 32 x 300 rows of
// 7168 into 2 x 2048).  starts[e], shorts[e]: blocks and short blocks before
// expert e, starts[L], shorts[L]: all of them; smalls: blocks of kSmall rows in all.
struct Table {
    int starts[kMaxExperts + 1], first[kMaxExperts], rows[kMaxExperts];
    uint16_t shorts[kMaxExperts + 2];
    int smalls;
};

__host__ __device__ constexpr int short_blocks(int n, int rows) { return n > 0 && n <= rows / 2; }
__host__ __device__ constexpr int whole_blocks(int n, int rows) { return short_blocks(n, rows) ? 0 : (n + rows - 1) / rows; }

// By one wavefront; SHORTS: short blocks are counted apart.  Returns whether a window reaches beyond its tensor.
template <bool SHORTS>
__device__ __forceinline__ bool scan_blocks(const Windows& w, int rows, Table* table, int lane) {
    const int per = (w.L + 63) / 64;
    const int e0 = lane * per, e1 = min(w.L, e0 + per);
    int whole = 0, brief = 0, small = 0;
    bool cut = false;
    for (int e = e0; e < e1; ++e) {
        int64_t at;
        const int n = window_rows(w, e, &at);
        cut |= n < w.count[e];
        table->first[e] = (int)at;
        table->rows[e] = n;
        whole += SHORTS ? whole_blocks(n, rows) : (n + rows - 1) / rows;
        brief += SHORTS ? short_blocks(n, rows) : 0;
        small += (n + kSmall - 1) / kSmall;
    }
    int w1 = whole, b1 = brief, s1 = small;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int u = __shfl_up(w1, d), v = __shfl_up(b1, d), w = __shfl_up(s1, d);
        if (lane >= d) { w1 += u; b1 += v; s1 += w; }
    }
    int wa = w1 - whole, ba = b1 - brief;
    for (int e = e0; e < e1; ++e) {
        table->starts[e] = wa;
        table->shorts[e] = (uint16_t)ba;
        const int n = table->rows[e];
        wa += SHORTS ? whole_blocks(n, rows) : (n + rows - 1) / rows;
        ba += SHORTS ? short_blocks(n, rows) : 0;
    }
    if (lane == 63) {
        table->starts[w.L] = w1;
        table->shorts[w.L] = (uint16_t)b1;
        table->smalls = s1;
    }
    return __any(cut);
}

// The same table in blocks of `rows` rows, none of them apart.  By one wavefront.
__device__ __forceinline__ void rescan_blocks(int L, int rows, Table* table, int lane) {
    const int per = (L + 63) / 64;
    const int e0 = lane * per, e1 = min(L, e0 + per);
    int all = 0;
    for (int e = e0; e < e1; ++e) all += (table->rows[e] + rows - 1) / rows;
    int upto = all;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int u = __shfl_up(upto, d);
        if (lane >= d) upto += u;
    }
    int at = upto - all;
    for (int e = e0; e < e1; ++e) {
        table->starts[e] = at;
        at += (table->rows[e] + rows - 1) / rows;
    }
    if (lane == 63) table->starts[L] = upto;
}

// The expert whose blocks hold block b: starts[e] <= b < starts[e + 1].
template <class T>
__device__ __forceinline__ int find_expert(const T* starts, int L, int b) {
    int lo = 0, hi = L;  // the answer is in [lo, hi)
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (starts[mid] <= b) lo = mid;
        else hi = mid;
    }
    return lo;
}

// ---- operand tiles -------------------------------------------------------------------------
//
// A tile of an operand is B indices x 64 contraction indices of bf16, in panels of 64 rows of 128 bytes (8 KiB).
// Contraction contiguous (KM): a panel is 64 indices; the 16-byte unit u of row r is stored at u ^ (r & 7), so that
// the 16 rows of a fragment read touch all banks.  Contraction along the rows: a panel is 64 contraction indices of 64
// neighbouring indices; the 32-byte block b of row k is stored at b ^ f(k), f(k) = k[1] | k[3] << 1: the eight rows
// that half a wave's transposing read takes lie in different banks.  Eight lanes load a row: whole 128-byte lines.

constexpr int kPanel = 64 * kBK * 2;

// A value that is the same in all lanes, where the compiler does not see that.
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(const void* p) {
    const uint64_t b = (uint64_t)p;
    const uint64_t at = (uint64_t)(uint32_t)uniform((int)(b >> 32)) << 32 | (uint32_t)uniform((int)b);
    return __builtin_amdgcn_make_buffer_rsrc((void*)at, 0, 0x7fffffff, 0x00027000);
}

__device__ __forceinline__ int spread(int k) { return ((k >> 1) & 1) | ((k >> 2) & 2); }

// Loads of sixteen bytes per lane from the buffer to LDS, lane after lane from the wave's address `at` on, the next load's STEP bytes
// behind.  Written in assembly, which has no output register: the compiler puts a wait for all such loads in front of every
// transposing LDS read when it knows of them, and would let none of them run ahead.  The waits are the caller's.
// A vector memory instruction may read an SGPR that a vector instruction has written (the descriptor's base, by readfirstlane)
// five wait states later at the earliest; the compiler sees to that for instructions of its own, not for these.  s_mov and
// s_nop 3 make up five, whatever stands in front; m0 itself needs one.  Once for all loads of a call: padded one by one they cost
// the products 1 to 5 % (32768 rows of 8 experts, 7168 into 2 x 2048: 1403 against 1385 us); one statement for both operands, 1 to 2 %.
// m0 is the compiler's own (it takes no word that an asm statement changes it), so nothing else in these kernels may use it.
#define EP_FIRST "s_mov_b32 m0, %0\n\ts_nop 3\n\t"
#define EP_NEXT "\n\ts_add_u32 m0, m0, %2\n\ts_nop 0\n\t"
#define EP_LOAD(n, hint) "buffer_load_dwordx4 %" #n ", %1, 0 offen " hint "lds"
#define EP_LOADS1(hint) EP_FIRST EP_LOAD(3, hint)
#define EP_LOADS2(hint) EP_LOADS1(hint) EP_NEXT EP_LOAD(4, hint)
#define EP_LOADS4(hint) EP_LOADS2(hint) EP_NEXT EP_LOAD(5, hint) EP_NEXT EP_LOAD(6, hint)
template <int STEP, int N>
__device__ __forceinline__ void load_to_lds(__amdgpu_buffer_rsrc_t rsrc, char* lds, const uint32_t (&off)[N], bool once) {
    static_assert(N == 1 || N == 2 || N == 4, "");
    const uint32_t at = (uint32_t)(uintptr_t)(lds_ptr)lds;
    if constexpr (N == 1) {
        if (once) asm volatile(EP_LOADS1("nt ") ::"s"(at), "s"(rsrc), "n"(STEP), "v"(off[0]) : "memory");
        else asm volatile(EP_LOADS1("") ::"s"(at), "s"(rsrc), "n"(STEP), "v"(off[0]) : "memory");
    } else if constexpr (N == 2) {
        if (once) asm volatile(EP_LOADS2("nt ") ::"s"(at), "s"(rsrc), "n"(STEP), "v"(off[0]), "v"(off[1]) : "memory", "scc");
        else asm volatile(EP_LOADS2("") ::"s"(at), "s"(rsrc), "n"(STEP), "v"(off[0]), "v"(off[1]) : "memory", "scc");
    } else {
        if (once) asm volatile(EP_LOADS4("nt ") ::"s"(at), "s"(rsrc), "n"(STEP), "v"(off[0]), "v"(off[1]), "v"(off[2]), "v"(off[3]) : "memory", "scc");
        else asm volatile(EP_LOADS4("") ::"s"(at), "s"(rsrc), "n"(STEP), "v"(off[0]), "v"(off[1]), "v"(off[2]), "v"(off[3]) : "memory", "scc");
    }
}
#undef EP_FIRST
#undef EP_NEXT
#undef EP_LOAD
#undef EP_LOADS1
#undef EP_LOADS2
#undef EP_LOADS4

template <int B, bool KM, int NW, bool HINT>
struct Operand {
    static constexpr int kLoads = B / 64 * 8 / NW;   // of 8 rows each, per wavefront
    static constexpr int kBytes = B * kBK * 2;
    uint32_t off[kLoads];
    const uint16_t* base;     // of the next contraction step to load
    int64_t step;             // elements per contraction step
    int k0;                   // contraction index of the lane's first unit (KM: the same in every load)
    // HINT: nobody else reads this tile, and it comes in whole lines: the non-temporal hint pays (1024 rows of 8 experts, 7168
    // into 2 x 2048: 101 -> 94 us).  On weights that several tiles read it costs, 46 -> 62 us where the memory-side cache holds them.
    int once = 0;

    // rows_of(r): the source row of tile row r relative to base, or -1
    template <class F>
    __device__ __forceinline__ void start_rows(const uint16_t* at, int64_t stride, int wave, int lane, F rows_of) {
        static_assert(KM, "");
        base = at;
        step = kBK;
        const int c = (lane & 7) ^ (lane >> 3);
        k0 = c * 8;
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int src = rows_of((j * NW + wave) * 8 + (lane >> 3));
            off[j] = src < 0 ? kNowhere : (uint32_t)(src * stride * 2) + c * 16;
        }
    }
    __device__ __forceinline__ void start_cols(const uint16_t* at, int64_t stride, int wave, int lane, int cols) {
        static_assert(!KM, "");
        base = at;
        step = kBK * stride;
        k0 = lane >> 3;
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int q = j * NW + wave, k = (q & 7) * 8 + (lane >> 3);
            const int c = (q >> 3) * 64 + ((((lane >> 1) & 3) ^ spread(k)) * 2 + (lane & 1)) * 8;
            off[j] = c < cols ? (uint32_t)((k * stride + c) * 2) : kNowhere;
        }
    }
    // Loads [j0, j1) of the tile of the current step; `left` = contraction indices that remain there.
    template <int J0, int J1>
    __device__ __forceinline__ void load(char* lds, int left, int wave) {
        const auto rsrc = buffer(base);
        const bool hint = HINT && uniform(once);
        uint32_t o[J1 - J0];
#pragma unroll
        for (int j = J0; j < J1; ++j) {
            const int k = KM ? k0 : k0 + ((j * NW + wave) & 7) * 8;
            o[j - J0] = k < left ? off[j] : kNowhere;
        }
        load_to_lds<NW * 1024>(rsrc, lds + (J0 * NW + wave) * 1024, o, hint);
    }
    __device__ __forceinline__ void next() { base += step; }
};

// What a lane adds to a tile's address to read its part of a fragment.
template <bool KM>
__device__ __forceinline__ uint32_t fragment_lane(int lane) {
    if constexpr (KM) return (lane & 15) * 128 + (((lane >> 4) ^ (lane & 7)) << 4);
    const int k = (lane >> 4) * 8 + ((lane & 15) >> 2);
    return k * 128 + spread(k) * 32 + (lane & 3) * 8;
}

// Fragment of the 16 indices from `at` (a multiple of 16) on and 32 contraction indices (half KS of the tile).
template <bool KM, int KS>
__device__ __forceinline__ bf16x8 fragment(const char* lds, int at, uint32_t mine) {
    if constexpr (KM) {
        return *(const bf16x8*)(lds + at * 128 + (mine ^ (KS * 64)));
    } else {
        const char* p = lds + (at >> 6) * kPanel + KS * 32 * 128 + (mine ^ (((at >> 4) & 3) * 32));
        s16x4 v[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) v[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(p + h * 512));
        const s16x8 both = __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7);
        return __builtin_bit_cast(bf16x8, both);
    }
}

__device__ __forceinline__ f32x4 widen(const u32x2& u) {
    return f32x4{__uint_as_float(u[0] << 16), __uint_as_float(u[0] & 0xffff0000u), __uint_as_float(u[1] << 16),
                 __uint_as_float(u[1] & 0xffff0000u)};
}

// Keeps what is computed from v inside the loop over the tiles: lifted out of it, it would hold registers all along.
__device__ __forceinline__ int opaque(int v) {
    asm volatile("" : "+v"(v));
    return v;
}

// Accesses of results: a lane that has nothing there reads zeros and writes nothing (offset kNowhere).
__device__ __forceinline__ f32x4 load4(__amdgpu_buffer_rsrc_t r, uint32_t off, int is_f32) {
    if (is_f32) return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, 0));
    return widen(__builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(r, off, 0, 0)));
}

// Four values each of two neighbouring fragments of P, for one index of Q, as bf16: the lanes of two neighbouring rows of
// 16 exchange halves, so that each writes eight values of one fragment, 16 bytes; four lanes write 64 in a row.
__device__ __forceinline__ void store8(__amdgpu_buffer_rsrc_t r, uint32_t off, const f32x4& v, const f32x4& w) {
    const auto lo = __builtin_amdgcn_permlane16_swap(pack2_bf16(v[0], v[1]), pack2_bf16(w[0], w[1]), false, false);
    const auto hi = __builtin_amdgcn_permlane16_swap(pack2_bf16(v[2], v[3]), pack2_bf16(w[2], w[3]), false, false);
    const u32x4 u = {lo[0], hi[0], lo[1], hi[1]};
    __builtin_amdgcn_raw_buffer_store_b128(u, r, off, 0, 0);
}

// Adds to them what lies there: store8's exchange again gives each lane the values of its own.
__device__ __forceinline__ void add8(const u32x4& u, f32x4& v, f32x4& w) {
    const auto lo = __builtin_amdgcn_permlane16_swap(u[0], u[2], false, false);
    const auto hi = __builtin_amdgcn_permlane16_swap(u[1], u[3], false, false);
    v += widen(u32x2{lo[0], hi[0]});
    w += widen(u32x2{lo[1], hi[1]});
}

// Four values of one fragment for one index of Q, as bf16.
__device__ __forceinline__ void store4(__amdgpu_buffer_rsrc_t r, uint32_t off, const f32x4& v) {
    __builtin_amdgcn_raw_buffer_store_b64(u32x2{pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3])}, r, off, 0, 0);
}

// A barrier that nothing is moved across; it waits for nobody's memory accesses.
__device__ __forceinline__ void barrier() {
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
}

constexpr int kWaves = 8;            // wavefronts of a workgroup
constexpr int kBlockRows = 256;      // rows per tile; short blocks: half
constexpr int kFlatStages = 3;
constexpr int kSmallStages = 4;      // of two steps each
// Tiles of 256 x 256 in two stages, half as large ones in three, or those of 64 x 64 in four times two.
constexpr int kLdsTiles = std::max({2 * (256 + 256) * kBK * 2, kFlatStages * (128 + 256) * kBK * 2, 2 * kSmallStages * (kSmall + kSmall) * kBK * 2});

// What the tiles of a launch are: every one 256 along P (I); along Q (J) first the whole blocks, then the short ones.
struct Tiling {
    int columns;                // along I
    int blocks, shorts;         // grad_W: per expert
    int64_t whole, all;         // tiles of whole blocks, all tiles
};

// Tiles of one workgroup, BI indices of P by BJ of Q:
//   256 x 256   tiles [t, end) of whole blocks in steps of the grid
//   256 x 128   tiles [t, end) of short blocks (120 rows each of 32 experts, 7168 into 2 x 2048: 373 us in tiles of 256, 316 so)
//   128 x 256   the halves of the tiles from `from` on, whatever their blocks
//    64 x 64    tiles [t, end) of blocks of 64, one or two per workgroup
template <int KIND, int BI, int BJ>
__device__ __forceinline__ void product_tiles(const Product& a, char* lds, const Table* table, const Tiling& tiling, int64_t& t, int64_t from, int64_t end) {
    constexpr int NW = kWaves, NWI = BJ == 128 ? 4 : 2, NWJ = NW / NWI;   // wavefronts along P and along Q
    constexpr bool WIDE = BI == 256 && BJ == 256, HALVES = BI == 128, SMALL = BJ == kSmall;
    constexpr int kBlock = SMALL ? kSmall : kBlockRows;
    constexpr bool kPK = KIND == FORWARD, kQK = KIND != GRAD_WEIGHTS;
    constexpr int WI = BI / NWI, WJ = BJ / NWJ, IT = WI / 16, JT = WJ / 16;
    constexpr bool kHint = !WIDE && KIND != GRAD_WEIGHTS;
    using P = Operand<BI, kPK, NW, kHint>;
    using Q = Operand<BJ, kQK, NW, false>;
    constexpr int kStage = P::kBytes + Q::kBytes;
    constexpr int kLoads = P::kLoads + Q::kLoads;
    // Results: a store takes kPair fragments of P for one of Q.  A tile issues at least kStores of them per lane, whether a lane has
    // something there or not, and half as many where a gate takes half of the accumulators; the waits for loads that were issued
    // before them count on that.
    constexpr int kPair = SMALL ? 1 : 2, kStores = IT / kPair * JT, kGatedStores = IT / 2 / kPair * JT;
    static_assert(IT % (2 * kPair) == 0, "whole stores, gated ones too");
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wi = wave % NWI, wj = wave / NWI;

    // A gated tile holds BI/2 outputs: their gate and their up columns.
    const int bi = KIND == FORWARD && a.gated ? BI / 2 : BI;
    const int ni = tiling.columns;

    // Tile t: expert by expert, within an expert in bands of eight row blocks, within a band column block by column block.
    // Workgroups of one XCD (blockIdx mod 8) take neighbouring tiles, so that its L2 serves both operands.
    struct Tile {
        int e, i0, j0, rows, first;
        int first_i, alone;    // the first block along I; the only one along J of its expert
    };
    auto locate = [&](int64_t u) {
        Tile c;
        const int half = HALVES && u >= end - from;   // first halves, then second halves
        const int64_t tile = HALVES ? from + (half ? u - (end - from) : u) : u;
        const bool brief = HALVES ? tile >= tiling.whole : BJ == 128;
        const int64_t mine = brief ? tile - tiling.whole : tile;
        const int block = (int)(mine / ni);
        int start, m, ib;
        if (KIND == GRAD_WEIGHTS) {
            m = brief ? tiling.shorts : tiling.blocks;
            c.e = block / m;
            start = c.e * m;
        } else if (brief) {
            c.e = uniform(find_expert(table->shorts, a.win.L, block));
            start = block;
            m = 1;
        } else {
            c.e = uniform(find_expert(table->starts, a.win.L, block));
            start = uniform(table->starts[c.e]);
            m = uniform(table->starts[c.e + 1]) - start;
        }
        const int64_t local = mine - (int64_t)start * ni;
        const int band = (int)(local / (8 * ni)), height = min(8, m - band * 8), in = (int)(local - (int64_t)band * 8 * ni);
        ib = uniform(in / height);
        c.rows = uniform(table->rows[c.e]);
        c.first = uniform(table->first[c.e]);
        c.j0 = uniform(band * 8 + in - ib * height) * kBlock;
        c.i0 = ib * (HALVES ? 2 * bi : bi) + half * bi;
        c.first_i = c.i0 == 0;
        c.alone = KIND != GRAD_WEIGHTS && c.rows <= kBlock;
        return c;
    };
    P p;
    Q q;
    auto steps_of = [&](const Tile& c) { return ((KIND == GRAD_WEIGHTS ? c.rows : a.Kc) + kBK - 1) / kBK; };
    // Small tiles: both steps of a turn.
    auto load_turn = [&](int stage, int left) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            char* to = lds + (stage * 2 + h) * kStage;
            p.template load<0, P::kLoads>(to, left - h * kBK, wave);
            q.template load<0, Q::kLoads>(to + P::kBytes, left - h * kBK, wave);
            p.next(); q.next();
        }
    };
    // Points the operands at a tile and issues its first loads: all of step 0, and of step 1 all (or what its phase 0 reads).
    auto begin = [&](const Tile& c) {
        const int lane = opaque(threadIdx.x & 63);
        const uint16_t* pb = a.p + c.e * a.p_expert;
        if (kHint) p.once = c.alone && a.p_lines;
        if constexpr (KIND == FORWARD) {
            const int I = a.I, gated = a.gated, i0 = c.i0;
            p.start_rows(pb + c.i0 * a.p_row, a.p_row, wave, lane, [=](int r) {
                if (!gated) return i0 + r < I ? r : -1;
                const int at = (r / WI) * (WI / 2) + r % (WI / 2);           // output column of the tile
                return i0 + at < I ? at + ((r % WI) / (WI / 2)) * I : -1;    // second half of a wave's rows: up
            });
        } else if constexpr (KIND == GRAD_ROWS) {
            p.start_cols(pb + c.i0, a.p_row, wave, lane, a.I - c.i0);
        } else {
            p.start_cols(pb + c.first * a.p_row + c.i0, a.p_row, wave, lane, a.I - c.i0);
        }
        const uint16_t* qb = a.q + c.e * a.q_expert + c.first * a.q_row;
        const int rows_left = c.rows - c.j0;
        if constexpr (kQK) q.start_rows(qb + c.j0 * a.q_row, a.q_row, wave, lane, [=](int r) { return r < rows_left ? r : -1; });
        else q.start_cols(qb + c.j0, a.q_row, wave, lane, a.J - c.j0);
        const int Kc = KIND == GRAD_WEIGHTS ? c.rows : a.Kc;
        if constexpr (SMALL) {
#pragma unroll
            for (int k = 0; k < kSmallStages - 1; ++k) load_turn(k, Kc - k * 2 * kBK);
        } else if (Kc > 0) {
            p.template load<0, P::kLoads>(lds, Kc, wave);
            q.template load<0, Q::kLoads>(lds + P::kBytes, Kc, wave);
            p.next(); q.next();
            if constexpr (WIDE) {
                if (Kc > kBK) {
                    p.template load<0, 1>(lds + kStage, Kc - kBK, wave);
                    p.template load<2, 3>(lds + kStage, Kc - kBK, wave);
                    q.template load<0, 4>(lds + kStage + P::kBytes, Kc - kBK, wave);
                }
            } else {
#pragma unroll
                for (int k = 1; k < kFlatStages - 1; ++k) {
                    if (k * kBK >= Kc) break;
                    p.template load<0, P::kLoads>(lds + k * kStage, Kc - k * kBK, wave);
                    q.template load<0, Q::kLoads>(lds + k * kStage + P::kBytes, Kc - k * kBK, wave);
                    p.next(); q.next();
                }
            }
        }
    };

    const int64_t tiles = HALVES ? 2 * (end - from) : end;
    Tile c;
    // The workgroup's next tile that is not empty, from t on.
    auto find = [&] {
        for (; t < tiles; t += gridDim.x) {
            c = locate(t);
            if (!HALVES || c.i0 < a.I) return true;   // the second half of a last tile may be empty
        }
        return false;
    };
    if (!find()) return;
    begin(c);
    int fresh = 1;   // since the tile's first loads no results have been stored, or fewer than a full tile's
    for (;;) {
        const int steps = steps_of(c);
        const int Kc = KIND == GRAD_WEIGHTS ? c.rows : a.Kc;
        f32x4 acc[IT][JT];
        f32x4 sums[JT];
#pragma unroll
        for (int jt = 0; jt < JT; ++jt) {
            sums[jt] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int it = 0; it < IT; ++it) acc[it][jt] = f32x4{0, 0, 0, 0};
        }
        const bool with_sums = uniform(KIND == GRAD_WEIGHTS && a.grad_b && c.first_i && wi == 0);

        // The residual, in the order of the stores (a small tile's per fragment, the others' in pairs).  A load behind stores
        // waits for them too, so it is read before the products: 99 -> 92 us with 3000 rows of 48 experts, 1000 into 2888.  The
        // wide tile has no registers for that and reads it as it stores.
        constexpr int kResidual = KIND != FORWARD || WIDE ? 1 : SMALL ? IT : IT / 2;
        using Residual = std::conditional_t<SMALL, u32x2, u32x4>;
        [[maybe_unused]] Residual res[kResidual][JT];
        auto read_residual = [&](const Tile& c) {
            const int mine = opaque(threadIdx.x & 63), g = mine >> 4;
            const int nit = a.gated ? IT / 2 : IT, iw = wi * (a.gated ? WI / 2 : WI) + (SMALL ? g * 4 : (g & 1) * 16 + (g >> 1) * 8), jw = wj * WJ + (mine & 15);
            const auto rr = buffer(a.res + c.e * a.res_expert + (c.first + c.j0) * a.res_row + c.i0);
#pragma unroll
            for (int k = 0; k < kResidual; ++k) {
                const int it = k * (SMALL ? 1 : 2);
                if (it < nit)
#pragma unroll
                    for (int jt = 0; jt < JT; ++jt) {
                        const int i = iw + it * 16, j = jw + jt * 16;
                        const uint32_t to = (j < c.rows - c.j0 ? (uint32_t)(j * a.res_row * 2) : kNowhere) + (i < a.I - c.i0 ? (uint32_t)(i * 2) : kNowhere - 1);
                        if constexpr (SMALL) res[k][jt] = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(rr, to, 0, 0));
                        else res[k][jt] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rr, to, 0, 0));
                    }
            }
        };
        if constexpr (KIND == FORWARD && !WIDE)
            if (a.res) read_residual(c);
        const uint32_t pl = fragment_lane<kPK>(lane), ql = fragment_lane<kQK>(lane);
        const bool idle = !WIDE && uniform(KIND != GRAD_WEIGHTS && wj * WJ >= c.rows - c.j0);   // none of the wavefront's rows exist
        const bool late = wave >= 4;
        const s16x8 one = {0x3f80, 0x3f80, 0x3f80, 0x3f80, 0x3f80, 0x3f80, 0x3f80, 0x3f80};
        if constexpr (WIDE) {
            // Two groups of four wavefronts, one of each per SIMD, half a phase apart: while one group multiplies, the
            // other reads fragments and issues loads.  A step has two phases, the halves of a wavefront's tile along P;
            // each is a load interval and a product interval of 32 instructions, and every interval ends in a barrier.
            // The tile two steps ahead takes the place of what all wavefronts have finished reading: P's first half and
            // Q after phase 0, P's second half after phase 1.  So six loads are issued in phase 1 of step k for step
            // k + 2 and two in phase 0 of step k + 1, and in both places waiting for all but the youngest eight leaves
            // what the next phase reads in LDS.
            static_assert(P::kLoads == 4 && Q::kLoads == 4 && NW == 8, "");
            constexpr int IH = IT / 2, kAhead = 1 + 1 + Q::kLoads;   // loads for step 1 that begin() issues
            if (steps) {
                // Step 0 has landed when only those for step 1 and the results stored since are on their way.
                if (steps == 1) {
                    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                } else if (uniform(fresh)) {
                    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kAhead) : "memory");
                } else if (KIND == FORWARD && a.gated) {
                    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kAhead + kGatedStores) : "memory");
                } else {
                    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kAhead + kStores) : "memory");
                }
                barrier();
                if (late) barrier();
            }
            for (int k = 0; k < steps; ++k) {
                char* cur = lds + (k & 1) * kStage;
                char* nxt = lds + ((k + 1) & 1) * kStage;
                const char* pc = cur + (wi * WI) * 128;
                const char* qc = cur + P::kBytes + (wj * WJ) * 128;
                bf16x8 pf[2][IH], qf[2][JT];
                auto read_p = [&](int half) {
#pragma unroll
                    for (int it = 0; it < IH; ++it) {
                        pf[0][it] = fragment<kPK, 0>(pc, (half * IH + it) * 16, pl);
                        pf[1][it] = fragment<kPK, 1>(pc, (half * IH + it) * 16, pl);
                    }
                };
                auto multiply = [&](int ih) {
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                    barrier();
                    __builtin_amdgcn_s_setprio(1);
#pragma unroll
                    for (int ks = 0; ks < 2; ++ks) {
#pragma unroll
                        for (int it = 0; it < IH; ++it)
#pragma unroll
                            for (int jt = 0; jt < JT; ++jt)
                                acc[ih * IH + it][jt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(pf[ks][it], qf[ks][jt], acc[ih * IH + it][jt], 0, 0, 0);
                        if (KIND == GRAD_WEIGHTS && ih == 0 && with_sums)  // sums over the rows as a product with ones
#pragma unroll
                            for (int jt = 0; jt < JT; ++jt)
                                sums[jt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, one), qf[ks][jt], sums[jt], 0, 0, 0);
                    }
                    __builtin_amdgcn_s_setprio(0);
                    barrier();
                };
                read_p(0);
#pragma unroll
                for (int jt = 0; jt < JT; ++jt) {
                    qf[0][jt] = fragment<kQK, 0>(qc, jt * 16, ql);
                    qf[1][jt] = fragment<kQK, 1>(qc, jt * 16, ql);
                }
                if (k + 1 < steps) {
                    p.template load<1, 2>(nxt, Kc - (k + 1) * kBK, wave);
                    p.template load<3, 4>(nxt, Kc - (k + 1) * kBK, wave);
                    p.next(); q.next();
                    asm volatile("s_waitcnt vmcnt(8)" ::: "memory");
                } else {
                    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                }
                multiply(0);
                read_p(1);
                if (k + 2 < steps) {
                    p.template load<0, 1>(cur, Kc - (k + 2) * kBK, wave);
                    p.template load<2, 3>(cur, Kc - (k + 2) * kBK, wave);
                    q.template load<0, 4>(cur + P::kBytes, Kc - (k + 2) * kBK, wave);
                    asm volatile("s_waitcnt vmcnt(8)" ::: "memory");
                } else {
                    asm volatile("s_waitcnt vmcnt(2)" ::: "memory");
                }
                multiply(1);
            }
            if (steps && !late) barrier();
        } else if constexpr (SMALL) {
            // Few tiles: what counts is how long one takes.  A turn is two steps of 64 and one barrier, in four stages, so that
            // the loads of three turns are on their way; behind the last step there are loads too, of nothing, which keeps
            // their number the same in every turn.  The barrier in front of turn k says that its tiles have landed and that
            // everybody has read turn k - 1, whose place the loads of turn k + 3 take.
            int stage = 0;
            for (int k = 0; k < steps; k += 2) {
                asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * (kSmallStages - 2) * kLoads) : "memory");
                barrier();
                const char* cur = lds + stage * 2 * kStage;
                bf16x8 pf[4][IT], qf[4][JT];
                if (!idle) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const char* pc = cur + h * kStage;
#pragma unroll
                        for (int it = 0; it < IT; ++it) {
                            pf[2 * h][it] = fragment<kPK, 0>(pc, wi * WI + it * 16, pl);
                            pf[2 * h + 1][it] = fragment<kPK, 1>(pc, wi * WI + it * 16, pl);
                        }
#pragma unroll
                        for (int jt = 0; jt < JT; ++jt) {
                            qf[2 * h][jt] = fragment<kQK, 0>(pc + P::kBytes, wj * WJ + jt * 16, ql);
                            qf[2 * h + 1][jt] = fragment<kQK, 1>(pc + P::kBytes, wj * WJ + jt * 16, ql);
                        }
                    }
                }
                load_turn(stage == 0 ? kSmallStages - 1 : stage - 1, Kc - (k / 2 + kSmallStages - 1) * 2 * kBK);
                stage = stage == kSmallStages - 1 ? 0 : stage + 1;
                if (idle) continue;
#pragma unroll
                for (int ks = 0; ks < 4; ++ks) {
#pragma unroll
                    for (int it = 0; it < IT; ++it)
#pragma unroll
                        for (int jt = 0; jt < JT; ++jt)
                            acc[it][jt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(pf[ks][it], qf[ks][jt], acc[it][jt], 0, 0, 0);
                    if (with_sums)
#pragma unroll
                        for (int jt = 0; jt < JT; ++jt)
                            sums[jt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, one), qf[ks][jt], sums[jt], 0, 0, 0);
                }
            }
            // everybody's loads, those of nothing too, are done before the next tile's take their places
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
            barrier();
        } else {
            // The same two groups with one load interval (all fragments of a step, 64 KiB of LDS reads per group) and one
            // product interval (32 instructions, as long) per step, and three stages: the loads of step k + 2 take the place
            // of step k - 1, which everybody has read.
            if (steps) {
                // besides step 1's loads the results stored since may be on their way
                if (steps == 1) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                else if (uniform(fresh)) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kLoads) : "memory");
                else asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kLoads + (KIND == FORWARD ? kGatedStores : kStores)) : "memory");
                barrier();
                if (late) barrier();
            }
            int stage = 0;
            for (int k = 0; k < steps; ++k) {
                const char* pc = lds + stage * kStage + wi * WI * 128;
                const char* qc = lds + stage * kStage + P::kBytes + wj * WJ * 128;
                bf16x8 pf[2][IT], qf[2][JT];
                if (!idle) {
#pragma unroll
                    for (int it = 0; it < IT; ++it) {
                        pf[0][it] = fragment<kPK, 0>(pc, it * 16, pl);
                        pf[1][it] = fragment<kPK, 1>(pc, it * 16, pl);
                    }
#pragma unroll
                    for (int jt = 0; jt < JT; ++jt) {
                        qf[0][jt] = fragment<kQK, 0>(qc, jt * 16, ql);
                        qf[1][jt] = fragment<kQK, 1>(qc, jt * 16, ql);
                    }
                }
                if (k + 2 < steps) {
                    char* to = lds + (stage == 0 ? 2 : stage - 1) * kStage;
                    p.template load<0, P::kLoads>(to, Kc - (k + 2) * kBK, wave);
                    q.template load<0, Q::kLoads>(to + P::kBytes, Kc - (k + 2) * kBK, wave);
                    p.next(); q.next();
                    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kLoads) : "memory");   // step k + 1 has landed
                } else {
                    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                }
                stage = stage == 2 ? 0 : stage + 1;
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                barrier();
                if (!idle) {
                    __builtin_amdgcn_s_setprio(1);
#pragma unroll
                    for (int ks = 0; ks < 2; ++ks) {
#pragma unroll
                        for (int it = 0; it < IT; ++it)
#pragma unroll
                            for (int jt = 0; jt < JT; ++jt)
                                acc[it][jt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(pf[ks][it], qf[ks][jt], acc[it][jt], 0, 0, 0);
                        if (with_sums)
#pragma unroll
                            for (int jt = 0; jt < JT; ++jt)
                                sums[jt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, one), qf[ks][jt], sums[jt], 0, 0, 0);
                    }
                    __builtin_amdgcn_s_setprio(0);
                }
                barrier();
            }
            if (steps && !late) barrier();
        }

        // The next tile's first loads run while this one's results are written.
        const Tile done = c;
        t += gridDim.x;
        const bool again = find();
        if (again) begin(c);

        // Results: lane l holds, for index j = l % 16 of a fragment of Q, the indices i = 4 (l / 16) .. + 3 of one of P;
        // stored in pairs of fragments (store8), eight of one: i8.
        const int mine = opaque(threadIdx.x & 63), g = mine >> 4;
        const int J = (KIND == GRAD_WEIGHTS ? a.J : done.rows) - done.j0;
        const int iw = wi * (KIND == FORWARD && a.gated ? WI / 2 : WI), jw = wj * WJ + (mine & 15);
        const int i4 = iw + g * 4, i8 = iw + (g & 1) * 16 + (g >> 1) * 8;
        const int Il = a.I - done.i0;   // columns of the tile that there are
        // Fragments of Q without a row: nothing to compute or to store (of a window with few rows most; the wide tile has few).
        auto gone = [&](int jt) { return !WIDE && KIND != GRAD_WEIGHTS && wj * WJ + jt * 16 >= J; };
        const int esize = KIND == GRAD_WEIGHTS && a.out_f32 ? 4 : 2;
        // Byte offset of (index j of fragment jt, column i) in a matrix whose rows are `row` elements apart.
        auto at = [&](int jt, int i, int64_t row, int size) {
            const int j = jw + jt * 16;
            return (j < J ? (uint32_t)(j * row * size) : kNowhere) + (i < Il ? (uint32_t)(i * size) : kNowhere - 1);
        };
        const char* out = (const char*)a.out;
        if constexpr (KIND == GRAD_WEIGHTS) out += (done.e * a.out_expert + done.j0 * a.out_row + done.i0) * esize;
        else out += (done.e * a.out_expert + (done.first + done.j0) * a.out_row + done.i0) * 2;
        const auto ro = buffer(out);
        if constexpr (KIND == FORWARD) {
            const int nit = a.gated ? IT / 2 : IT;
            if (a.bias) {
                const int size = a.bias_f32 ? 4 : 2;
                const auto rb = buffer((const char*)a.bias + (done.e * a.bias_stride + done.i0) * size);
#pragma unroll
                for (int it = 0; it < IT; ++it) {
                    const int i = i4 + (it < nit ? it : it - nit) * 16;
                    const f32x4 b = load4(rb, i < Il ? (uint32_t)((it < nit ? i : i + a.I) * size) : kNowhere, a.bias_f32);
#pragma unroll
                    for (int jt = 0; jt < JT; ++jt)
#pragma unroll
                        for (int r = 0; r < 4; ++r) acc[it][jt][r] += b[r];
                }
            }
            if (a.pre) {
                const auto rp = buffer(a.pre + done.e * a.pre_expert + (done.first + done.j0) * a.pre_row + done.i0);
#pragma unroll
                for (int it = 0; it < IT; it += kPair)
#pragma unroll
                    for (int jt = 0; jt < JT; ++jt) {
                        if (gone(jt)) continue;
                        const int i = (SMALL ? i4 : i8) + (it < nit ? it : it - nit) * 16;
                        const uint32_t to = at(jt, i, a.pre_row, 2) + (it < nit || i >= Il ? 0 : a.I * 2);
                        if constexpr (SMALL) store4(rp, to, acc[it][jt]);
                        else store8(rp, to, acc[it][jt], acc[it + 1][jt]);
                    }
            }
            const auto rr = buffer(a.res + done.e * a.res_expert + (done.first + done.j0) * a.res_row + done.i0);
            auto finish = [&](auto activation, auto gate) {
                constexpr int kN = decltype(gate)::value ? IT / 2 : IT;
#pragma unroll
                for (int it = 0; it < kN; it += kPair) {
#pragma unroll
                    for (int jt = 0; jt < JT; ++jt) {
                        if (gone(jt)) continue;
                        f32x4 v[kPair];
#pragma unroll
                        for (int h = 0; h < kPair; ++h)
#pragma unroll
                            for (int r = 0; r < 4; ++r) {
                                v[h][r] = activate(decltype(activation)::value, acc[it + h][jt][r]);
                                if (decltype(gate)::value) v[h][r] *= acc[(it + h + IT / 2) % IT][jt][r];
                            }
                        if (a.res) {
                            if constexpr (WIDE) {
#pragma unroll
                                for (int h = 0; h < kPair; ++h) v[h] += load4(rr, at(jt, i4 + (it + h) * 16, a.res_row, 2), 0);
                            } else if constexpr (SMALL) v[0] += widen(res[it][jt]);
                            else add8(res[it / 2 % kResidual][jt], v[0], v[1]);
                        }
                        if constexpr (SMALL) store4(ro, at(jt, i4 + it * 16, a.out_row, 2), v[0]);
                        else store8(ro, at(jt, i8 + it * 16, a.out_row, 2), v[0], v[1]);
                    }
                }
            };
            auto with = [&](auto activation) {
                if (a.gated) finish(activation, std::true_type());
                else finish(activation, std::false_type());
            };
            if (a.act == EP_ACT_SILU) with(std::integral_constant<int, EP_ACT_SILU>());
            else if (a.act == EP_ACT_GELU) with(std::integral_constant<int, EP_ACT_GELU>());
            else with(std::integral_constant<int, EP_ACT_NONE>());
        } else {
            if (KIND == GRAD_WEIGHTS && with_sums && g == 0) {
#pragma unroll
                for (int jt = 0; jt < JT; ++jt) {
                    if (jw + jt * 16 >= J) continue;
                    const int64_t to = done.e * a.gb_stride + done.j0 + jw + jt * 16;
                    if (a.out_f32) {
                        float* b = (float*)a.grad_b + to;
                        *b = a.accumulate ? *b + sums[jt][0] : sums[jt][0];
                    } else {
                        uint16_t* b = (uint16_t*)a.grad_b + to;
                        *b = (uint16_t)pack2_bf16(a.accumulate ? bf16_f32(*b) + sums[jt][0] : sums[jt][0], 0.0f);
                    }
                }
            }
            auto finish = [&](auto wide, auto accumulate) {
                constexpr int kSize = decltype(wide)::value ? 4 : 2;
#pragma unroll
                for (int it = 0; it < IT; it += 2)
#pragma unroll
                    for (int jt = 0; jt < JT; ++jt) {
                        if (gone(jt)) continue;
                        f32x4 v[2];
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            v[h] = acc[it + h][jt];
                            const uint32_t to = at(jt, i4 + (it + h) * 16, a.out_row, kSize);
                            if (decltype(accumulate)::value) {
                                const f32x4 old = load4(ro, to, kSize == 4);
#pragma unroll
                                for (int r = 0; r < 4; ++r) v[h][r] += old[r];
                            }
                            if (kSize == 4) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v[h]), ro, to, 0, 0);
                        }
                        if (kSize == 2) store8(ro, at(jt, i8 + it * 16, a.out_row, 2), v[0], v[1]);
                    }
            };
            if constexpr (KIND == GRAD_WEIGHTS) {
                if (a.out_f32) {
                    if (a.accumulate) finish(std::true_type(), std::true_type());
                    else finish(std::true_type(), std::false_type());
                } else {
                    if (a.accumulate) finish(std::false_type(), std::true_type());
                    else finish(std::false_type(), std::false_type());
                }
            } else {
                finish(std::false_type(), std::false_type());
            }
        }
        if (!again) return;
        fresh = uniform(gone(JT - 1));   // fewer results stored than the waits count on
    }
}

// All tiles of a product, by the workgroups of the grid, as the table has them.  `in`: the workgroup's place among those of
// its XCD.  Returns how many of each XCD had a tile of the last pass (0: any).
template <int KIND>
__device__ __forceinline__ int product(const Product& a, char* lds, Table* table, int in) {
    // The tiles go in rounds of the workgroups.  Where the last round would leave half of them without a tile it takes halves
    // instead, whose steps take 5/8 of the time: all of them for small inputs, in one round (64 rows each of 48 experts, 1000
    // into 2888: 94 us in whole tiles, 83 so).  Where even tiles of 64 x 64 fit one round, those: 2 rows of 20 experts,
    // 4704 into 944, take 45.5 us in halves and 18.1 so.  Or two rounds, where the contraction is long: 300 rows of one expert, 4096
    // into 4096, 54 us in halves and 38 so, but 2000 rows of 16 experts, 1000 into 520, 17 and 19.
    const int64_t experts = KIND == GRAD_WEIGHTS ? a.win.L : 1;
    const int per = gridDim.x >> 3;
    // The place of this workgroup in a round of n tiles, as many on each XCD and neighbours together; n where it has none.
    auto place = [&](int64_t n) {
        const int each = (int)(n + 7) >> 3;
        return in < each ? (int64_t)(blockIdx.x & 7) * each + in : n;
    };
    Tiling small = {(a.I * (KIND == FORWARD && a.gated ? 2 : 1) + kSmall - 1) / kSmall,
                    KIND == GRAD_WEIGHTS ? (a.J + kSmall - 1) / kSmall : uniform(table->smalls), 0, 0, 0};
    small.all = experts * small.blocks * small.columns;
    if (small.all <= (KIND != GRAD_WEIGHTS && a.Kc >= 2048 ? 2 : 1) * (int64_t)gridDim.x) {
        if (KIND != GRAD_WEIGHTS) {   // whose entries nobody has read yet
            if (threadIdx.x < 64) rescan_blocks(a.win.L, kSmall, table, threadIdx.x);
            __syncthreads();
        }
        int64_t at = small.all <= gridDim.x ? place(small.all) : (int64_t)(blockIdx.x & 7) * per + in;
        product_tiles<KIND, kSmall, kSmall>(a, lds, table, small, at, 0, small.all);
        return ((int)(small.all + 7) >> 3) % per;
    }
    Tiling t;
    t.columns = (a.I * (KIND == FORWARD && a.gated ? 2 : 1) + 255) / 256;
    t.blocks = KIND == GRAD_WEIGHTS ? whole_blocks(a.J, kBlockRows) : uniform(table->starts[a.win.L]);
    t.shorts = KIND == GRAD_WEIGHTS ? short_blocks(a.J, kBlockRows) : uniform(table->shorts[a.win.L]);
    t.whole = experts * t.blocks * t.columns;
    t.all = t.whole + experts * t.shorts * t.columns;
    int64_t rest = t.all % gridDim.x;
    if (2 * rest > gridDim.x) rest = 0;
    const int64_t mine = (int64_t)(blockIdx.x & 7) * per + in;
    int64_t at = mine;
    product_tiles<KIND, 256, 256>(a, lds, table, t, at, 0, min(t.whole, t.all - rest));
    product_tiles<KIND, 256, 128>(a, lds, table, t, at, 0, t.all - rest);
    at = place(2 * rest);
    product_tiles<KIND, 128, 256>(a, lds, table, t, at, t.all - rest, t.all);
    return (int)(2 * rest + 7) >> 3;
}

template <int KIND>
__global__ __launch_bounds__(64 * kWaves, 2) void product_kernel(const Product a) {
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    Table* table = (Table*)(lds + kLdsTiles);
    if (threadIdx.x < 64) {
        const bool cut = scan_blocks<true>(a.win, kBlockRows, table, threadIdx.x);
        if (KIND == FORWARD && cut && a.status && blockIdx.x == 0 && threadIdx.x == 0) atomicOr(a.status, STATUS_OUTPUT_OVERFLOW);
    }
    __syncthreads();
    product<KIND>(a, lds, table, blockIdx.x >> 3);
}

// Both gradients in one launch: where the tiles of grad_x do not fill the last round, those of grad_W begin.
__global__ __launch_bounds__(64 * kWaves, 2) void gradients_kernel(const Product x, const Product w) {
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    Table* table = (Table*)(lds + kLdsTiles);
    if (threadIdx.x < 64) scan_blocks<true>(x.win, kBlockRows, table, threadIdx.x);
    __syncthreads();
    const int per = gridDim.x >> 3, in = blockIdx.x >> 3;
    const int used = product<GRAD_ROWS>(x, lds, table, in) % per;
    product<GRAD_WEIGHTS>(w, lds, table, in >= used ? in - used : in - used + per);
}

// grad_pre = grad_out * d out / d pre, a workgroup per block of 16 rows: 16384 rows of 2 x 1408 in 49 us, 4.7 TB/s.  It is rounded
// to bf16 once, as the gradient that the caller gets, and the products read that: their errors then are those of two roundings
// (2.3e-3 against the 1.7e-3 of one).  A second bf16 part for them would double the matrix instructions that bound them.
constexpr int kActRows = 16;

__device__ __forceinline__ void unpack8(const uint4& u, float (&f)[8]) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        f[2 * c] = __uint_as_float(w[c] << 16);
        f[2 * c + 1] = __uint_as_float(w[c] & 0xffff0000u);
    }
}

__device__ __forceinline__ uint4 pack8(const float (&f)[8]) {
    return make_uint4(pack2_bf16(f[0], f[1]), pack2_bf16(f[2], f[3]), pack2_bf16(f[4], f[5]), pack2_bf16(f[6], f[7]));
}

__global__ __launch_bounds__(256) void act_backward_kernel(const ActBackwardArgs a) {
    __shared__ Table table;
    if (threadIdx.x < 64) scan_blocks<false>(a.win, kActRows, &table, threadIdx.x);
    __syncthreads();
    const int units = a.No / 8;
    for (int b = blockIdx.x; b < table.starts[a.win.L]; b += gridDim.x) {
        const int e = find_expert(table.starts, a.win.L, b);
        const int64_t first = table.first[e];
        const int r0 = (b - table.starts[e]) * kActRows, n = min(kActRows, table.rows[e] - r0);
        for (int i = threadIdx.x; i < n * units; i += 256) {
            const int r = r0 + i / units, c = (i % units) * 8;
            const uint16_t* pre = a.pre.base + e * a.pre.expert_stride + (first + r) * a.pre.row_stride + c;
            uint16_t* gp = a.grad_pre.base + e * a.grad_pre.expert_stride + (first + r) * a.grad_pre.row_stride + c;
            float g[8], v[8], u[8], o[8];
            unpack8(*(const uint4*)(a.grad_out.base + e * a.grad_out.expert_stride + (first + r) * a.grad_out.row_stride + c), g);
            unpack8(*(const uint4*)pre, v);
            if (a.gated) unpack8(*(const uint4*)(pre + a.No), u);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                float value;
                const float d = activate_grad(a.act, v[k], &value);
                o[k] = g[k] * d * (a.gated ? u[k] : 1.0f);
                u[k] = g[k] * value;
            }
            *(uint4*)gp = pack8(o);
            if (a.gated) *(uint4*)(gp + a.No) = pack8(u);
        }
    }
}

// Blocks of `rows` rows that there can be at most: every expert's last one may be short.
int64_t most_blocks(const Windows& w, int rows) {
    if (!w.offset) return (int64_t)w.L * ((w.cap + rows - 1) / rows);
    return w.cap / rows + w.L;
}

// Tiles of a product that there can be at most, small ones.
int64_t most_tiles(const Windows& w, int columns, int per_expert) {
    return (per_expert ? (int64_t)w.L * per_expert : most_blocks(w, kSmall)) * columns;
}

uint32_t product_grid(int64_t most) {
    const int64_t cus = std::max(8, compute_units() / 8 * 8);
    return (uint32_t)std::min(cus, (most + 7) / 8 * 8);
}

constexpr int kLds = kLdsTiles + (int)sizeof(Table);
static_assert(kLds <= 160 * 1024, "a compute unit's LDS");

template <int KIND>
hipError_t launch(const Product& a, int64_t most, hipStream_t s) {
    if (most <= 0) return hipSuccess;
    hipLaunchKernelGGL(product_kernel<KIND>, dim3(product_grid(most)), dim3(64 * kWaves), kLds, s, a);
    return hipGetLastError();
}

int small_blocks(int n) { return (n + kSmall - 1) / kSmall; }

}  // namespace

int compute_units() {
    static std::atomic<int> known[64];
    int dev = -1, n = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0) return 256;
    if (dev < 64 && (n = known[dev].load(std::memory_order_relaxed)) > 0) return n;
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n < 1) return 256;
    if (dev < 64) known[dev].store(n, std::memory_order_relaxed);
    return n;
}

hipError_t launch_product(const ProductArgs& a, hipStream_t s) {
    Product p = {};
    p.win = a.win;
    p.p = a.w; p.p_expert = a.w_expert; p.p_row = a.w_row;
    p.p_lines = (uintptr_t)a.w % 128 == 0 && a.w_expert % 64 == 0 && a.w_row % 64 == 0;
    p.q = a.x.base; p.q_expert = a.x.expert_stride; p.q_row = a.x.row_stride;
    p.out = a.out.base; p.out_expert = a.out.expert_stride; p.out_row = a.out.row_stride;
    p.I = a.No; p.Kc = a.Kd;
    p.act = a.act; p.gated = a.gated;
    p.bias = a.bias; p.bias_stride = a.bias_stride; p.bias_f32 = a.bias_f32;
    p.pre = a.pre.base; p.pre_expert = a.pre.expert_stride; p.pre_row = a.pre.row_stride;
    p.res = a.res.base; p.res_expert = a.res.expert_stride; p.res_row = a.res.row_stride;
    p.status = a.status;
    return launch<FORWARD>(p, most_tiles(a.win, small_blocks(a.gated ? 2 * a.No : a.No), 0), s);
}

hipError_t launch_gradients(const GradRowsArgs* rows, const GradWeightsArgs* weights, hipStream_t s) {
    Product x = {}, w = {};
    int64_t most_x = 0, most_w = 0;
    if (rows) {
        const GradRowsArgs& a = *rows;
        x.win = a.win;
        x.p = a.w; x.p_expert = a.w_expert; x.p_row = a.w_row;
        x.p_lines = (uintptr_t)a.w % 128 == 0 && a.w_expert % 64 == 0 && a.w_row % 64 == 0;
        x.q = a.grad_pre.base; x.q_expert = a.grad_pre.expert_stride; x.q_row = a.grad_pre.row_stride;
        x.out = a.grad_x.base; x.out_expert = a.grad_x.expert_stride; x.out_row = a.grad_x.row_stride;
        x.I = a.Kd; x.Kc = a.N;
        most_x = most_tiles(a.win, small_blocks(a.Kd), 0);
    }
    if (weights) {
        const GradWeightsArgs& a = *weights;
        w.win = a.win;
        w.p = a.x.base; w.p_expert = a.x.expert_stride; w.p_row = a.x.row_stride;
        w.q = a.grad_pre.base; w.q_expert = a.grad_pre.expert_stride; w.q_row = a.grad_pre.row_stride;
        w.out = (uint16_t*)a.grad_w; w.out_expert = a.gw_expert; w.out_row = a.gw_row;
        w.out_f32 = a.gw_f32; w.accumulate = a.accumulate;
        w.grad_b = a.grad_b; w.gb_stride = a.gb_stride;
        w.I = a.Kd; w.J = a.N;
        most_w = most_tiles(a.win, small_blocks(a.Kd), small_blocks(a.N));
    }
    if (!weights) return launch<GRAD_ROWS>(x, most_x, s);
    if (!rows) return launch<GRAD_WEIGHTS>(w, most_w, s);
    if (most_x + most_w <= 0) return hipSuccess;
    hipLaunchKernelGGL(gradients_kernel, dim3(product_grid(most_x + most_w)), dim3(64 * kWaves), kLds, s, x, w);
    return hipGetLastError();
}

hipError_t launch_act_backward(const ActBackwardArgs& a, hipStream_t s) {
    const int64_t most = most_blocks(a.win, kActRows);
    if (most <= 0) return hipSuccess;
    hipLaunchKernelGGL(act_backward_kernel, dim3((uint32_t)std::min<int64_t>(most, 8 * (int64_t)compute_units())), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace ep
