// Attention of a step's new tokens over the cache and, masked, over one another (sm_100a).
//
// Token i of sequence b sees the cached positions [begin, len) and the new tokens j, at positions len + j, whose bit its mask
// row has.  For a KV head the new tokens' queries, G per token, are the rows of a matrix Q; over the sequence's tokens
//     S = Q K^T,   m = row max of scale S,   P = e^{scale S - m},   l = row sum of P,   O = P V,   out = O / l,   lse = m + ln l
// with S = -inf where a token is not seen.  K and V are read once for up to 256 rows: below about 120 rows a KV head their stream
// from HBM is the bound at the measured rates, above that the tensor cores.
//
// Both products run on tcgen05.mma with accumulators in tensor memory, tiles of 128 tokens in two STREAMS per CTA, each with four
// softmax warps.  P is rounded to the inputs' type: a weight is off by at most half a step, as the result itself is; l is the sum
// of the unrounded weights.  With fp16 a half step is 2^-11 of a weight only down to 2^-14, and 2^-25 below, so its weights are
// 2^7 times as large (up to 2^15, since a reference may lie 2^8 below the maximum): 2^-11 of themselves or 2^-32 of the largest.
// Two forms:
//   many rows (ROWS = 0)   the rows are the products' M: S = Q K^T is 128 x 128, a thread owns a row, P goes back to tensor memory
//           as the A operand of P V.  A UNIT is (sequence, KV head, whole new tokens with up to 256 rows): wide, more than 128
//           rows, where the streams take 128 rows each and share every K and V tile; or narrow, up to 128 rows, where the streams
//           take alternate tiles.
//   few rows (ROWS = 16, 32: the most of a unit)   the tokens are M: S^T = K Q^T is 128 x ROWS, a thread owns a token, so the
//           exponentials are ROWS a tile and thread instead of 128 whatever the number of rows; P^T goes to shared memory as the
//           B operand of O^T = V^T P^T.  All units are narrow.
// A narrow unit's streams are joined at its end, both in the lanes of tensor memory that the same row (component) has in either.
//
// Work is dealt by cost: the units' tiles stand in a row, and each of the persistent CTAs (one per SM) takes an equal stretch of
// it.  So long and short sequences balance by themselves; a CTA finishes the units that lie wholly in its stretch, the host's
// partials included, and leaves softmax partials of the at most two that its ends cut, which tree_merge_kernel joins.
//
// Roles: warps 0-7 softmax and (many rows) epilogue; 8 and 9 load K and V tiles (TMA, a ring each; one warp for both would leave
// free slots waiting behind taken ones: 204 instead of 168 us at one new token, 8 sequences, 64/8 heads, 32 768 tokens); 10 issues
// the products; 11 finds the CTA's stretch, publishes its pieces up to four ahead and loads their queries (TMA, a box of G heads by
// whole tokens); 12-15 (few rows) finish the pieces while the softmax warps are at the next.  Every wait is bounded.
//
// The roles share the instruction cache, so what runs once a piece or less often is kept small (rolled loops, estimates in place of
// 64-bit quotients, one place that clears V rows).  Code of 107 KB became 88 (few rows) and 134 became 107: 128 sequences, 8 heads of
// 64, 2 new and up to 1500 tokens went from 62 to 83 us, by the run, to a steady 59; the last step, V rows cleared in one place, took
// 60 sequences, 40 heads, up to 48 new and 873 tokens from 207 to 190.
//
// Measured (K and V larger than the L2), us, in a loop / the floor at the measured rates: one new token, 8 sequences, 64/8 heads,
// 32 768 tokens: 169 / 167; the same with 64 components and twice the tokens: 166 / 167; 8 new tokens: 173 / 167, 16: 179 to 182 / 168
// (many rows); 32 and 131 072 tokens, one sequence: 133 to 163 / 84, by the power cap's clock (bound by the exponentials and products of
// a pair of tiles, some 3400 cycles where the products take 2048).  Short units cost more than their bytes (first tile, masked
// last tile, join, some 5000 cycles in all with many rows): 60 sequences, 40/40 heads, up to 873 tokens, up to 32, 48 and 200 new
// ones: 162 / 85, 187 to 190 / 88 and 329 / 115.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "hg_device.cuh"
#include "hg_partial.cuh"
#include "hg_tcgen05.cuh"

namespace hg {

constexpr int TREE_TILE = 128;                // tokens per tile, rows per stream
template <int ROWS> __host__ __device__ constexpr int tree_threads() { return ROWS ? 512 : 384; }
constexpr int TREE_K_WARP = 8, TREE_V_WARP = 9, TREE_MMA_WARP = 10, TREE_ITEM_WARP = 11, TREE_END_WARP = 12;
// registers of the softmax warps and of the others: together the 384 x 168 (many rows) or 512 x 128 (few rows) of the launch
template <int ROWS> __host__ __device__ constexpr int tree_regs_softmax() { return ROWS ? 160 : 200; }
constexpr int TREE_REGS_OTHER = 96;
constexpr int TREE_ITEMS = 4;                 // pieces published ahead
// Costs for the dealing: a tile, and a unit on top of its tiles (start, first tile, end).  Measured at 2, 4, 6, 8, 12 and 16 tiles a
// unit: 16 sequences, 56 heads, 5 new tokens, up to 16 384 tokens: 310 (2), 285 us (from 4 on); 48 sequences, 32/8 heads, up to
// 32 and 16 384: 299 (2 to 6), 302, 305, 309; 128 sequences, 8 heads of 64, 2 and 1 500: 70, 62, 63, 63, 65, 64.
constexpr int TREE_COST_TILE = 4, TREE_COST_UNIT = 16;
constexpr int TREE_MIN_STRETCH = 8;

// Powers of two on the weights: what fp16 has room for above the 2^8 by which a logit may pass its reference.
constexpr float TREE_PAST = 8.f;
template <bool BF16> __host__ __device__ constexpr float tree_lift() { return BF16 ? 0.f : 7.f; }

template <int D> __host__ __device__ constexpr int tree_tile_bytes() { return TREE_TILE * D * 2; }
// Ring slots for K and V tiles: what shared memory has room for.  K and V have rings of their own: the S products run ahead of the
// P V products, so that in a common ring a slot's use before the last might be unfinished when its next one is waited for, and a
// barrier's parity does not tell the two apart.
template <int D, int ROWS> __host__ __device__ constexpr int tree_k_slots() { return D == 64 ? 6 : ROWS ? 3 : 2; }
template <int D, int ROWS> __host__ __device__ constexpr int tree_v_slots() { return D == 128 ? 3 : 6; }
// Queries of a stream (two buffers), weights of a stream (two buffers; many rows have them in tensor memory).
template <int D, int ROWS> __host__ __device__ constexpr int tree_q_bytes() { return (ROWS ? ROWS : TREE_TILE) * D * 2; }
template <int ROWS> __host__ __device__ constexpr int tree_p_bytes() { return ROWS * TREE_TILE * 2; }

struct TreeSources {
    const float* o[HG_MAX_MERGE_SRC];
    const float* m[HG_MAX_MERGE_SRC];
    const float* l[HG_MAX_MERGE_SRC];
    int nc[HG_MAX_MERGE_SRC];
    int n;
};

// A cut unit, as the CTA with its first tile leaves it for the merge: its partials are in slot 2 c + 1 of that CTA c and in slots
// 2 c' of the CTAs behind it up to `last`, as far as these say that they have one.
struct TreeCut { int row0, nodes, h, last; };
struct TreeWorkspace {
    TreeCut* cut;                    // [CTAs]
    int32_t* valid;                  // [2 CTAs]
    float* o;                        // [2 CTAs][256][D]
    float* m;                        // [2 CTAs][256]
    float* l;
};

struct TreeParams {
    const int32_t* block_table;      // [B][max_pages], or NULL: identity paging
    const uint16_t* v;               // (for the look at single rows)
    int64_t page_stride, head_stride, tok_stride;
    const int32_t* seq_lens;
    const int32_t* tok_begin;        // or NULL
    const int32_t* cu;
    const uint32_t* mask;            // or NULL: chains
    uint16_t* out;
    float* lse;
    int32_t* status;
    TreeWorkspace ws;
    TreeSources src;
    int B, Hq, Hkv, G, N, max_nodes, words;
    int nodes;                       // new tokens of a stream's rows: 128 (ROWS) / G
    int page_size, page_shift, max_pages, num_pages;
    int reread, test_stall;          // reread: several units of a KV head read the same tiles
    float scale, scale_log2;
    FastDiv div_G, div_wide;         // of G, of 2 nodes
    uint64_t inv_ctas;               // 2^64 / CTAs, rounded up
};

// What a sequence has to do.
struct TreeSeq { int row0, n, len, lo, hi, tiles, wides, narrow; bool bad; };

__device__ __forceinline__ TreeSeq tree_seq(const TreeParams& p, int b) {
    TreeSeq s;
    s.row0 = p.cu[b];
    const int next = p.cu[b + 1];
    s.bad = next > s.row0 && (s.row0 < 0 || next > p.N || next - s.row0 > p.max_nodes);
    s.n = s.row0 < 0 || next <= s.row0 ? 0 : max(0, min(min(next, p.N) - s.row0, p.max_nodes));
    s.len = max(p.seq_lens[b], 0);
    const long long room = (long long)p.max_pages << p.page_shift, end = (long long)s.len + s.n;
    s.lo = (int)min((long long)min(max(p.tok_begin ? p.tok_begin[b] : 0, 0), s.len), room);
    s.hi = (int)min(end, room);
    if (s.n > 0 && end > room) s.bad = true;
    s.tiles = s.hi > s.lo ? (s.hi - (s.lo & ~(TREE_TILE - 1)) + TREE_TILE - 1) / TREE_TILE : 1;     // (none at all: one that shows nothing)
    s.wides = fast_div(s.n, p.div_wide);
    const int rest = s.n - s.wides * 2 * p.nodes;
    s.wides += rest > p.nodes ? 1 : 0;
    s.narrow = rest > 0 && rest <= p.nodes ? rest : 0;
    return s;
}
__device__ __forceinline__ long long tree_cost(const TreeSeq& s) { return TREE_COST_UNIT + (long long)s.tiles * TREE_COST_TILE; }   // of a unit
__device__ __forceinline__ long long tree_head_cost(const TreeSeq& s) { return (s.wides + (s.narrow ? 1 : 0)) * tree_cost(s); }
// Quotients below 2^17 (heads, units of a head): an estimate in floats is off by one at most (it has 2^-21 of itself).
__device__ __forceinline__ int tree_div(long long a, long long b) {
    const int q = (int)__fdividef((float)a, (float)b);
    return q * b > a ? q - 1 : (q + 1) * b <= a ? q + 1 : q;
}
// Where the stretch of CTA c of n begins: floor(total c / n).  For all CTAs of the launch by a product (inv_ctas = 2^64 / CTAs
// rounded up: exact below 2^56); with fewer CTAs there is less than TREE_MIN_STRETCH a CTA.
__device__ __forceinline__ long long tree_stretch(const TreeParams& p, long long total, int c, int n) {
    if (n == (int)gridDim.x) return (long long)__umul64hi((unsigned long long)total * (unsigned)c, p.inv_ctas);
    return (long long)((uint32_t)total * (uint32_t)c / (uint32_t)n);
}
// How many CTAs share the work: where there is little, stretches have a tile for each stream.
__device__ __forceinline__ int tree_ctas(long long total) {
    return total >= (long long)TREE_MIN_STRETCH * gridDim.x ? (int)gridDim.x : max(1, (int)total / TREE_MIN_STRETCH);
}
// The CTA that a place belongs to.
__device__ __forceinline__ int tree_cta_of(const TreeParams& p, long long place, long long total, int n) {
    int c = min(n - 1, (int)__fdividef((float)place * (float)n, (float)total));
#pragma unroll 1
    while (c > 0 && tree_stretch(p, total, c, n) > place) --c;
#pragma unroll 1
    while (c + 1 < n && tree_stretch(p, total, c + 1, n) <= place) ++c;
    return c;
}
// A unit's tile t stands at TREE_COST_UNIT + t * TREE_COST_TILE behind the unit's begin; how many stand in front of a place in it.
__device__ __forceinline__ int tree_tiles_before(int place, int tiles) {
    const int x = place - TREE_COST_UNIT;
    return x <= 0 ? 0 : min(tiles, (x + TREE_COST_TILE - 1) / TREE_COST_TILE);
}

// Which new tokens 32 w .. 32 w + 31 token i (packed row `row`) sees.
__device__ __forceinline__ uint32_t tree_word(const TreeParams& p, int row, int i, int w) {
    if (p.mask) return w < p.words ? p.mask[(size_t)row * p.words + w] : 0u;
    const int last = i - w * 32;
    return last >= 31 ? ~0u : last < 0 ? 0u : (2u << last) - 1u;
}

// A piece of a unit, published by the item warp.
struct TreeItem {
    int valid;                       // 0: no more of them
    int b, h, wide;
    int row0, i0, nodes;             // packed row and number of its first new token, how many
    int n, len, lo, hi;              // the sequence's new tokens, position of the first, tokens in the pool
    int first, tiles;                // first token of the first tile, tiles
    int whole, slot;                 // all of the unit's tiles, else where the partials go
    int q;                           // buffer of the queries (wide: both)
};

template <int D, int ROWS>
struct TreeCtl {
    static constexpr int S = tree_k_slots<D, ROWS>() + tree_v_slots<D, ROWS>();
    uint64_t full[S], empty[S];      // K slots, then V slots
    uint64_t s_full[2], s_read[2], p_free[2], p_full[2][ROWS ? 1 : 4];   // p_full: (many rows) the quarters of a tile's tokens
    uint64_t o_full[2][2];           // per stream, with few rows for even and odd pieces
    uint64_t q_full[2], q_free[2], drain;
    uint64_t join_sync[ROWS ? 1 : 4];        // (many rows) the two warps that join 32 rows of a narrow unit's streams
    uint64_t vote[2];                // (few rows) a stream's warps
    uint64_t sums_full, sums_free, o_free[2];      // (few rows) the pieces' way to the warps that finish them
    uint64_t item_full[TREE_ITEMS], item_empty[TREE_ITEMS];
    TreeItem item[TREE_ITEMS];
    int poisoned[TREE_ITEMS];        // something in the V rows of the item's new tokens is not finite
    uint32_t tmem;
    int abort;
    uint8_t bad[16];                 // per tile, in load order: 16-token pieces of the tile whose page was refused
    uint8_t stream_bad[2];           // the same for the tile a stream's softmax warps are about to read
    int moved[3][2];                 // (few rows) in turns: the last tile, counted, in which a stream's references had to move
    // many rows: per stream, rows' reference and sum.  Few rows: per stream, rows' references as the exponents' summand, and, in
    // turns, the maxima of a tile as ordered integers
    union __align__(16) {
        float2 join[2][ROWS ? 1 : TREE_TILE];
        struct {
            float off[2][ROWS ? ROWS : 1];
            uint32_t top[3][2][ROWS ? ROWS : 1];
            float sums[2][4][ROWS ? ROWS : 1], ref[2][ROWS ? ROWS : 1];      // of a piece: per stream and warp, and references
        } col;
    };
    long long part[4];
    long long start_base;
    int start_b;
    int left[TREE_ITEMS];            // (few rows) products of S still to issue, by item
    int issued[2], q_issued[2];      // tiles of K and V, and items' queries by buffer, that were requested (for the unwinding)
};

template <int D, int ROWS> constexpr size_t tree_smem_bytes() {
    return (size_t)TreeCtl<D, ROWS>::S * tree_tile_bytes<D>() + 2 * tree_q_bytes<D, ROWS>() + 2 * tree_p_bytes<ROWS>() + sizeof(TreeCtl<D, ROWS>);
}

// Tiles of a stream; number of its tile i in load order.
__device__ __forceinline__ int tree_stream_tiles(const TreeItem& it, int s) { return it.wide ? it.tiles : (it.tiles + 1 - s) / 2; }
__device__ __forceinline__ int tree_tile_index(const TreeItem& it, int s, int i) { return it.wide ? i : 2 * i + s; }

// Eight 16-bit numbers: bits 15 or 31 of the result tell that one of them is not finite (all exponent bits set).
template <bool BF16>
__device__ __forceinline__ uint32_t not_finite(uint4 x) {
    constexpr uint32_t ONE = BF16 ? 0x00800080u : 0x04000400u;     // carries out of the exponent exactly then
    return ((x.x & 0x7fff7fffu) + ONE) | ((x.y & 0x7fff7fffu) + ONE) | ((x.z & 0x7fff7fffu) + ONE) | ((x.w & 0x7fff7fffu) + ONE);
}

// Whether a row sees a new token, among the piece's, with something in its V row that is not finite.  (Looked at only where one
// has been met.)
template <int D, bool BF16>
__device__ __forceinline__ bool tree_poisoned(const TreeParams& p, const TreeItem& it, int row, int node) {
    const int first = max(it.first - it.len, 0), last = min(min(it.hi, it.first + it.tiles * TREE_TILE) - it.len, it.n);
#pragma unroll 1
    for (int j = first; j < last; ++j) {
        if (!((tree_word(p, row, node, j >> 5) >> (j & 31)) & 1u)) continue;
        const int t = it.len + j;
        const size_t e = (size_t)it.b * p.max_pages + (t >> p.page_shift);
        const long long page = p.block_table ? p.block_table[e] : (long long)e;
        if (page < 0 || page >= p.num_pages) continue;
        const uint4* const v = reinterpret_cast<const uint4*>(p.v + page * p.page_stride + it.h * p.head_stride + (t & (p.page_size - 1)) * p.tok_stride);
#pragma unroll 1
        for (int c = 0; c < D / 8; ++c)
            if (not_finite<BF16>(v[c]) & 0x80008000u) return true;
    }
    return false;
}

// Floats as integers of the same order (NaN aside); 0 is below all of them.
__device__ __forceinline__ uint32_t ordered(float x) {
    const uint32_t u = __float_as_uint(x);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t u) { return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u); }

// N values a lane, over the lanes that differ in the bits of N - 1: lane i gets the maximum (sum) of value i mod N.
template <int N, bool MAX>
__device__ __forceinline__ float lanes_fold(const float* x, int lane) {
    if constexpr (N == 1) return x[0];
    else {
        constexpr int H = N / 2;
        float v[H];
        const bool up = lane & H;
#pragma unroll
        for (int i = 0; i < H; ++i) {
            const float keep = up ? x[i + H] : x[i], give = up ? x[i] : x[i + H], got = __shfl_xor_sync(0xffffffffu, give, H);
            v[i] = MAX ? fmaxf(keep, got) : keep + got;
        }
        return lanes_fold<H, MAX>(v, lane);
    }
}
// ... over all 32 lanes.
template <int N, bool MAX>
__device__ __forceinline__ float across_lanes(const float* x, int lane) {
    float r = lanes_fold<N, MAX>(x, lane);
    if constexpr (N == 16) {
        const float got = __shfl_xor_sync(0xffffffffu, r, 16);
        r = MAX ? fmaxf(r, got) : r + got;
    }
    return r;
}

// What the host's partials make of a row's own (m, l): the maximum of all, the sum of weights.  Returns the factor on the row's own.
__device__ __forceinline__ float tree_join_host(const TreeParams& p, size_t orow, float m, float& l, float& top) {
    constexpr float LOG2E = 1.4426950408889634f;
    const float none = __int_as_float(0xff800000);
    top = m;
    if (p.src.n == 0) return 1.f;
#pragma unroll 1
    for (int x = 0; x < p.src.n; ++x)
#pragma unroll 1
        for (int c = 0; c < p.src.nc[x]; ++c) top = fmaxf(top, p.src.m[x][orow * p.src.nc[x] + c]);
    const float own = m == none ? 0.f : fast_exp2((m - top) * LOG2E);
    l *= own;
#pragma unroll 1
    for (int x = 0; x < p.src.n; ++x)
#pragma unroll 1
        for (int c = 0; c < p.src.nc[x]; ++c) {
            const float hm = p.src.m[x][orow * p.src.nc[x] + c];
            if (hm != none) l += p.src.l[x][orow * p.src.nc[x] + c] * fast_exp2((hm - top) * LOG2E);
        }
    return own;
}

template <int D, bool BF16, int ROWS>
__global__ void __launch_bounds__(tree_threads<ROWS>(), 1) tree_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                                                               const __grid_constant__ CUtensorMap tmV, const __grid_constant__ TreeParams p) {
    constexpr bool FEW = ROWS > 0;
    constexpr int KS = tree_k_slots<D, ROWS>(), VS = tree_v_slots<D, ROWS>(), S = KS + VS;
    constexpr int TILE_BYTES = tree_tile_bytes<D>(), Q_BYTES = tree_q_bytes<D, ROWS>(), P_BYTES = tree_p_bytes<ROWS>();
    constexpr int HALVES = D / 64;
    constexpr uint32_t HALF_BYTES = TREE_TILE * 128, Q_HALF_BYTES = Q_BYTES / HALVES;
    constexpr uint32_t FMT = BF16 ? 1u : 0u;
    // weights are 2^LIFT e^(scale (logit - reference)): as softmax statistics, sums that refer to LIFT ln 2 below the reference
    constexpr float LIFT = tree_lift<BF16>(), LIFT_LN = LIFT * 0.693147180559945309f;
    // instruction descriptors: fp32 accumulator, 16-bit A and B.  Many rows: M = 128; S: both K-major, N = 128 tokens; O: B (V)
    // with its components contiguous (N-major), N = D.  Few rows: S^T: both K-major, M = 128 tokens, N = ROWS; O^T: A (V) with its
    // components contiguous (M-major), M = D, and B (P) with a token's rows contiguous (N-major)
    constexpr uint32_t IDESC = (1u << 4) | (FMT << 7) | (FMT << 10);
    constexpr uint32_t IDESC_S = IDESC | (((FEW ? (uint32_t)ROWS : 128u) >> 3) << 17) | ((128u >> 4) << 24);
    constexpr uint32_t IDESC_O = FEW ? IDESC | (1u << 15) | (1u << 16) | (((uint32_t)ROWS >> 3) << 17) | (((uint32_t)D >> 4) << 24)
                                     : IDESC | (1u << 16) | (((uint32_t)D >> 3) << 17) | ((128u >> 4) << 24);
    // many rows with 128 components fill tensor memory, and P takes the place of half of S; else P lies beside S, and the next S is
    // computed while the weights of this one are
    constexpr bool BESIDE = FEW || D == 64;
    constexpr uint32_t S_STRIDE = FEW ? ROWS : 128, O_COL = 2 * S_STRIDE, O_STRIDE = FEW ? ROWS : D;
    constexpr uint32_t P_COL = BESIDE ? 384 : 0, P_STRIDE = BESIDE ? 64 : 128;     // (many rows)
    constexpr uint32_t TMEM_COLS = FEW ? 8 * ROWS : 512;           // (few rows: S, and O for even and odd pieces, 6 * ROWS of them)
    const float NEG_INF = __int_as_float(0xff800000);

    extern __shared__ __align__(1024) uint8_t tree_raw[];
    uint8_t* const q_smem = tree_raw;
    uint8_t* const p_smem = tree_raw + 2 * Q_BYTES;
    uint8_t* const ring = p_smem + 2 * P_BYTES;
    TreeCtl<D, ROWS>& ctl = *reinterpret_cast<TreeCtl<D, ROWS>*>(ring + S * TILE_BYTES);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    volatile int* const abort_flag = &ctl.abort;

    if (tid == 0) {
        prefetch_tensormap(&tmQ);
        prefetch_tensormap(&tmK);
        prefetch_tensormap(&tmV);
        for (int i = 0; i < S; ++i) { mbar_init(&ctl.full[i], 1); mbar_init(&ctl.empty[i], 1); }
        for (int s = 0; s < 2; ++s) {
            mbar_init(&ctl.s_full[s], 2);                          // the products' completion, and the tile's description
            mbar_init(&ctl.s_read[s], 4);
            mbar_init(&ctl.p_free[s], 1);
            for (int c = 0; c < (FEW ? 1 : 4); ++c) mbar_init(&ctl.p_full[s][c], 4);
            mbar_init(&ctl.o_full[s][0], 1);
            mbar_init(&ctl.o_full[s][1], 1);
            mbar_init(&ctl.o_free[s], 4);
            mbar_init(&ctl.q_full[s], 1);
            mbar_init(&ctl.q_free[s], 1);
            mbar_init(&ctl.vote[s], 4);
        }
        for (int i = 0; i < TREE_ITEMS; ++i) { mbar_init(&ctl.item_full[i], 1); mbar_init(&ctl.item_empty[i], FEW ? 8 + 3 + 4 : 8 + 3); }
        for (int i = 0; i < (FEW ? 1 : 4); ++i) mbar_init(&ctl.join_sync[i], 2);
        mbar_init(&ctl.sums_full, 8);
        mbar_init(&ctl.sums_free, 4);
        mbar_init(&ctl.drain, 1);
        ctl.abort = 0;
        fence_barrier_init();
    }
    if (FEW)
        for (int i = tid; i < 6 * (FEW ? ROWS : 1); i += tree_threads<ROWS>()) (&ctl.col.top[0][0][0])[i] = 0;
    if (tid < 6) (&ctl.moved[0][0])[tid] = 0;
    if (warp == TREE_MMA_WARP) {
        tmem_alloc(&ctl.tmem, TMEM_COLS);
        tmem_relinquish();
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(&ctl.tmem);

    int issued = 0;                                                // (loader) tiles requested so far
    uint32_t q_armed[2] = {0, 0};                                  // (item warp) queries requested, by barrier
    cudaTriggerProgrammaticLaunchCompletion();
    auto timed_out = [&]() { return p.status && (*reinterpret_cast<volatile int32_t*>(p.status) & HG_DEV_WAIT_TIMEOUT); };
    if (warp >= 8 && warp < TREE_END_WARP) {
      reg_shrink<TREE_REGS_OTHER>();
      cudaGridDependencySynchronize();
      const int me = tid - 256, cta = blockIdx.x;
      long long total = 0;
      if (p.B > 32) {
          // ---- the sequences' costs, and where this CTA's stretch begins: 128 threads, a run of sequences each.  (The item warp
          // alone does it where its lanes have room for all sequences) ----
          if (me == 3) ctl.start_b = -1;
          const int run = (p.B + 127) / 128, b_first = min(p.B, me * run), b_last = min(p.B, b_first + run);
          long long mine = 0;
          bool trouble = false;
#pragma unroll 1
          for (int b = b_first; b < b_last; ++b) {
              const TreeSeq s = tree_seq(p, b);
              mine += tree_head_cost(s) * p.Hkv;
              trouble = trouble || s.bad;
          }
          if (trouble && cta == 0 && p.status) atomicOr(p.status, HG_DEV_RANGE);
          long long upto = mine;
#pragma unroll
          for (int o = 1; o < 32; o <<= 1) {
              const long long y = __shfl_up_sync(0xffffffffu, upto, o);
              if (lane >= o) upto += y;
          }
          if (lane == 31) ctl.part[warp - 8] = upto;
          asm volatile("bar.sync 1, 128;" ::: "memory");
          for (int w = 0; w < 4; ++w) {
              if (w < warp - 8) upto += ctl.part[w];
              total += ctl.part[w];
          }
          const int n = tree_ctas(total);
          const long long from = cta < n ? tree_stretch(p, total, cta, n) : total;
          if (from >= upto - mine && from < upto) {
              long long base = upto - mine;
#pragma unroll 1
              for (int b = b_first; b < b_last; ++b) {
                  const long long cost = tree_head_cost(tree_seq(p, b)) * p.Hkv;
                  if (from < base + cost) { ctl.start_b = b; ctl.start_base = base; break; }
                  base += cost;
              }
          }
          asm volatile("bar.sync 1, 128;" ::: "memory");
      }
      if (warp == TREE_ITEM_WARP) {
        // =============================== item warp: the stretch's pieces, some ahead, and their queries ===============================
        // (after an earlier call that ran into its limit there is no work until the caller has cleared the word)
        const bool skip = timed_out();
        // nothing is cut so far: cleared by the warp that sets these words for the pieces, so that its own order holds for both
        if (lane < 2) p.ws.valid[2 * cta + lane] = 0;
        if (lane == 2) p.ws.cut[cta].nodes = 0;
        __syncwarp();
        int ub = 0;                                                // first of the 32 sequences in the lanes
        long long base = 0;                                        // ... its place in the row of tiles
        if (p.B > 32) { ub = ctl.start_b < 0 ? p.B : ctl.start_b; base = ctl.start_base; }
        TreeSeq sq;
        long long cost = 0, before = 0, block = 0;
        auto load_sequences = [&]() {
            sq.n = 0;
            sq.bad = false;
            cost = 0;
            if (ub + lane < p.B) {
                sq = tree_seq(p, ub + lane);
                cost = tree_head_cost(sq) * p.Hkv;
            }
            long long x = cost;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const long long y = __shfl_up_sync(0xffffffffu, x, o);
                if (lane >= o) x += y;
            }
            before = x - cost;
            block = __shfl_sync(0xffffffffu, x, 31);
        };
        load_sequences();
        if (p.B <= 32) {
            total = block;
            if (sq.bad && cta == 0 && p.status) atomicOr(p.status, HG_DEV_RANGE);
        }
        const int sharing = tree_ctas(total);
        long long at = cta < sharing ? tree_stretch(p, total, cta, sharing) : total;       // place in the row of tiles
        const long long to = cta + 1 < sharing ? tree_stretch(p, total, cta + 1, sharing) : total;
        if (ub == p.B || skip) at = to;
        bool ok = true;
        int last_q = 1;
        uint32_t q_uses[2] = {0, 0};                               // of the buffers
        const int row_bytes = p.G * p.nodes * 128;                 // a query box
        for (int k = 0; ok; ++k) {
            TreeItem it;
            it.valid = 0;
            long long last_place = 0;
#pragma unroll 1
            while (at < to) {                                      // the next piece with a tile in it
#pragma unroll 1
                while (at >= base + block && ub < p.B) { base += block; ub += 32; load_sequences(); }
                if (ub >= p.B) { at = to; break; }
                const int src = __ffs(__ballot_sync(0xffffffffu, at >= base + before && at < base + before + cost)) - 1;
                TreeSeq s;
                s.row0 = __shfl_sync(0xffffffffu, sq.row0, src); s.n = __shfl_sync(0xffffffffu, sq.n, src);
                s.len = __shfl_sync(0xffffffffu, sq.len, src); s.lo = __shfl_sync(0xffffffffu, sq.lo, src);
                s.hi = __shfl_sync(0xffffffffu, sq.hi, src); s.tiles = __shfl_sync(0xffffffffu, sq.tiles, src);
                s.wides = __shfl_sync(0xffffffffu, sq.wides, src); s.narrow = __shfl_sync(0xffffffffu, sq.narrow, src);
                const long long begin = base + __shfl_sync(0xffffffffu, before, src);
                const long long head = tree_head_cost(s), unit_cost = tree_cost(s);
                const int h = tree_div(at - begin, head);
                const long long in_head = (at - begin) - head * h;
                const int u = s.wides == 0 ? 0 : tree_div(in_head, unit_cost);
                const bool is_wide = u < s.wides;
                const long long unit = begin + head * h + unit_cost * u;
                const int t0 = tree_tiles_before((int)(at - unit), s.tiles);
                const int t1 = to >= unit + unit_cost ? s.tiles : tree_tiles_before((int)(to - unit), s.tiles);
                at = min(to, unit + unit_cost);
                if (t0 >= t1) continue;
                it.valid = 1;
                it.b = ub + src; it.h = h; it.wide = is_wide;
                it.i0 = u * 2 * p.nodes;
                it.nodes = is_wide ? min(2 * p.nodes, s.n - it.i0) : s.narrow;
                it.row0 = s.row0 + it.i0;
                it.n = s.n; it.len = s.len; it.lo = s.lo; it.hi = s.hi;
                it.first = (s.lo & ~(TREE_TILE - 1)) + t0 * TREE_TILE;
                it.tiles = t1 - t0;
                it.whole = t0 == 0 && t1 == s.tiles;
                it.slot = 2 * cta + (t0 == 0 ? 1 : 0);
                it.q = is_wide ? 0 : last_q ^ 1;
                last_q = is_wide ? 1 : it.q;
                // (of the unit's last tile, for the merge)
                last_place = unit + TREE_COST_UNIT + (long long)(s.tiles - 1) * TREE_COST_TILE;
                break;
            }
            const int j = k % TREE_ITEMS;
            if (k >= TREE_ITEMS) ok = pfx_warp_wait(&ctl.item_empty[j], (uint32_t)(k / TREE_ITEMS - 1) & 1u, abort_flag);
            if (!ok) break;
            if (lane == 0) {
                ctl.item[j] = it;
                ctl.poisoned[j] = 0;
                mbar_arrive(&ctl.item_full[j]);
            }
            __syncwarp();
            if (!it.valid) break;
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                if (!it.wide && x != it.q) continue;
                if (ok && q_uses[x] > 0) ok = pfx_warp_wait(&ctl.q_free[x], (q_uses[x] - 1) & 1u, abort_flag);
                ++q_uses[x];
            }
            if (!ok) break;
            if (lane == 0) {                                       // (wide: both buffers, on the first one's barrier)
                const int boxes = HALVES * (it.wide ? 2 : 1);
                mbar_arrive_expect_tx(&ctl.q_full[it.q], (uint32_t)(boxes * row_bytes));
#pragma unroll 1
                for (int x = 0; x < boxes; ++x) {
                    const int s = x / HALVES, half = x % HALVES;
                    tma_load_3d(q_smem + (it.q + s) * Q_BYTES + half * Q_HALF_BYTES, &tmQ, &ctl.q_full[it.q], half * 64, it.h * p.G, it.row0 + s * p.nodes);
                }
            }
            if (it.q) ++q_armed[1]; else ++q_armed[0];
            if (!it.whole && lane == 0) {
                p.ws.valid[it.slot] = 1;
                if (it.slot & 1) *reinterpret_cast<int4*>(&p.ws.cut[cta]) = make_int4(it.row0, it.nodes, it.h, tree_cta_of(p, last_place, total, sharing));
            }
        }
      } else if (warp == TREE_K_WARP || warp == TREE_V_WARP) {
        // =============================== loaders of K tiles and of V tiles ===============================
        const bool is_k = warp == TREE_K_WARP;
        const CUtensorMap* const tm = is_k ? &tmK : &tmV;
        const uint64_t policy = p.reread ? l2_evict_normal_policy() : l2_evict_first_policy();
        const int box_rows = min(p.page_size, TREE_TILE), boxes = TREE_TILE / box_rows * HALVES;
        const int piece = lane / HALVES, half = lane % HALVES;     // this lane's box: a page (or part of one) and a half
        bool ok = true;
        int n = 0;                                                 // tiles of earlier items
        // block-table entries of 32 pages in the lanes, from page `from` on of a row whose tokens are [lo, hi)
        auto look_up = [&](int b, int lo, int hi, int from) {
            const int pg = from + lane;
            if (pg > (hi - 1) >> p.page_shift || pg < lo >> p.page_shift || hi <= lo) return -1;
            const long long e = (long long)b * p.max_pages + pg;
            return p.block_table ? p.block_table[e] : (int)e;
        };
        // those at the beginning of the item behind this one are requested as soon as it is published: a unit of a few tiles would
        // wait for them as long as it takes
        int ahead = 0;
        bool looked = false;
        for (int k = 0; ok; ++k) {
            const int j = k % TREE_ITEMS;
            ok = pfx_warp_wait(&ctl.item_full[j], (uint32_t)(k / TREE_ITEMS) & 1u, abort_flag);
            if (!ok) break;
            const TreeItem it = ctl.item[j];
            if (!it.valid) break;
            const int page0 = it.first >> p.page_shift, pages = p.page_size < TREE_TILE ? TREE_TILE >> p.page_shift : 1;
            // (a tile's pages never straddle the 32 in the lanes and the next 32)
            int base = page0, now = looked ? ahead : look_up(it.b, it.lo, it.hi, base), next = look_up(it.b, it.lo, it.hi, base + 32);
            looked = false;
#pragma unroll 1
            for (int x = 0; x < it.tiles; ++x) {
                const int t_x = it.first + x * TREE_TILE, t_box = t_x + piece * box_rows, row = t_box & (p.page_size - 1);
                if ((t_x >> p.page_shift) + pages > base + 32) {
                    base += 32;
                    now = next;
                    next = look_up(it.b, it.lo, it.hi, base + 32);
                }
                const int entry = __shfl_sync(0xffffffffu, now, (t_box >> p.page_shift) - base);
                const bool want = lane < boxes && t_box < it.hi && t_box + box_rows > it.lo;
                const int e = !want ? -1 : ((uint32_t)entry < (uint32_t)p.num_pages ? entry : -2);      // -1: not wanted, -2: refused
                const int y = n + x, use = is_k ? y / KS : y / VS, slot = is_k ? y % KS : KS + y % VS;
                const uint32_t bytes = (uint32_t)__popc(__ballot_sync(0xffffffffu, e >= 0)) * (uint32_t)box_rows * 128u;
                uint32_t bad = 0;
                if (is_k && __any_sync(0xffffffffu, e == -2)) {
                    if (e == -2) {
                        bad = ((1u << (box_rows >> 4)) - 1u) << (piece * (box_rows >> 4));
                        if (p.status) atomicOr(p.status, HG_DEV_BAD_PAGE);
                    }
                    bad = __reduce_or_sync(0xffffffffu, bad);
                }
                if (use > 0) ok = pfx_warp_wait(&ctl.empty[slot], (uint32_t)(use - 1) & 1u, abort_flag);
                if (!ok || p.test_stall) break;
                if (lane == 0) {
                    if (is_k) ctl.bad[(n + x) & 15] = (uint8_t)bad;
                    mbar_arrive_expect_tx(&ctl.full[slot], bytes);
                }
                __syncwarp();
                if (e >= 0) tma_load_5d(ring + slot * TILE_BYTES + half * HALF_BYTES + piece * box_rows * 128, tm, &ctl.full[slot], 0, row, half, it.h, e, policy);
                issued = n + x + 1;
                const int j1 = (k + 1) % TREE_ITEMS;
                if (!looked && __all_sync(0xffffffffu, mbar_test(&ctl.item_full[j1], (uint32_t)((k + 1) / TREE_ITEMS) & 1u))) {
                    const TreeItem& it1 = ctl.item[j1];
                    if (it1.valid) ahead = look_up(it1.b, it1.lo, it1.hi, it1.first >> p.page_shift);
                    looked = true;
                }
            }
            n += it.tiles;
            __syncwarp();
            if (lane == 0) mbar_arrive(&ctl.item_empty[j]);
            if (p.test_stall) break;
        }
      } else {
        // =============================== tensor-core warp: one thread issues all products ===============================
        if constexpr (FEW) {
          if (elect_one()) {
            // Few rows: whatever is ready next, looked for in turn.  Each stream goes from tile to tile and from item to item without
            // a stop: S^T as soon as K and Q are there and the S before is read, at most two tiles ahead of O^T, which needs P and V
            struct Stream {
                int k, i, tiles, total, base;      // next to score: item, tile; the item's tiles of this stream and of both, its first tile
                bool loaded, end;
                uint32_t scored, valued;           // tiles so far
                int x0, x1;                        // the tiles scored and not valued (even and odd ones): number in load order,
                uint32_t about0, about1;           // and bit 0: first of its item, 1: last, from 2 on the item
            };
            Stream st0 = {0, 0, 0, 0, 0, false, false, 0, 0, 0, 0, 0, 0}, st1 = st0;
            uint32_t seen = 0;                                     // items loaded by one stream (bits)
            const uint64_t q_desc = tc_smem_desc(smem_u32(q_smem), 16u, 1024u, 2u), k_desc = tc_smem_desc(smem_u32(ring), 16u, 1024u, 2u);
            const uint64_t v_desc = tc_smem_desc(smem_u32(ring), HALF_BYTES, 1024u, 2u);
            const uint64_t p_desc = tc_smem_desc(smem_u32(p_smem), 128u, 2048u, 0u);       // 8 tokens 128 bytes apart, 8 rows 2048
            // A barrier's phase is looked at only when the one before is known to be over: a ring slot's use before last may be the
            // other stream's, so a stream is never a whole ring ahead of the other
            auto step = [&](auto which) -> bool {                  // one product of a stream, if there is one to issue
                constexpr int s = decltype(which)::value;
                Stream& t = s ? st1 : st0;
                const Stream& u = s ? st0 : st1;
                const int u_score = u.end ? 0x7fffffff : u.loaded ? u.base + 2 * u.i + (1 - s) : u.base;     // the other's next tiles
                const int u_value = u.valued == u.scored ? u_score : u.valued & 1 ? u.x1 : u.x0;
                if (t.valued != t.scored) {                        // O^T += V^T P^T
                    const int x = t.valued & 1 ? t.x1 : t.x0, slot = KS + x % VS;
                    const uint32_t about = t.valued & 1 ? t.about1 : t.about0;
                    const int item = (int)(about >> 2);
                    if (x - u_value < VS && mbar_test(&ctl.p_full[s][0], t.valued & 1u) && mbar_test(&ctl.full[slot], (uint32_t)(x / VS) & 1u) &&
                        (!(about & 1u) || item < 2 || mbar_test(&ctl.o_free[item & 1], (uint32_t)(item / 2 - 1) & 1u))) {
                        tc_fence_after_sync();
                        const uint64_t v = v_desc + (uint32_t)(slot * (TILE_BYTES >> 4)), w = p_desc + (uint32_t)(s * (P_BYTES >> 4));
                        const uint32_t acc = tmem + O_COL + ((item & 1) * 2 + s) * O_STRIDE;
#pragma unroll
                        for (int kk = 0; kk < 8; ++kk)             // 16 tokens
                            tc_mma_f16_ss(acc, v + (uint32_t)(kk * 2048 >> 4), w + (uint32_t)(kk * 256 >> 4), IDESC_O, kk || !(about & 1u) ? 1u : 0u);
                        tc_commit(&ctl.empty[slot]);
                        tc_commit(&ctl.p_free[s]);
                        if (about & 2u) tc_commit(&ctl.o_full[s][item & 1]);
                        ++t.valued;
                        return true;
                    }
                }
                while (!t.loaded && !t.end) {                      // the next item with a tile for this stream, if it is published
                    const int j = t.k % TREE_ITEMS;
                    if (!mbar_test(&ctl.item_full[j], (uint32_t)(t.k / TREE_ITEMS) & 1u)) break;
                    const volatile TreeItem& it = ctl.item[j];
                    if (!it.valid) { t.end = true; break; }
                    t.total = it.tiles;
                    t.tiles = (t.total + 1 - s) / 2;
                    t.i = 0;
                    if ((seen >> j) & 1u) mbar_arrive(&ctl.item_empty[j]);       // both streams have it
                    else ctl.left[j] = t.total;
                    seen ^= 1u << j;
                    if (t.tiles > 0) t.loaded = true;
                    else { t.base += t.total; ++t.k; }
                }
                if (!t.loaded || t.scored - t.valued >= 2) return false;
                const int x = t.base + 2 * t.i + s, slot = x % KS, j = t.k % TREE_ITEMS;
                // (x against u_value: the softmax warps may look at the tile's V slot)
                if (x - u_score >= KS || x - u_value >= VS || (t.scored > 0 && !mbar_test(&ctl.s_read[s], (t.scored - 1) & 1u)) ||
                    !mbar_test(&ctl.full[slot], (uint32_t)(x / KS) & 1u)) return false;
                // (items take the two Q buffers in turn; the one before last is over when the other stream is at most one behind)
                if (t.i == 0 && ((!u.end && t.k - u.k >= 2) || !mbar_test(&ctl.q_full[t.k & 1], (uint32_t)(t.k / 2) & 1u))) return false;
                ctl.stream_bad[s] = ctl.bad[x & 15];               // S^T = K Q^T
                tc_fence_after_sync();
                const uint64_t kd = k_desc + (uint32_t)(slot * (TILE_BYTES >> 4)), qd = q_desc + (uint32_t)((t.k & 1) * (Q_BYTES >> 4));
                const uint32_t acc = tmem + s * S_STRIDE;
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk)                // 16 components: 32 bytes of a 128-byte row, halves apart
                    tc_mma_f16_ss(acc, kd + ((uint32_t)((kk >> 2) * HALF_BYTES + (kk & 3) * 32) >> 4), qd + ((uint32_t)((kk >> 2) * Q_HALF_BYTES + (kk & 3) * 32) >> 4),
                                  IDESC_S, kk ? 1u : 0u);
                tc_commit(&ctl.s_full[s]);
                tc_commit(&ctl.empty[slot]);
                if (--ctl.left[j] == 0) tc_commit(&ctl.q_free[t.k & 1]);
                mbar_arrive(&ctl.s_full[s]);
                const uint32_t about = (t.i == 0 ? 1u : 0u) | (t.i == t.tiles - 1 ? 2u : 0u) | (uint32_t)t.k << 2;
                if (t.scored & 1) { t.x1 = x; t.about1 = about; }
                else { t.x0 = x; t.about0 = about; }
                ++t.scored;
                if (++t.i == t.tiles) { t.loaded = false; t.base += t.total; ++t.k; }
                return true;
            };
            long long since = clock64();
            for (;;) {
                const bool first = step(std::integral_constant<int, 0>()), second = step(std::integral_constant<int, 1>());
                if (st0.end && st1.end && st0.valued == st0.scored && st1.valued == st1.scored) break;
                if (first || second) since = clock64();
                else if (*abort_flag || clock64() - since > PFX_WAIT_CYCLES) { *abort_flag = 1; break; }
            }
            int none = 0;                                          // nothing is in flight when the tensor memory is given back
            tc_commit(&ctl.drain);
            pfx_wait(&ctl.drain, 0u, &none);
          }
        } else if (elect_one()) {
            bool ok = true;
            int n = 0, prev_n = 0;                                 // tiles before this item, and before the previous one
            uint32_t np[2] = {0, 0}, nsc[2] = {0, 0}, nq[2] = {0, 0};      // P tiles taken, S tiles computed per stream; queries per buffer
            bool held = false;                                     // stream 1's last products of the item before are still to come
            TreeItem it, prev;
            const uint64_t q_desc = tc_smem_desc(smem_u32(q_smem), 16u, 1024u, 2u);
            const uint64_t k_desc = tc_smem_desc(smem_u32(ring), 16u, 1024u, 2u);
            const uint64_t v_desc = tc_smem_desc(smem_u32(ring), HALF_BYTES, 1024u, 2u);
            auto scores = [&](int s, int i, bool last) {           // S = Q K^T of a stream's tile
                const int x = n + tree_tile_index(it, s, i), slot = x % KS;
                ok = pfx_wait(&ctl.full[slot], (uint32_t)(x / KS) & 1u, abort_flag);
                if (BESIDE && ok && nsc[s] > 0) ok = pfx_wait(&ctl.s_read[s], (nsc[s] - 1) & 1u, abort_flag);
                if (!ok) return;
                ++nsc[s];
                ctl.stream_bad[s] = ctl.bad[x & 15];
                tc_fence_after_sync();
                const uint64_t a = q_desc + (uint32_t)((it.wide ? s : it.q) * (Q_BYTES >> 4)), b = k_desc + (uint32_t)(slot * (TILE_BYTES >> 4));
                const uint32_t acc = tmem + s * S_STRIDE;
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk) {              // 16 components: 32 bytes of a 128-byte row, halves apart
                    const uint32_t off_k = (uint32_t)((kk >> 2) * HALF_BYTES + (kk & 3) * 32) >> 4;
                    const uint32_t off_q = (uint32_t)((kk >> 2) * Q_HALF_BYTES + (kk & 3) * 32) >> 4;
                    tc_mma_f16_ss(acc, a + off_q, b + off_k, IDESC_S, kk ? 1u : 0u);
                }
                tc_commit(&ctl.s_full[s]);
                if (!it.wide || s == 1) tc_commit(&ctl.empty[slot]);
                if (last && (it.wide || it.q == 0)) tc_commit(&ctl.q_free[0]);
                if (last && (it.wide || it.q == 1)) tc_commit(&ctl.q_free[1]);
                mbar_arrive(&ctl.s_full[s]);
            };
            auto values = [&](const TreeItem& im, int n0, int s, int i) {     // O += P V of a stream's tile, quarter by quarter
                const int x = n0 + tree_tile_index(im, s, i), slot = KS + x % VS;
                ok = pfx_wait(&ctl.full[slot], (uint32_t)(x / VS) & 1u, abort_flag);
                const uint64_t b = v_desc + (uint32_t)(slot * (TILE_BYTES >> 4));
                const uint32_t acc = tmem + O_COL + s * O_STRIDE;
                const uint32_t a = tmem + P_COL + s * P_STRIDE;
#pragma unroll
                for (int part = 0; part < 4; ++part) {
                    ok = ok && pfx_wait(&ctl.p_full[s][part], np[s] & 1u, abort_flag);
                    if (!ok) return;
                    tc_fence_after_sync();
#pragma unroll
                    for (int kk = part * 2; kk < part * 2 + 2; ++kk)       // 16 tokens: 8 columns of P
                        tc_mma_f16_ts(acc, a + kk * 8, b + (uint32_t)(kk * 2048 >> 4), IDESC_O, kk ? 1u : (i ? 1u : 0u));
                }
                ++np[s];
                if (!im.wide || s == 1) tc_commit(&ctl.empty[slot]);
                if (BESIDE) tc_commit(&ctl.p_free[s]);
                if (i == tree_stream_tiles(im, s) - 1) tc_commit(&ctl.o_full[s][0]);
            };
            auto release = [&]() {                                 // the held products, where there is nothing to put in front of them
                if (held) values(prev, prev_n, 1, tree_stream_tiles(prev, 1) - 1);
                held = false;
            };
            for (int k = 0; ok; ++k) {
                const int j = k % TREE_ITEMS;
                if (!mbar_test(&ctl.item_full[j], (uint32_t)(k / TREE_ITEMS) & 1u)) release();
                ok = ok && pfx_wait(&ctl.item_full[j], (uint32_t)(k / TREE_ITEMS) & 1u, abort_flag);
                if (!ok) break;
                it = ctl.item[j];
                mbar_arrive(&ctl.item_empty[j]);
                if (!it.valid) break;
                const uint32_t q_parity = (it.q ? nq[1]++ : nq[0]++) & 1u;
                if (!mbar_test(&ctl.q_full[it.q], q_parity) || !mbar_test(&ctl.full[n % KS], (uint32_t)(n / KS) & 1u)) release();
                ok = ok && pfx_wait(&ctl.q_full[it.q], q_parity, abort_flag);
                if (!ok) break;
                const int n0 = tree_stream_tiles(it, 0), n1 = tree_stream_tiles(it, 1);      // n0 >= n1, n0 >= 1
                int left = n0 + n1;                                // score products still to issue
                scores(0, 0, --left == 0);
                if (ok) release();
                if (ok && n1 > 0) scores(1, 0, --left == 0);
                for (int i = 0; i < n0 && ok; ++i) {
                    if (BESIDE && i + 1 < n0) scores(0, i + 1, --left == 0);
                    if (ok) values(it, n, 0, i);
                    if (!BESIDE && ok && i + 1 < n0) scores(0, i + 1, --left == 0);
                    if (!ok || i >= n1) break;
                    if (i + 1 == n0) { held = true; break; }       // behind the next item's first scores
                    if (BESIDE && i + 1 < n1) scores(1, i + 1, --left == 0);
                    if (ok) values(it, n, 1, i);
                    if (!BESIDE && ok && i + 1 < n1) scores(1, i + 1, --left == 0);
                }
                prev = it;
                prev_n = n;
                n += it.tiles;
            }
            if (ok) release();
            int none = 0;                                          // nothing is in flight when the tensor memory is given back
            tc_commit(&ctl.drain);
            pfx_wait(&ctl.drain, 0u, &none);
        }
        __syncwarp();
      }
    } else if (warp < 8) {
        reg_grow<tree_regs_softmax<ROWS>()>();
        // =============================== softmax warps: S -> P, epilogue ===============================
        const int s = warp >> 2, w4 = warp & 3;                    // stream, quarter of its lanes
        const uint32_t lanes = (uint32_t)(w4 * 32) << 16;
        const uint32_t s_tmem = tmem + s * S_STRIDE + lanes, o_tmem = tmem + O_COL + lanes;     // (o_tmem: of stream 0)
        const int r = w4 * 32 + lane;                              // row of the stream (token of the tile)
        const float sc = p.scale_log2;
        const uint64_t keep = l2_evict_last_policy();
        bool ok = true;
        uint32_t ns = 0, no1 = 0, nj = 0;                          // tiles of this stream, items with tiles of stream 1, joins so far
        auto join_sync = [&]() {                                   // with the other warps that join the streams
            uint64_t* const bar = &ctl.join_sync[w4];
            __syncwarp();
            if (lane == 0) mbar_arrive(bar);
            return pfx_warp_wait(bar, nj++ & 1u, abort_flag);
        };
        // V rows outside the slice, and of refused pages, hold anything (NaN patterns among it) and meet weights of 0, and so do rows
        // of new tokens with those that do not see them.  They are cleared before the tile's weights are handed over: thread r looks
        // at token r.  (Where the streams share a tile both do, and write the same.)
        auto clear_v = [&](int x, bool clear, bool look, int j) {  // x: the tile's number
            if (!__any_sync(0xffffffffu, clear || look)) return true;
            const int slot = KS + x % VS;
            if (!pfx_warp_wait(&ctl.full[slot], (uint32_t)(x / VS) & 1u, abort_flag)) return false;
            if (clear || look)
#pragma unroll 1
                for (int hf = 0; hf < HALVES; ++hf) {              // whole 128-byte rows: the swizzle does not matter
                    const uint32_t a = smem_u32(ring) + slot * TILE_BYTES + hf * HALF_BYTES + r * 128;
                    bool zero = clear;
                    if (!clear) {
                        uint32_t found = 0;
#pragma unroll
                        for (int u = 0; u < 8; ++u) found |= not_finite<BF16>(lds128(a + ((u + lane) & 7) * 16));
                        zero = found & 0x80008000u;
                        if (zero) *reinterpret_cast<volatile int*>(&ctl.poisoned[j]) = 1;
                    }
                    if (zero)
#pragma unroll
                        for (int u = 0; u < 8; ++u) sts128_zero(a + ((u + lane) & 7) * 16);
                }
            fence_proxy_async();
            return true;
        };
        int n = 0;                                                 // tiles of earlier items
        cudaGridDependencySynchronize();
        for (int k = 0; ok; ++k) {
            const int j = k % TREE_ITEMS;
            ok = pfx_warp_wait(&ctl.item_full[j], (uint32_t)(k / TREE_ITEMS) & 1u, abort_flag);
            if (!ok) break;
            const TreeItem it = ctl.item[j];
            if (!it.valid) break;
            const int tiles = tree_stream_tiles(it, s), tiles1 = tree_stream_tiles(it, 1);
            if constexpr (FEW) {
                // ---- a thread is a token.  Lane i speaks for row i mod ROWS of the unit, the rows' references being the same in all
                // warps of the stream ----
                const int rows = it.nodes * p.G;
                float ref = NEG_INF, l[ROWS];                      // of this lane's row; over this thread's tokens
#pragma unroll
                for (int c = 0; c < ROWS; ++c) l[c] = 0.f;
                for (int i = 0; i < tiles; ++i) {
                    ok = pfx_warp_wait(&ctl.s_full[s], ns & 1u, abort_flag);
                    if (!ok) break;
                    ++ns;
                    tc_fence_after_sync();
                    const int t = it.first + tree_tile_index(it, s, i) * TREE_TILE;
                    const uint32_t bad = *reinterpret_cast<volatile uint8_t*>(&ctl.stream_bad[s]);
                    float x[ROWS], e[ROWS];
                    if constexpr (ROWS == 16) tmem_ld_32x16(s_tmem, *reinterpret_cast<uint32_t(*)[16]>(&x[0]));
                    else tmem_ld_32x32(s_tmem, *reinterpret_cast<uint32_t(*)[32]>(&x[0]));
                    tmem_ld_wait();
                    tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&ctl.s_read[s]);
                    if (t < it.lo || t + TREE_TILE > min(it.hi, it.len) || bad) {      // tokens outside the slice, of refused pages, not seen
                        uint32_t hide = t + r < it.lo || t + r >= it.hi || ((bad >> (r >> 4)) & 1u) ? ~0u : 0u;
                        const int d = t + r - it.len;              // which new token this is
                        ok = clear_v(n + tree_tile_index(it, s, i), hide != 0, d >= 0, j);
                        if (!ok) break;
                        if (d >= 0 && hide == 0) {
                            if (!p.mask) hide = d * p.G >= 32 ? ~0u : (1u << (d * p.G)) - 1u;          // tokens in front of it
                            else {
                                const uint32_t group = p.G >= 32 ? ~0u : (1u << p.G) - 1u;
                                const uint32_t* const words = p.mask + (size_t)it.row0 * p.words + (d >> 5);
#pragma unroll 2
                                for (int u = 0; u < it.nodes; ++u)
                                    if (!((words[(size_t)u * p.words] >> (d & 31)) & 1u)) hide |= group << (u * p.G);
                            }
                        }
#pragma unroll
                        for (int c = 0; c < ROWS; ++c) x[c] = (hide >> c) & 1u ? NEG_INF : x[c];
                    }
                    auto exponents = [&]() {                       // scale (x - reference), in powers of 2, lifted
                        const float2 sc2 = make_float2(sc, sc);
#pragma unroll
                        for (int c = 0; c < ROWS; c += 4) {
                            const float4 a = *reinterpret_cast<const float4*>(&ctl.col.off[s][c]);
                            const float2 lo = fma2(make_float2(x[c], x[c + 1]), sc2, make_float2(a.x, a.y));
                            const float2 hi = fma2(make_float2(x[c + 2], x[c + 3]), sc2, make_float2(a.z, a.w));
                            e[c] = lo.x; e[c + 1] = lo.y; e[c + 2] = hi.x; e[c + 3] = hi.y;
                        }
                    };
                    exponents();
                    // a row's reference moves only when a logit is more than 2^8 above it (then the weights would leave the 16-bit
                    // types' comfortable range), and at a unit's first tile.  The four warps find out by a vote; those that want
                    // to move leave their maxima
                    const bool up = i == 0 || __any_sync(0xffffffffu, row_max<ROWS>(e) > TREE_PAST + LIFT);
                    const int turn = (int)(ns % 3);
                    if (up) {
                        const float mx = across_lanes<ROWS, true>(x, lane);
                        if (lane < ROWS) atomicMax(&ctl.col.top[turn][s][lane], ordered(mx));
                        if (lane == 0) *reinterpret_cast<volatile int*>(&ctl.moved[turn][s]) = (int)ns;
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&ctl.vote[s]);
                    ok = pfx_warp_wait(&ctl.vote[s], (ns - 1) & 1u, abort_flag);
                    if (!ok) break;
                    // the last turn's maxima have been read by all: cleared for the one after the next
                    if (w4 == 0 && lane < ROWS) ctl.col.top[(ns + 2) % 3][s][lane] = 0;
                    if (ns > 1) {                                  // the last tile's weights are used up, and its products in O
                        ok = pfx_warp_wait(&ctl.p_free[s], (ns - 2) & 1u, abort_flag);
                        if (!ok) break;
                        tc_fence_after_sync();
                    }
                    if (*reinterpret_cast<volatile int*>(&ctl.moved[turn][s]) == (int)ns) {
                        const int c = lane & (ROWS - 1);
                        const uint32_t m = *reinterpret_cast<volatile uint32_t*>(&ctl.col.top[turn][s][c]);
                        const float now = fmaxf(ref, m ? unordered(m) : NEG_INF), f = ref == NEG_INF ? 0.f : fast_exp2((ref - now) * sc);
                        ref = now;
                        // the exponents' summand (the same from all warps): for a row that has not seen anything yet one that lifts any
                        // finite logit over the limit, for one that does not exist one that lifts none
                        ctl.col.off[s][c] = c >= rows ? NEG_INF : now == NEG_INF ? 1e30f : fmaf(-now, sc, LIFT);
                        __syncwarp();
                        exponents();
                        if (i > 0) {
#pragma unroll
                            for (int u = 0; u < ROWS; ++u) l[u] *= __shfl_sync(0xffffffffu, f, u);
#pragma unroll 1
                            for (int c0 = 0; c0 < ROWS; c0 += 8) {
                                uint32_t y[8];
                                tmem_ld_32x8(o_tmem + ((k & 1) * 2 + s) * O_STRIDE + c0, y);
                                tmem_ld_wait();
#pragma unroll
                                for (int u = 0; u < 8; ++u) y[u] = __float_as_uint(__uint_as_float(y[u]) * __shfl_sync(0xffffffffu, f, c0 + u));
                                tmem_st_32x8(o_tmem + ((k & 1) * 2 + s) * O_STRIDE + c0, y);
                            }
                            tmem_st_wait();
                        }
                    }
                    uint8_t* const dst = p_smem + s * P_BYTES + r * 16;
#pragma unroll
                    for (int c = 0; c < ROWS; c += 8) {
                        uint32_t w[4];
#pragma unroll
                        for (int u = 0; u < 8; ++u) {
                            e[c + u] = fast_exp2(e[c + u]);
                            l[c + u] += e[c + u];
                        }
#pragma unroll
                        for (int u = 0; u < 4; ++u) w[u] = pack2<BF16>(e[c + 2 * u], e[c + 2 * u + 1]);
                        *reinterpret_cast<uint4*>(dst + (c / 8) * 2048) = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                    fence_proxy_async();                           // the tensor core reads P through the asynchronous proxy
                    tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&ctl.p_full[s][0]);
                }
                if (!ok) break;
                // ---- the piece's end: its references and sums of weights go to the warps that finish it ----
                const float sum = across_lanes<ROWS, false>(l, lane);
                if (k >= 1) ok = pfx_warp_wait(&ctl.sums_free, (uint32_t)(k - 1) & 1u, abort_flag);
                if (!ok) break;
                if (lane < ROWS) {
                    ctl.col.sums[s][w4][lane] = sum;
                    if (w4 == 0) ctl.col.ref[s][lane] = ref;
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(&ctl.sums_full);
            } else {
                // ---- a thread is a row ----
                const uint32_t p_tmem = tmem + P_COL + s * P_STRIDE + lanes;
                const int r_node = fast_div(r, p.div_G);
                const int at = (it.wide ? s * p.nodes : 0) + r_node;    // this row's new token in the unit
                const bool exists = r_node < p.nodes && at < it.nodes;
                const bool live = __any_sync(0xffffffffu, exists); // some row of this warp exists
                const int node = it.i0 + at, row = it.row0 + at;
                float m_true = NEG_INF, m_ref = NEG_INF, l = 0.f;  // the maximum, and the one the weights refer to (raw logits)
                for (int i = 0; i < tiles; ++i) {
                    ok = pfx_warp_wait(&ctl.s_full[s], ns & 1u, abort_flag);
                    if (!ok) break;
                    ++ns;
                    tc_fence_after_sync();
                    const int t = it.first + tree_tile_index(it, s, i) * TREE_TILE;
                    const int c_lo = max(it.lo - t, 0), c_hi = min(it.hi - t, TREE_TILE);
                    const uint32_t bad = *reinterpret_cast<volatile uint8_t*>(&ctl.stream_bad[s]);
                    const bool tail = t + TREE_TILE > it.len, edge = c_lo > 0 || c_hi < TREE_TILE || tail || bad;
                    auto clear = [&]() { return !edge || clear_v(n + tree_tile_index(it, s, i), r < c_lo || r >= c_hi || ((bad >> (r >> 4)) & 1u), t + r >= it.len, j); };
                    // (where S may be overwritten early, that comes first; else the row is not in registers yet)
                    if (!BESIDE) ok = clear();
                    if (!ok) break;
                    if (live) {
                        float x[TREE_TILE];
#pragma unroll
                        for (int c0 = 0; c0 < TREE_TILE; c0 += 32) tmem_ld_32x32(s_tmem + c0, *reinterpret_cast<uint32_t(*)[32]>(&x[c0]));
                        tmem_ld_wait();
                        if (BESIDE) {
                            tc_fence_before_sync();
                            __syncwarp();
                            if (lane == 0) mbar_arrive(&ctl.s_read[s]);
                        }
                        if (BESIDE) ok = clear();
                        if (!ok) break;
                        if (edge) {                                // columns outside the slice, of refused pages, of tokens not seen
#pragma unroll
                            for (int c = 0; c < 4; ++c) {
                                uint32_t out = ((bad >> (2 * c)) & 1u ? 0xffffu : 0u) | ((bad >> (2 * c + 1)) & 1u ? 0xffff0000u : 0u);
                                const int below = c_lo - c * 32, in = c_hi - c * 32;
                                out |= below >= 32 ? ~0u : (below > 0 ? (1u << below) - 1u : 0u);
                                out |= in <= 0 ? ~0u : (in < 32 ? ~0u << in : 0u);
                                const int d0 = t + c * 32 - it.len;    // the new token at the first of these columns
                                if (tail && exists && d0 > -32) {
                                    const int w = max(d0, 0) >> 5;
                                    const uint32_t a = tree_word(p, row, node, w);
                                    if (d0 < 0) out |= ~a << -d0;
                                    else out |= ~__funnelshift_r(a, (d0 & 31) ? tree_word(p, row, node, w + 1) : 0u, d0 & 31);
                                }
#pragma unroll
                                for (int u = 0; u < 32; ++u) x[c * 32 + u] = (out >> u) & 1u ? NEG_INF : x[c * 32 + u];
                            }
                        }
                        const float mx = row_max<TREE_TILE>(x);
                        m_true = fmaxf(m_true, mx);
                        // a row's sums follow its maximum only when that has moved by more than 2^8 (then the weights would leave
                        // the 16-bit types' comfortable range).  Each row decides by itself, so its result does not depend on its
                        // neighbours (rows that do not exist among them)
                        const bool moved = (m_true - m_ref) * sc > TREE_PAST;
                        if (BESIDE && ns > 1) {            // the last tile's weights are used up, and its products in O
                            ok = pfx_warp_wait(&ctl.p_free[s], (ns - 2) & 1u, abort_flag);
                            if (!ok) break;
                            tc_fence_after_sync();
                        }
                        if (__any_sync(0xffffffffu, moved && exists)) {
                            const float f = !moved ? 1.f : m_ref == NEG_INF ? 0.f : fast_exp2((m_ref - m_true) * sc);
                            if (moved) m_ref = m_true;
                            if (i > 0) {
                                l *= f;
#pragma unroll 1
                                for (int c0 = 0; c0 < D; c0 += 8) {
                                    uint32_t y[8];
                                    tmem_ld_32x8(o_tmem + s * O_STRIDE + c0, y);
                                    tmem_ld_wait();
#pragma unroll
                                    for (int u = 0; u < 8; ++u) y[u] = __float_as_uint(__uint_as_float(y[u]) * f);
                                    tmem_st_32x8(o_tmem + s * O_STRIDE + c0, y);
                                }
                            }
                        }
                        const float off = m_ref == NEG_INF ? 0.f : fmaf(-m_ref, sc, LIFT);
                        const float2 sc2 = make_float2(sc, sc), off2 = make_float2(off, off);
                        float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
                        // a quarter of the tokens at a time; each is handed over when the next one's weights are computed (a store
                        // into tensor memory takes some 300 cycles to complete while the tensor cores work)
                        auto hand_over = [&](int c) {
                            tmem_st_wait();
                            tc_fence_before_sync();
                            __syncwarp();
                            if (lane == 0) mbar_arrive(&ctl.p_full[s][c]);
                        };
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            uint32_t w[16];
#pragma unroll
                            for (int u = 0; u < 16; ++u) {
                                float2 e = fma2(make_float2(x[c * 32 + 2 * u], x[c * 32 + 2 * u + 1]), sc2, off2);
                                e.x = fast_exp2(e.x);
                                e.y = fast_exp2(e.y);
                                sum[u & 1] = add2(sum[u & 1], e);
                                w[u] = pack2<BF16>(e.x, e.y);
                            }
                            if (c > 0) hand_over(c - 1);
                            tmem_st_32x16(p_tmem + c * 16, w);
                        }
                        hand_over(3);
                        l += (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
                    } else {
                        if (BESIDE) ok = clear();
                        if (!ok) break;
                        tc_fence_before_sync();
                        __syncwarp();
                        if (BESIDE && lane == 0) mbar_arrive(&ctl.s_read[s]);
                        if (BESIDE && ns > 1) ok = pfx_warp_wait(&ctl.p_free[s], (ns - 2) & 1u, abort_flag);
                        if (!ok) break;
                        if (lane < 4) mbar_arrive(&ctl.p_full[s][lane]);
                    }
                }
                if (!ok) break;
                // ---- the piece's end.  Stream 0 has a tile always; where the streams share their rows, each takes half of the
                // components of both streams' sums ----
                if (it.wide ? s == 0 : true) ok = pfx_warp_wait(&ctl.o_full[0][0], (uint32_t)k & 1u, abort_flag);
                if (ok && tiles1 > 0 && (it.wide ? s == 1 : true)) ok = pfx_warp_wait(&ctl.o_full[1][0], no1 & 1u, abort_flag);
                if (!ok) break;
                if (tiles1 > 0) ++no1;
                tc_fence_after_sync();
                if (live) {
                    // sums refer to m_ref, at most 2^8 below the maximum: as good a reference as the maximum itself
                    float m_raw = m_ref, f0 = m_ref == NEG_INF ? 0.f : 1.f, f1 = 0.f;      // factors on the two sums
                    bool both = false;
                    uint32_t o0 = o_tmem + s * O_STRIDE, o1 = o0;
                    int c_begin = 0, c_end = D;
                    if (!it.wide) {
                        ctl.join[s][r] = make_float2(m_ref, l);
                        ok = join_sync();
                        if (!ok) break;
                        const float2 other = ctl.join[s ^ 1][r];
                        m_raw = fmaxf(m_ref, other.x);
                        const float a = m_ref == NEG_INF ? 0.f : fast_exp2((m_ref - m_raw) * sc), b = other.x == NEG_INF ? 0.f : fast_exp2((other.x - m_raw) * sc);
                        l = l * a + other.y * b;
                        f0 = s == 0 ? a : b;
                        f1 = s == 0 ? b : a;
                        both = tiles1 > 0;
                        o0 = o_tmem;
                        o1 = o0 + O_STRIDE;
                        c_begin = s * (D / 2);
                        c_end = c_begin + D / 2;
                    }
                    const size_t orow = (size_t)row * p.Hq + it.h * p.G + (r - r_node * p.G);
                    const float m = m_raw == NEG_INF ? NEG_INF : fmaf(m_raw, p.scale, -LIFT_LN);
                    const bool last_word = it.wide || s == 0;      // who writes the row's single numbers
                    if (__builtin_expect(exists && *reinterpret_cast<volatile int*>(&ctl.poisoned[j]) && tree_poisoned<D, BF16>(p, it, row, node), 0)) {
                        f0 = __int_as_float(0x7fc00000);
                        f1 = 0.f;
                    }
                    float top = m, inv = 1.f;
                    if (it.whole && exists) {
                        const float own = tree_join_host(p, orow, m, l, top);
                        inv = l == 0.f ? 0.f : 1.f / l;
                        f0 *= own * inv;
                        f1 *= own * inv;
                        if (p.lse && last_word) p.lse[orow] = l == 0.f ? NEG_INF : top + logf(l);
                    }
                    const size_t prow = (size_t)it.slot * 256 + (it.wide ? s * TREE_TILE : 0) + r;
                    if (!it.whole && exists && last_word) { p.ws.m[prow] = m; p.ws.l[prow] = l; }
#pragma unroll 1
                    for (int c0 = c_begin; c0 < c_end; c0 += 32) {
                        float y[32];
                        __syncwarp();                              // (tensor memory is read by whole warps)
                        tmem_ld_32x32(o0 + c0, *reinterpret_cast<uint32_t(*)[32]>(&y[0]));
                        tmem_ld_wait();
#pragma unroll
                        for (int u = 0; u < 32; ++u) y[u] = f0 == 0.f ? 0.f : y[u] * f0;
                        if (both) {
                            float z[32];
                            tmem_ld_32x32(o1 + c0, *reinterpret_cast<uint32_t(*)[32]>(&z[0]));
                            tmem_ld_wait();
#pragma unroll
                            for (int u = 0; u < 32; ++u) y[u] = f1 == 0.f ? y[u] : fmaf(z[u], f1, y[u]);
                        }
                        if (!exists) continue;
                        if (!it.whole) {
#pragma unroll
                            for (int u = 0; u < 32; u += 8) st_global_hint8(p.ws.o + prow * D + c0 + u, *reinterpret_cast<const float(*)[8]>(&y[u]), keep);
                            continue;
                        }
#pragma unroll 1
                        for (int x = 0; x < p.src.n; ++x)
#pragma unroll 1
                            for (int c = 0; c < p.src.nc[x]; ++c) {
                                const size_t q = orow * p.src.nc[x] + c;
                                const float hm = p.src.m[x][q];
                                if (hm == NEG_INF) continue;       // (its o row is not read)
                                const float w = fast_exp2((hm - top) * 1.4426950408889634f) * inv;
                                const float4* const ho = reinterpret_cast<const float4*>(p.src.o[x] + q * D + c0);
#pragma unroll
                                for (int u = 0; u < 8; ++u) {
                                    const float4 v = ho[u];
                                    y[4 * u] = fmaf(v.x, w, y[4 * u]); y[4 * u + 1] = fmaf(v.y, w, y[4 * u + 1]);
                                    y[4 * u + 2] = fmaf(v.z, w, y[4 * u + 2]); y[4 * u + 3] = fmaf(v.w, w, y[4 * u + 3]);
                                }
                            }
                        uint4* const dst = reinterpret_cast<uint4*>(p.out + orow * D + c0);
#pragma unroll
                        for (int u = 0; u < 4; ++u)
                            dst[u] = make_uint4(pack2<BF16>(y[8 * u], y[8 * u + 1]), pack2<BF16>(y[8 * u + 2], y[8 * u + 3]),
                                                pack2<BF16>(y[8 * u + 4], y[8 * u + 5]), pack2<BF16>(y[8 * u + 6], y[8 * u + 7]));
                    }
                    if (!it.wide) {                                // both streams' sums are read: either may begin anew
                        tc_fence_before_sync();
                        ok = join_sync();
                        if (!ok) break;
                    }
                }
            }
            n += it.tiles;
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(&ctl.item_empty[j]);
        }
    } else if constexpr (FEW) {
        if (warp >= TREE_END_WARP) {
        reg_shrink<TREE_REGS_OTHER>();
        // =============================== (few rows) the pieces' ends: sums of both streams, the host's partials, the result ===============================
        cudaGridDependencySynchronize();
        const int w4 = warp & 3, r = w4 * 32 + lane;
        const float sc = p.scale_log2;
        const uint64_t keep = l2_evict_last_policy();
        uint32_t no1[2] = {0, 0};                                  // even and odd pieces with tiles of stream 1 so far
        bool ok = true;
        for (int k = 0; ok; ++k) {
            const int j = k % TREE_ITEMS;
            ok = pfx_warp_wait(&ctl.item_full[j], (uint32_t)(k / TREE_ITEMS) & 1u, abort_flag);
            if (!ok) break;
            const TreeItem it = ctl.item[j];
            if (!it.valid) break;
            const int tiles1 = tree_stream_tiles(it, 1), rows = it.nodes * p.G;
            const uint32_t o_tmem = tmem + O_COL + (k & 1) * 2 * O_STRIDE + ((uint32_t)(w4 * 32) << 16);      // of stream 0
            ok = pfx_warp_wait(&ctl.sums_full, (uint32_t)k & 1u, abort_flag);
            if (!ok) break;
            const int c = lane & (ROWS - 1), node = fast_div(c, p.div_G);       // this lane's row
            const bool exists = c < rows, both = tiles1 > 0;
            const float ref0 = ctl.col.ref[0][c], ref1 = ctl.col.ref[1][c], m_raw = fmaxf(ref0, ref1);
            float f0 = ref0 == NEG_INF ? 0.f : fast_exp2((ref0 - m_raw) * sc), f1 = ref1 == NEG_INF || !both ? 0.f : fast_exp2((ref1 - m_raw) * sc);
            float lsum = (ctl.col.sums[0][0][c] + ctl.col.sums[0][1][c] + ctl.col.sums[0][2][c] + ctl.col.sums[0][3][c]) * f0 +
                         (ctl.col.sums[1][0][c] + ctl.col.sums[1][1][c] + ctl.col.sums[1][2][c] + ctl.col.sums[1][3][c]) * f1;
            __syncwarp();
            if (lane == 0) mbar_arrive(&ctl.sums_free);
            const int row = it.row0 + node;
            const size_t orow = (size_t)row * p.Hq + it.h * p.G + (c - node * p.G);
            const size_t prow = (size_t)it.slot * 256 + c;
            const float m = m_raw == NEG_INF ? NEG_INF : fmaf(m_raw, p.scale, -LIFT_LN);
            if (__builtin_expect(exists && *reinterpret_cast<volatile int*>(&ctl.poisoned[j]) && tree_poisoned<D, BF16>(p, it, row, it.i0 + node), 0)) {
                f0 = __int_as_float(0x7fc00000);
                f1 = 0.f;
            }
            float top = m, inv = 1.f;
            if (it.whole && exists) {
                const float own = tree_join_host(p, orow, m, lsum, top);
                inv = lsum == 0.f ? 0.f : 1.f / lsum;
                f0 *= own * inv;
                f1 *= own * inv;
                if (p.lse && w4 == 0 && lane < ROWS) p.lse[orow] = lsum == 0.f ? NEG_INF : top + logf(lsum);
            }
            if (!it.whole && exists && w4 == 0 && lane < ROWS) { p.ws.m[prow] = m; p.ws.l[prow] = lsum; }
            // lane l of tensor memory holds component l of the rows (128 components), or, for M = 64 products, lane 32 w + i
            // holds component 16 w + i (i < 16; lanes 16-31 of each quarter unused)
            const int d = D == 128 ? r : w4 * 16 + lane;
            const bool holds = D == 128 || lane < 16;
            const int to_row = (int)orow;
            ok = pfx_warp_wait(&ctl.o_full[0][k & 1], (uint32_t)(k / 2) & 1u, abort_flag);
            if (ok && both) ok = pfx_warp_wait(&ctl.o_full[1][k & 1], ((k & 1 ? no1[1]++ : no1[0]++)) & 1u, abort_flag);
            if (!ok) break;
            tc_fence_after_sync();
#pragma unroll 1
            for (int c0 = 0; c0 < rows; c0 += 8) {
                uint32_t y0[8], y1[8];
                __syncwarp();                                  // (tensor memory is read by whole warps)
                tmem_ld_32x8(o_tmem + c0, y0);
                tmem_ld_32x8(o_tmem + (both ? O_STRIDE : 0) + c0, y1);
                tmem_ld_wait();
                float y[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    const float g0 = __shfl_sync(0xffffffffu, f0, c0 + u), g1 = __shfl_sync(0xffffffffu, f1, c0 + u);
                    y[u] = g0 == 0.f ? 0.f : __uint_as_float(y0[u]) * g0;
                    if (g1 != 0.f) y[u] = fmaf(__uint_as_float(y1[u]), g1, y[u]);
                }
                const int left = min(8, rows - c0);
                if (it.whole) {
#pragma unroll 1
                    for (int z = 0; z < p.src.n; ++z)
#pragma unroll 1
                        for (int e = 0; e < p.src.nc[z]; ++e) {          // (an empty partial's o row is not read)
                            float w = 0.f;
                            if (exists) {
                                const float hm = p.src.m[z][orow * p.src.nc[z] + e];
                                if (hm != NEG_INF) w = fast_exp2((hm - top) * 1.4426950408889634f) * inv;
                            }
#pragma unroll
                            for (int u = 0; u < 8; ++u) {
                                const float wu = __shfl_sync(0xffffffffu, w, c0 + u);
                                const size_t q = (size_t)__shfl_sync(0xffffffffu, to_row, c0 + u) * p.src.nc[z] + e;
                                if (wu != 0.f && u < left && holds) y[u] = fmaf(p.src.o[z][q * D + d], wu, y[u]);
                            }
                        }
#pragma unroll
                    for (int u = 0; u < 8; ++u) {
                        const size_t q = (size_t)__shfl_sync(0xffffffffu, to_row, c0 + u);
                        if (u < left && holds) p.out[q * D + d] = (uint16_t)pack2<BF16>(y[u], 0.f);
                    }
                } else {
                    float* const dst = p.ws.o + ((size_t)it.slot * 256 + c0) * D + d;
#pragma unroll
                    for (int u = 0; u < 8; ++u)
                        if (u < left && holds) st_global_hint(dst + u * D, y[u], keep);
                }
            }
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(&ctl.o_free[k & 1]);
                mbar_arrive(&ctl.item_empty[j]);
            }
        }
        }
    }
    __syncthreads();
    if (*abort_flag) {                                             // (nobody raises it any more: all threads agree)
        if (lane == 0) {
            if (warp == TREE_K_WARP || warp == TREE_V_WARP) ctl.issued[warp - TREE_K_WARP] = issued;
            if (warp == TREE_ITEM_WARP) { ctl.q_issued[0] = (int)q_armed[0]; ctl.q_issued[1] = (int)q_armed[1]; }
        }
        __syncthreads();
        // unwinding: copies into this CTA's shared memory may still be on their way.  A warp per slot of the ring and per buffer of
        // the queries, so that the waits' limits do not add up
        if (lane == 0) {
            int none = 0;
            if (warp < S) {
                // the last tile requested into the slot is the only one that can still be coming
                const int slots = warp < KS ? KS : VS, at = warp < KS ? warp : warp - KS, tiles = ctl.issued[warp < KS ? 0 : 1];
                if (tiles > at) pfx_wait(&ctl.full[warp], (uint32_t)((tiles - 1 - at) / slots) & 1u, &none);
            }
            const int buffer = warp - TREE_MMA_WARP;               // (two buffers; with few rows there are four more warps)
            if (buffer >= 0 && buffer < 2 && ctl.q_issued[buffer] > 0) pfx_wait(&ctl.q_full[buffer], (uint32_t)(ctl.q_issued[buffer] - 1) & 1u, &none);
        }
        if (tid == 0 && p.status) atomicOr(p.status, HG_DEV_WAIT_TIMEOUT);
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    if (warp == TREE_MMA_WARP) tmem_dealloc(tmem, TMEM_COLS);
}

// Joins the pieces of the units that the ends of the CTAs' stretches cut, and the host's partials.  Grid (CTAs of the kernel in
// front, splits of a unit's rows), a warp per row.
constexpr int TREE_MERGE_THREADS = 256;

template <int D, bool BF16>
__global__ void __launch_bounds__(TREE_MERGE_THREADS) tree_merge_kernel(const __grid_constant__ TreeParams p) {
    constexpr int W = D / 32;                                      // components per lane
    constexpr float LOG2E = 1.4426950408889634f;
    const float NEG_INF = __int_as_float(0xff800000);
    cudaTriggerProgrammaticLaunchCompletion();
    cudaGridDependencySynchronize();
    const int4 cut = *reinterpret_cast<const int4*>(&p.ws.cut[blockIdx.x]);       // row0, nodes, h, last
    const int bits = p.status ? *reinterpret_cast<volatile int32_t*>(p.status) : 0;
    if (cut.y <= 0 || (bits & HG_DEV_WAIT_TIMEOUT)) return;
    const int lane = threadIdx.x & 31, first = blockIdx.x, pieces = cut.w - first + 1, stream_rows = p.nodes * p.G;
#pragma unroll 1
    for (int x = blockIdx.y * (TREE_MERGE_THREADS / 32) + (threadIdx.x >> 5); x < cut.y * p.G; x += gridDim.y * (TREE_MERGE_THREADS / 32)) {
        const int node = fast_div(x, p.div_G), s = x >= stream_rows ? 1 : 0;
        const size_t orow = (size_t)(cut.x + node) * p.Hq + cut.z * p.G + (x - node * p.G);
        const int r = s * TREE_TILE + x - s * stream_rows;
        // a lane holds a piece's (m, l), of 32 pieces at a time; most units have fewer
        auto slot_of = [&](int e) { return e == 0 ? 2 * first + 1 : 2 * (first + e); };
        auto load = [&](int e, float& m, float& pl) {
            m = NEG_INF;
            pl = 0.f;
            if (e >= pieces) return;
            const size_t q = (size_t)slot_of(e) * 256 + r;
            const int valid = p.ws.valid[slot_of(e)];
            const float pm = p.ws.m[q];
            pl = p.ws.l[q];
            if (valid) m = pm;
        };
        float m0, l0, top, l = 0.f, acc[W];
        load(lane, m0, l0);
        top = m0;
#pragma unroll 1
        for (int e = lane + 32; e < pieces; e += 32) {
            float m, pl;
            load(e, m, pl);
            top = fmaxf(top, m);
        }
#pragma unroll 1
        for (int y = 0; y < p.src.n; ++y)
#pragma unroll 1
            for (int c = lane; c < p.src.nc[y]; c += 32) top = fmaxf(top, p.src.m[y][orow * p.src.nc[y] + c]);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
#pragma unroll
        for (int u = 0; u < W; ++u) acc[u] = 0.f;
        // adds up `n` partials whose weights the lanes hold, eight rows of sums requested at a time (one of weight 0 is not read)
        auto add = [&](float m, float pl, int n, auto row_of) {
            const float w = m == NEG_INF ? 0.f : fast_exp2((m - top) * LOG2E);
            l = m == NEG_INF ? l : fmaf(pl, w, l);
#pragma unroll 1
            for (int e0 = 0; e0 < n; e0 += 8) {
                __align__(16) float v[8][W];
                float we[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    we[u] = __shfl_sync(0xffffffffu, w, (e0 + u) & 31);
                    if (e0 + u >= n) we[u] = 0.f;
                    const float* const o = row_of(e0 + u) + lane * W;
#pragma unroll
                    for (int z = 0; z < W; ++z) v[u][z] = 0.f;
                    if (we[u] != 0.f) {
                        if constexpr (W == 4) *reinterpret_cast<float4*>(v[u]) = *reinterpret_cast<const float4*>(o);
                        else *reinterpret_cast<float2*>(v[u]) = *reinterpret_cast<const float2*>(o);
                    }
                }
#pragma unroll
                for (int u = 0; u < 8; ++u)
#pragma unroll
                    for (int z = 0; z < W; ++z) acc[z] = fmaf(v[u][z], we[u], acc[z]);
            }
        };
#pragma unroll 1
        for (int e0 = 0; e0 < pieces; e0 += 32) {
            if (e0 > 0) load(e0 + lane, m0, l0);
            add(m0, l0, min(32, pieces - e0), [&](int e) { return p.ws.o + ((size_t)slot_of(e0 + e) * 256 + r) * D; });
        }
#pragma unroll 1
        for (int y = 0; y < p.src.n; ++y)
#pragma unroll 1
            for (int c0 = 0; c0 < p.src.nc[y]; c0 += 32) {
                const size_t q = orow * p.src.nc[y] + c0;
                const bool is = c0 + lane < p.src.nc[y];
                add(is ? p.src.m[y][q + lane] : NEG_INF, is ? p.src.l[y][q + lane] : 0.f, min(32, p.src.nc[y] - c0),
                    [&](int e) { return p.src.o[y] + (q + e) * D; });
            }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
        const float inv = l == 0.f ? 0.f : 1.f / l;
        if (lane == 0 && p.lse) p.lse[orow] = l == 0.f ? NEG_INF : top + logf(l);
        uint32_t w[W / 2];
#pragma unroll
        for (int u = 0; u < W / 2; ++u) w[u] = pack2<BF16>(acc[2 * u] * inv, acc[2 * u + 1] * inv);
        if constexpr (W == 4) *reinterpret_cast<uint2*>(p.out + orow * D + lane * 4) = make_uint2(w[0], w[1]);
        else *reinterpret_cast<uint32_t*>(p.out + orow * D + lane * 2) = w[0];
    }
}

}  // namespace hg
