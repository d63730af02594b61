// Attention of a step's new tokens over the cache and, masked, over one another (sm_100a).
//
// Token i of sequence b sees the cached positions [begin, len) and the new tokens j, at positions len + j, whose bit its mask
// row has.  For a KV head the new tokens' queries, G per token, are the rows of a matrix Q; over the sequence's tokens
//     S = Q K^T,   m = row max of scale S,   P = e^{scale S - m},   l = row sum of P,   O = P V,   out = O / l,   lse = m + ln l
// with S = -inf where a token is not seen.  K and V are read once for up to 256 rows: below about 120 rows a KV head their stream
// from HBM is the bound at the measured rates, above that the tensor cores.
//
// Both products run on tcgen05.mma with accumulators in tensor memory, two STREAMS of 128 rows per CTA, tiles of 128 tokens: a
// stream's four softmax warps (a thread owns a row) turn S into P, 16-bit in half of S's columns, the A operand of P V.  P is
// rounded to the inputs' type: a weight is off by at most half a step, as the result itself is; l is the sum of the unrounded
// weights.  A UNIT is (sequence, KV head, whole new tokens with up to 256 rows):
//   wide    more than 128 rows: the streams take 128 rows each and share every K and V tile;
//   narrow  up to 128 rows: the streams take alternate tiles and are joined at the end, both in the lanes of tensor memory that
//           the same row has in either.
//
// Work is dealt by cost: the units' tiles stand in a row, and each of the persistent CTAs (one per SM) takes an equal stretch of
// it.  So long and short sequences balance by themselves; a CTA finishes the units that lie wholly in its stretch, the host's
// partials included, and leaves softmax partials of the at most two that its ends cut, which tree_merge_kernel joins.
//
// Roles: warps 0-7 softmax and epilogue; 8 and 9 load K and V tiles (TMA, a ring of tiles that alternates the two); 10 issues the
// products; 11 finds the CTA's stretch, publishes its pieces and loads the queries (TMA, a box of G heads by whole tokens).
// Every wait is bounded.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "hg_device.cuh"
#include "hg_partial.cuh"
#include "hg_ring.h"
#include "hg_tcgen05.cuh"

namespace hg {

constexpr int TREE_TILE = 128;                // tokens per tile, rows per stream
constexpr int TREE_THREADS = 384;
constexpr int TREE_K_WARP = 8, TREE_V_WARP = 9, TREE_MMA_WARP = 10, TREE_ITEM_WARP = 11;
constexpr int TREE_REGS_SOFTMAX = 208, TREE_REGS_OTHER = 72;   // of the 384 x 168 of the launch
constexpr int TREE_MAX_SLOTS = 10;
constexpr uint32_t TREE_S_COL = 0, TREE_O_COL = 256;           // tensor memory: S of the streams, 128 columns each, then their O
constexpr uint32_t TREE_P_COL = 384;                           // ... and with 64 components P beside them, 64 columns each
// Costs of a unit and of its tiles, for the dealing: what starting a unit takes, a tile for two streams and for one.
constexpr int TREE_COST_UNIT = 6, TREE_COST_WIDE = 4, TREE_COST_NARROW = 3;

template <int D> __host__ __device__ constexpr int tree_tile_bytes() { return TREE_TILE * D * 2; }
template <int D> __host__ __device__ constexpr int tree_slots() { return D == 128 ? 5 : 10; }

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
    int nodes;                       // new tokens of a stream's rows: 128 / G
    int page_size, page_shift, max_pages, num_pages;
    int reread, test_stall;          // reread: several units of a KV head read the same tiles
    float scale, scale_log2;
    FastDiv div_G;
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
    const int rest = s.n % (2 * p.nodes);
    s.wides = s.n / (2 * p.nodes) + (rest > p.nodes ? 1 : 0);
    s.narrow = rest > 0 && rest <= p.nodes ? rest : 0;
    return s;
}
__device__ __forceinline__ long long tree_unit_cost(const TreeSeq& s, bool wide) {
    return TREE_COST_UNIT + (long long)s.tiles * (wide ? TREE_COST_WIDE : TREE_COST_NARROW);
}
__device__ __forceinline__ long long tree_head_cost(const TreeSeq& s) {
    return s.wides * tree_unit_cost(s, true) + (s.narrow ? tree_unit_cost(s, false) : 0);
}
// Where the stretch of CTA c of n begins; the CTA that a place belongs to.
__device__ __forceinline__ long long tree_stretch(long long total, int c, int n) { return total / n * c + total % n * c / n; }
__device__ __forceinline__ int tree_cta_of(long long place, long long total, int n) {
    int c = (int)min((long long)n - 1, (long long)((double)place / (double)total * n));
    while (c > 0 && tree_stretch(total, c, n) > place) --c;
    while (c + 1 < n && tree_stretch(total, c + 1, n) <= place) ++c;
    return c;
}
// A unit's tile t stands at TREE_COST_UNIT + t * cost behind the unit's begin; how many stand in front of a place.
__device__ __forceinline__ int tree_tiles_before(long long place, int cost, int tiles) {
    return place <= TREE_COST_UNIT ? 0 : (int)min((long long)tiles, (place - TREE_COST_UNIT + cost - 1) / cost);
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
};

struct TreeCtl {
    uint64_t full[TREE_MAX_SLOTS], empty[TREE_MAX_SLOTS];
    uint64_t s_full[2], s_read[2], p_free[2], p_full[2][4], o_full[2];   // p_full: the quarters of a tile's tokens
    uint64_t edge, q_full, q_free, drain;
    uint64_t join_sync[4];           // the two warps that share 32 rows of a narrow unit
    uint64_t item_full[2], item_empty[2];
    TreeItem item[2];
    uint32_t tmem;
    int abort;
    uint8_t bad[16];                 // per tile, in load order: 16-token pieces of the tile whose page was refused
    uint8_t stream_bad[2];           // the same for the tile a stream's softmax warps are about to read
    uint32_t poison[2][HG_MAX_TREE_NODES / 32];    // new tokens of an item with something not finite in their V rows
    float2 join[2][TREE_TILE];       // per stream, rows' reference and sum (narrow)
    long long part[4];
    long long start_base;
    int start_b;
    int issued[2], q_issued, edge_open;      // tiles, items' queries and edge tiles that were requested (for the unwinding)
};

template <int D> constexpr size_t tree_smem_bytes() { return (size_t)(2 + tree_slots<D>()) * tree_tile_bytes<D>() + sizeof(TreeCtl); }

// Tiles of a stream; number of its tile i in load order.
__device__ __forceinline__ int tree_stream_tiles(const TreeItem& it, int s) { return it.wide ? it.tiles : (it.tiles + 1 - s) / 2; }
__device__ __forceinline__ int tree_tile_index(const TreeItem& it, int s, int i) { return it.wide ? i : 2 * i + s; }

template <bool BF16>
__device__ __forceinline__ bool not_finite(uint4 x) {
    constexpr uint32_t E = BF16 ? 0x7f807f80u : 0x7c007c00u;
    bool any = false;
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int u = 0; u < 4; ++u) any = any || (w[u] & E & 0xffffu) == (E & 0xffffu) || (w[u] & E & 0xffff0000u) == (E & 0xffff0000u);
    return any;
}

template <int D, bool BF16>
__global__ void __launch_bounds__(TREE_THREADS, 1) tree_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                                                               const __grid_constant__ CUtensorMap tmV, const __grid_constant__ TreeParams p) {
    constexpr int S = tree_slots<D>();
    constexpr int TILE_BYTES = tree_tile_bytes<D>();
    constexpr int HALVES = D / 64;
    constexpr uint32_t HALF_BYTES = TREE_TILE * 128;
    constexpr uint32_t FMT = BF16 ? 1u : 0u;
    // instruction descriptors: fp32 accumulator, 16-bit A and B, M = 128; S: both K-major, N = 128 tokens; O: B (V) with
    // its components contiguous (N-major), N = D
    constexpr uint32_t IDESC_S = (1u << 4) | (FMT << 7) | (FMT << 10) | ((128u >> 3) << 17) | ((128u >> 4) << 24);
    constexpr uint32_t IDESC_O = (1u << 4) | (FMT << 7) | (FMT << 10) | (1u << 16) | (((uint32_t)D >> 3) << 17) | ((128u >> 4) << 24);
    // with 64 components tensor memory has room for P beside S: the next S is computed while the weights of this one are
    constexpr bool BESIDE = D == 64;
    constexpr uint32_t P_COL = BESIDE ? TREE_P_COL : TREE_S_COL, P_STRIDE = BESIDE ? 64 : 128, O_STRIDE = BESIDE ? 64 : 128;
    const float NEG_INF = __int_as_float(0xff800000);

    extern __shared__ __align__(1024) uint8_t tree_raw[];
    uint8_t* const ring = tree_raw + 2 * TILE_BYTES;               // Q of the two streams in front
    TreeCtl& ctl = *reinterpret_cast<TreeCtl*>(tree_raw + (2 + S) * TILE_BYTES);
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
            for (int c = 0; c < 4; ++c) mbar_init(&ctl.p_full[s][c], 4);
            mbar_init(&ctl.o_full[s], 1);
            mbar_init(&ctl.item_full[s], 1);
            mbar_init(&ctl.item_empty[s], 8 + 3);
        }
        for (int i = 0; i < 4; ++i) mbar_init(&ctl.join_sync[i], 2);
        mbar_init(&ctl.q_full, 1);
        mbar_init(&ctl.q_free, 1);
        mbar_init(&ctl.drain, 1);
        mbar_init(&ctl.edge, 1);
        ctl.abort = 0;
        fence_barrier_init();
    }
    if (warp == TREE_MMA_WARP) {
        tmem_alloc(&ctl.tmem, 512);
        tmem_relinquish();
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(&ctl.tmem);

    int issued = 0, q_issued = 0;                                  // (loaders) tiles, (item warp) queries requested so far
    uint32_t edges = 0;                                            // (V loader) tiles that went over the edge barrier
    bool edge_open = false;                                        // ... and one that is still on its way
    cudaTriggerProgrammaticLaunchCompletion();
    auto timed_out = [&]() { return p.status && (*reinterpret_cast<volatile int32_t*>(p.status) & HG_DEV_WAIT_TIMEOUT); };
    if (warp >= 8) {
      reg_shrink<TREE_REGS_OTHER>();
      cudaGridDependencySynchronize();
      // ---- the sequences' costs, and where this CTA's stretch begins: 128 threads, a run of sequences each ----
      const int me = tid - 256, cta = blockIdx.x, ctas = gridDim.x;
      if (me < 2) p.ws.valid[2 * cta + me] = 0;
      if (me == 2) p.ws.cut[cta].nodes = 0;
      if (me == 3) ctl.start_b = -1;
      const int run = (p.B + 127) / 128, b_first = min(p.B, me * run), b_last = min(p.B, b_first + run);
      long long mine = 0;
      bool trouble = false;
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
      long long total = 0;
      for (int w = 0; w < 4; ++w) {
          if (w < warp - 8) upto += ctl.part[w];
          total += ctl.part[w];
      }
      const long long from = tree_stretch(total, cta, ctas), to = tree_stretch(total, cta + 1, ctas);
      if (from < to && from >= upto - mine && from < upto) {
          long long base = upto - mine;
          for (int b = b_first; b < b_last; ++b) {
              const long long cost = tree_head_cost(tree_seq(p, b)) * p.Hkv;
              if (from < base + cost) { ctl.start_b = b; ctl.start_base = base; break; }
              base += cost;
          }
      }
      asm volatile("bar.sync 1, 128;" ::: "memory");
      if (warp == TREE_ITEM_WARP) {
        // =============================== item warp: the stretch's pieces, one ahead, and their queries ===============================
        long long at = from, base = ctl.start_base;                // place in the row of tiles; that of the lanes' first sequence
        int ub = ctl.start_b < 0 ? p.B : ctl.start_b;              // first of the 32 sequences in the lanes
        // (after an earlier call that ran into its limit there is no work until the caller has cleared the word)
        if (ub == p.B || __any_sync(0xffffffffu, timed_out())) at = to;
        TreeSeq sq;
        long long cost = 0, before = 0, block = 0;
        auto load_sequences = [&]() {
            sq.n = 0;
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
        bool ok = true;
        int k = 0;
        const int row_bytes = p.G * p.nodes * 128;                 // a query box
        while (ok) {
            TreeItem it;
            it.valid = 0;
            while (at < to) {                                      // the next piece with a tile in it
                while (at >= base + block && ub < p.B) { base += block; ub += 32; load_sequences(); }
                if (ub >= p.B) { at = to; break; }
                const int src = __ffs(__ballot_sync(0xffffffffu, at >= base + before && at < base + before + cost)) - 1;
                TreeSeq s;
                s.row0 = __shfl_sync(0xffffffffu, sq.row0, src); s.n = __shfl_sync(0xffffffffu, sq.n, src);
                s.len = __shfl_sync(0xffffffffu, sq.len, src); s.lo = __shfl_sync(0xffffffffu, sq.lo, src);
                s.hi = __shfl_sync(0xffffffffu, sq.hi, src); s.tiles = __shfl_sync(0xffffffffu, sq.tiles, src);
                s.wides = __shfl_sync(0xffffffffu, sq.wides, src); s.narrow = __shfl_sync(0xffffffffu, sq.narrow, src);
                const long long begin = base + __shfl_sync(0xffffffffu, before, src);
                const long long head = tree_head_cost(s), wide = tree_unit_cost(s, true);
                const int h = (int)((at - begin) / head);
                const long long in_head = (at - begin) - head * h;
                const int u = (int)min((long long)s.wides, in_head / wide);
                const bool is_wide = u < s.wides;
                const long long unit = begin + head * h + wide * u, unit_cost = tree_unit_cost(s, is_wide);
                const int tile_cost = is_wide ? TREE_COST_WIDE : TREE_COST_NARROW;
                const int t0 = tree_tiles_before(at - unit, tile_cost, s.tiles);
                const int t1 = to >= unit + unit_cost ? s.tiles : tree_tiles_before(to - unit, tile_cost, s.tiles);
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
                if (!it.whole && lane == 0) {
                    p.ws.valid[it.slot] = 1;
                    if (t0 == 0) {
                        const int last = tree_cta_of(unit + TREE_COST_UNIT + (long long)(s.tiles - 1) * tile_cost, total, ctas);
                        *reinterpret_cast<int4*>(&p.ws.cut[cta]) = make_int4(it.row0, it.nodes, h, last);
                    }
                }
                break;
            }
            const int j = k & 1;
            if (k >= 2) ok = pfx_warp_wait(&ctl.item_empty[j], (uint32_t)((k - 2) >> 1) & 1u, abort_flag);
            if (!ok) break;
            if (lane == 0) {
                ctl.item[j] = it;
                mbar_arrive(&ctl.item_full[j]);
            }
            __syncwarp();
            if (!it.valid) break;
            if (k >= 1) ok = pfx_warp_wait(&ctl.q_free, (uint32_t)(k - 1) & 1u, abort_flag);
            if (!ok) break;
            if (lane == 0) {
                const int boxes = HALVES * (it.wide ? 2 : 1);
                mbar_arrive_expect_tx(&ctl.q_full, (uint32_t)(boxes * row_bytes));
                for (int x = 0; x < boxes; ++x) {
                    const int s = x / HALVES, half = x % HALVES;
                    tma_load_3d(tree_raw + s * TILE_BYTES + half * HALF_BYTES, &tmQ, &ctl.q_full, half * 64, it.h * p.G, it.row0 + s * p.nodes);
                }
            }
            q_issued = ++k;
        }
      } else if (warp == TREE_K_WARP || warp == TREE_V_WARP) {
        // =============================== loaders: K tiles and V tiles, alternately in the ring ===============================
        const bool is_k = warp == TREE_K_WARP;
        const CUtensorMap* const tm = is_k ? &tmK : &tmV;
        const uint64_t policy = p.reread ? l2_evict_normal_policy() : l2_evict_first_policy();
        const int box_rows = min(p.page_size, TREE_TILE), boxes = TREE_TILE / box_rows * HALVES;
        const int piece = lane / HALVES, half = lane % HALVES;     // this lane's box: a page (or part of one) and a half
        bool ok = true;
        int n = 0;                                                 // tiles of earlier items
        for (int k = 0; ok; ++k) {
            const int j = k & 1;
            ok = pfx_warp_wait(&ctl.item_full[j], (uint32_t)(k >> 1) & 1u, abort_flag);
            if (!ok) break;
            const TreeItem it = ctl.item[j];
            if (!is_k && it.valid && lane < HG_MAX_TREE_NODES / 32) ctl.poison[j][lane] = 0;
            __syncwarp();
            if (lane == 0) mbar_arrive(&ctl.item_empty[j]);
            if (!it.valid) break;
            // the block-table entry of this lane's box of tile x, as it comes: nothing looks at it before its tile's turn, so the
            // look-up, two tiles ahead, is not waited for
            struct Box { int e; bool want; };
            auto look_up = [&](int x) -> Box {
                Box v;
                const int t = it.first + x * TREE_TILE + piece * box_rows;
                v.want = lane < boxes && x < it.tiles && t < it.hi && t + box_rows > it.lo;
                v.e = it.b * p.max_pages + (t >> p.page_shift);
                if (v.want && p.block_table) v.e = p.block_table[(size_t)it.b * p.max_pages + (t >> p.page_shift)];
                return v;
            };
            Box b0 = look_up(0), b1 = look_up(1);
            for (int x = 0; x < it.tiles; ++x) {
                const int t_x = it.first + x * TREE_TILE, row = (t_x + piece * box_rows) & (p.page_size - 1);
                const int e = !b0.want ? -1 : ((uint32_t)b0.e < (uint32_t)p.num_pages ? b0.e : -2);      // -1: not wanted, -2: refused
                b0 = b1;
                b1 = look_up(x + 2);
                const int seq = 2 * (n + x) + (is_k ? 0 : 1), slot = seq % S;
                const uint32_t bytes = (uint32_t)__popc(__ballot_sync(0xffffffffu, e >= 0)) * (uint32_t)box_rows * 128u;
                uint32_t bad = 0;
                if (__any_sync(0xffffffffu, e == -2)) {
                    if (e == -2) {
                        bad = ((1u << (box_rows >> 4)) - 1u) << (piece * (box_rows >> 4));
                        if (p.status && is_k) atomicOr(p.status, HG_DEV_BAD_PAGE);
                    }
                    bad = __reduce_or_sync(0xffffffffu, bad);
                }
                if (seq >= S) ok = pfx_warp_wait(&ctl.empty[slot], (uint32_t)(seq / S - 1) & 1u, abort_flag);
                if (!ok || p.test_stall) break;
                // V rows outside the slice, and of refused pages, hold anything (NaN patterns among it) and meet weights of 0, and
                // so do rows of new tokens with those that do not see them: such a tile lands on a barrier of its own and is handed
                // on when those rows are cleared
                const int c_lo = max(it.lo - t_x, 0), c_hi = min(it.hi - t_x, TREE_TILE), c_new = max(min(it.len - t_x, TREE_TILE), c_lo);
                const bool edge = !is_k && (c_lo > 0 || c_hi < TREE_TILE || c_new < TREE_TILE || bad);
                uint64_t* const landed = edge ? &ctl.edge : &ctl.full[slot];
                uint8_t* const tile = ring + slot * TILE_BYTES;
                if (lane == 0) {
                    if (is_k) ctl.bad[(n + x) & 15] = (uint8_t)bad;
                    mbar_arrive_expect_tx(landed, bytes);
                }
                if (e >= 0) tma_load_5d(tile + half * HALF_BYTES + piece * box_rows * 128, tm, landed, 0, row, half, it.h, e, policy);
                if (edge) {
                    ok = pfx_warp_wait(&ctl.edge, edges & 1u, abort_flag);
                    if (!ok) { edge_open = true; break; }
                    ++edges;
                    for (int u = lane; u < TREE_TILE * HALVES * 8; u += 32) {     // whole 128-byte rows: the swizzle does not matter
                        const int r = (u >> 3) % TREE_TILE, hf = (u >> 3) / TREE_TILE;
                        const uint32_t a = smem_u32(tile) + hf * HALF_BYTES + r * 128 + (u & 7) * 16;
                        if (r < c_lo || r >= c_hi || ((bad >> (r >> 4)) & 1u)) sts128_zero(a);
                        else if (r >= c_new && not_finite<BF16>(lds128(a))) {
                            const int node = t_x + r - it.len;
                            atomicOr(&ctl.poison[j][node >> 5], 1u << (node & 31));
                            sts128_zero(a);
                        }
                    }
                    fence_proxy_async();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&ctl.full[slot]);
                }
                issued = n + x + 1;
            }
            n += it.tiles;
            if (p.test_stall) break;
        }
      } else {
        // =============================== tensor-core warp: one thread issues all products ===============================
        if (elect_one()) {
            bool ok = true;
            int n = 0, prev_n = 0;                                 // tiles before this item, and before the previous one
            uint32_t np[2] = {0, 0}, nsc[2] = {0, 0};              // P tiles taken, S tiles computed per stream
            bool held = false;                                     // stream 1's last products of the item before are still to come
            TreeItem it, prev;
            const uint64_t q_desc = tc_smem_desc(smem_u32(tree_raw), 16u, 1024u, 2u);
            const uint64_t k_desc = tc_smem_desc(smem_u32(ring), 16u, 1024u, 2u);
            const uint64_t v_desc = tc_smem_desc(smem_u32(ring), HALF_BYTES, 1024u, 2u);
            auto scores = [&](int s, int i, bool last) {           // S = Q K^T of a stream's tile
                const int x = n + tree_tile_index(it, s, i), seq = 2 * x, slot = seq % S;
                ok = pfx_wait(&ctl.full[slot], (uint32_t)(seq / S) & 1u, abort_flag);
                if (BESIDE && ok && nsc[s] > 0) ok = pfx_wait(&ctl.s_read[s], (nsc[s] - 1) & 1u, abort_flag);
                if (!ok) return;
                ++nsc[s];
                ctl.stream_bad[s] = ctl.bad[x & 15];
                tc_fence_after_sync();
                const uint64_t a = q_desc + (uint32_t)((it.wide ? s : 0) * (TILE_BYTES >> 4)), b = k_desc + (uint32_t)(slot * (TILE_BYTES >> 4));
                const uint32_t acc = tmem + TREE_S_COL + s * 128;
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk) {              // 16 components: 32 bytes of a 128-byte row, halves apart
                    const uint32_t off = (uint32_t)((kk >> 2) * HALF_BYTES + (kk & 3) * 32) >> 4;
                    tc_mma_f16_ss(acc, a + off, b + off, IDESC_S, kk ? 1u : 0u);
                }
                tc_commit(&ctl.s_full[s]);
                if (!it.wide || s == 1) tc_commit(&ctl.empty[slot]);
                if (last) tc_commit(&ctl.q_free);
                mbar_arrive(&ctl.s_full[s]);
            };
            auto values = [&](const TreeItem& im, int n0, int s, int i) {     // O += P V of a stream's tile, quarter by quarter
                const int x = n0 + tree_tile_index(im, s, i), seq = 2 * x + 1, slot = seq % S;
                ok = pfx_wait(&ctl.full[slot], (uint32_t)(seq / S) & 1u, abort_flag);
                const uint64_t b = v_desc + (uint32_t)(slot * (TILE_BYTES >> 4));
                const uint32_t acc = tmem + TREE_O_COL + s * O_STRIDE, a = tmem + P_COL + s * P_STRIDE;
#pragma unroll
                for (int part = 0; part < 4; ++part) {
                    ok = ok && pfx_wait(&ctl.p_full[s][part], np[s] & 1u, abort_flag);
                    if (!ok) return;
                    tc_fence_after_sync();
#pragma unroll
                    for (int kk = part * 2; kk < part * 2 + 2; ++kk)           // 16 tokens: 8 columns of P
                        tc_mma_f16_ts(acc, a + kk * 8, b + (uint32_t)(kk * 2048 >> 4), IDESC_O, kk ? 1u : (i ? 1u : 0u));
                }
                ++np[s];
                if (!im.wide || s == 1) tc_commit(&ctl.empty[slot]);
                if (BESIDE) tc_commit(&ctl.p_free[s]);
                if (i == tree_stream_tiles(im, s) - 1) tc_commit(&ctl.o_full[s]);
            };
            for (int k = 0; ok; ++k) {
                const int j = k & 1;
                ok = pfx_wait(&ctl.item_full[j], (uint32_t)(k >> 1) & 1u, abort_flag);
                if (!ok) break;
                it = ctl.item[j];
                mbar_arrive(&ctl.item_empty[j]);
                if (!it.valid) break;
                ok = pfx_wait(&ctl.q_full, (uint32_t)k & 1u, abort_flag);
                if (!ok) break;
                const int n0 = tree_stream_tiles(it, 0), n1 = tree_stream_tiles(it, 1);      // n0 >= n1, n0 >= 1
                int left = n0 + n1;                                // score products still to issue
                scores(0, 0, --left == 0);
                if (ok && held) values(prev, prev_n, 1, tree_stream_tiles(prev, 1) - 1);
                held = false;
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
            if (ok && held) values(prev, prev_n, 1, tree_stream_tiles(prev, 1) - 1);
            int none = 0;                                          // nothing is in flight when the tensor memory is given back
            tc_commit(&ctl.drain);
            pfx_wait(&ctl.drain, 0u, &none);
        }
        __syncwarp();
      }
    } else {
        reg_grow<TREE_REGS_SOFTMAX>();
        // =============================== softmax warps: S -> P, epilogue ===============================
        const int s = warp >> 2, w4 = warp & 3;                    // stream, quarter of its rows
        const uint32_t lanes = (uint32_t)(w4 * 32) << 16;
        const uint32_t s_tmem = tmem + TREE_S_COL + s * 128 + lanes, p_tmem = tmem + P_COL + s * P_STRIDE + lanes;
        const uint32_t o_tmem = tmem + TREE_O_COL + s * O_STRIDE + lanes;
        const int r = w4 * 32 + lane;                              // row of the stream
        const int r_node = fast_div(r, p.div_G), r_head = r - r_node * p.G;
        const float sc = p.scale_log2;
        const uint64_t keep = l2_evict_last_policy();
        bool ok = true;
        uint32_t ns = 0, no1 = 0, nj = 0;                          // tiles of this stream, items with tiles of stream 1, joins so far
        auto join_sync = [&]() {                                   // with the other stream's warp of these rows
            __syncwarp();
            if (lane == 0) mbar_arrive(&ctl.join_sync[w4]);
            return pfx_warp_wait(&ctl.join_sync[w4], nj++ & 1u, abort_flag);
        };
        // Round -1 runs a tile's code on whatever stands in tensor memory and hands nothing on, before the wait for the
        // kernel in front of this one: the tile's instructions are in the caches when the first S is there
        for (int k = -1; ok; ++k) {
            const int j = k & 1;
            const bool dry = k < 0;
            int tiles = 1, tiles1 = 0;
            bool exists = true;
            TreeItem it;
            it.wide = 0; it.first = 0; it.lo = 0; it.hi = it.len = TREE_TILE; it.nodes = p.nodes; it.i0 = it.row0 = 0;      // (of the dry round)
            if (!dry) {
                ok = pfx_warp_wait(&ctl.item_full[j], (uint32_t)(k >> 1) & 1u, abort_flag);
                if (!ok) break;
                it = ctl.item[j];
                if (!it.valid) break;
                tiles = tree_stream_tiles(it, s);
                tiles1 = tree_stream_tiles(it, 1);
            }
            const int at = (it.wide ? s * p.nodes : 0) + r_node;    // this row's new token in the unit
            exists = r_node < p.nodes && at < it.nodes;
            const bool live = __any_sync(0xffffffffu, exists);     // some row of this warp exists
            const int node = it.i0 + at, row = it.row0 + at;
            float m_true = NEG_INF, m_ref = NEG_INF, l = 0.f;      // the maximum, and the one the weights refer to (raw logits)
            for (int i = 0; i < tiles; ++i) {
                if (!dry) {
                    ok = pfx_warp_wait(&ctl.s_full[s], ns & 1u, abort_flag);
                    if (!ok) break;
                    ++ns;
                }
                tc_fence_after_sync();
                if (live) {
                    const int t = it.first + tree_tile_index(it, s, i) * TREE_TILE;
                    const int c_lo = max(it.lo - t, 0), c_hi = min(it.hi - t, TREE_TILE);
                    const uint32_t bad = dry ? 0u : *reinterpret_cast<volatile uint8_t*>(&ctl.stream_bad[s]);
                    const bool tail = t + TREE_TILE > it.len, edge = c_lo > 0 || c_hi < TREE_TILE || tail || bad;
                    float x[TREE_TILE];
#pragma unroll
                    for (int c0 = 0; c0 < TREE_TILE; c0 += 32) tmem_ld_32x32(s_tmem + c0, *reinterpret_cast<uint32_t(*)[32]>(&x[c0]));
                    tmem_ld_wait();
                    if (BESIDE) {
                        tc_fence_before_sync();
                        __syncwarp();
                        if (lane == 0 && !dry) mbar_arrive(&ctl.s_read[s]);
                    }
                    if (edge) {                                    // columns outside the slice, of refused pages, of tokens not seen
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
                    // the 16-bit types' comfortable range); the difference is put right at the end.  Each row decides by
                    // itself, so its result does not depend on its neighbours (rows that do not exist among them)
                    const bool moved = (m_true - m_ref) * sc > 8.f;
                    if (BESIDE && !dry && ns > 1) {                // the last tile's weights are used up, and its products in O
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
                                tmem_ld_32x8(o_tmem + c0, y);
                                tmem_ld_wait();
#pragma unroll
                                for (int u = 0; u < 8; ++u) y[u] = __float_as_uint(__uint_as_float(y[u]) * f);
                                tmem_st_32x8(o_tmem + c0, y);
                            }
                        }
                    }
                    const float off = m_ref == NEG_INF ? 0.f : -m_ref * sc;
                    const float2 sc2 = make_float2(sc, sc), off2 = make_float2(off, off);
                    float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
                    // a quarter of the tokens at a time; each is handed over when the next one's weights are computed (a store
                    // into tensor memory takes some 300 cycles to complete while the tensor cores work)
                    auto hand_over = [&](int c) {
                        tmem_st_wait();
                        tc_fence_before_sync();
                        __syncwarp();
                        if (lane == 0 && !dry) mbar_arrive(&ctl.p_full[s][c]);
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
                        if (!dry) tmem_st_32x16(p_tmem + c * 16, w);
                    }
                    hand_over(3);
                    l += (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
                } else {
                    tc_fence_before_sync();
                    __syncwarp();
                    if (BESIDE && lane == 0) mbar_arrive(&ctl.s_read[s]);
                    if (BESIDE && ns > 1) ok = pfx_warp_wait(&ctl.p_free[s], (ns - 2) & 1u, abort_flag);
                    if (!ok) break;
                    if (lane < 4) mbar_arrive(&ctl.p_full[s][lane]);
                }
            }
            if (dry) {
                cudaGridDependencySynchronize();
                continue;
            }
            if (!ok) break;
            // ---- the piece's end.  Stream 0 has a tile always; where the streams share their rows, each takes half of the
            // components of both streams' sums ----
            if (it.wide ? s == 0 : true) ok = pfx_warp_wait(&ctl.o_full[0], (uint32_t)k & 1u, abort_flag);
            if (ok && tiles1 > 0 && (it.wide ? s == 1 : true)) ok = pfx_warp_wait(&ctl.o_full[1], no1 & 1u, abort_flag);
            if (!ok) break;
            if (tiles1 > 0) ++no1;
            tc_fence_after_sync();
            if (live) {
                // sums refer to m_ref, at most 2^8 below the maximum: as good a reference as the maximum itself
                float m_raw = m_ref, f0 = 1.f, f1 = 0.f;           // factors on the two sums
                bool both = false;
                uint32_t o0 = o_tmem, o1 = o_tmem;
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
                    o0 = tmem + TREE_O_COL + lanes;
                    o1 = o0 + O_STRIDE;
                    c_begin = s * (D / 2);
                    c_end = c_begin + D / 2;
                } else if (m_ref == NEG_INF) f0 = 0.f;
                const int head = it.h * p.G + r_head;
                const size_t orow = (size_t)row * p.Hq + head;
                const float m = m_raw == NEG_INF ? NEG_INF : m_raw * p.scale;
                float top = m;
                const bool last_word = it.wide || s == 0;          // who writes the row's single numbers
                // tokens that this row sees and whose V rows are not finite: no finite result
                if (it.hi > it.len && it.first + it.tiles * TREE_TILE > it.len && exists) {
                    for (int w = 0; w * 32 < it.n; ++w) {
                        const uint32_t bad = *reinterpret_cast<volatile uint32_t*>(&ctl.poison[j][w]);
                        if (bad && (bad & tree_word(p, row, node, w))) { f0 = __int_as_float(0x7fc00000); both = false; }
                    }
                }
                float scale0 = f0, scale1 = f1, unit = 1.f;
                if (it.whole && exists) {
                    for (int x = 0; x < p.src.n; ++x)
                        for (int c = 0; c < p.src.nc[x]; ++c) top = fmaxf(top, p.src.m[x][orow * p.src.nc[x] + c]);
                    unit = m == NEG_INF ? 0.f : fast_exp2((m - top) * 1.4426950408889634f);
                    l *= unit;
                    for (int x = 0; x < p.src.n; ++x)
                        for (int c = 0; c < p.src.nc[x]; ++c) {
                            const size_t q = orow * p.src.nc[x] + c;
                            const float hm = p.src.m[x][q];
                            if (hm != NEG_INF) l += p.src.l[x][q] * fast_exp2((hm - top) * 1.4426950408889634f);
                        }
                    if (p.lse && last_word) p.lse[orow] = l == 0.f ? NEG_INF : top + logf(l);
                    unit = l == 0.f ? 0.f : 1.f / l;
                    const float mine_f = m == NEG_INF ? 0.f : fast_exp2((m - top) * 1.4426950408889634f);
                    scale0 = f0 * mine_f * unit;
                    scale1 = f1 * mine_f * unit;
                }
                const size_t prow = (size_t)it.slot * 256 + (it.wide ? s * TREE_TILE : 0) + r;
                if (!it.whole && exists && last_word) { p.ws.m[prow] = m; p.ws.l[prow] = l; }
#pragma unroll 1
                for (int c0 = c_begin; c0 < c_end; c0 += 32) {
                    float y[32];
                    tmem_ld_32x32(o0 + c0, *reinterpret_cast<uint32_t(*)[32]>(&y[0]));
                    tmem_ld_wait();
#pragma unroll
                    for (int u = 0; u < 32; ++u) y[u] = scale0 == 0.f ? 0.f : y[u] * scale0;
                    if (both) {
                        float z[32];
                        tmem_ld_32x32(o1 + c0, *reinterpret_cast<uint32_t(*)[32]>(&z[0]));
                        tmem_ld_wait();
#pragma unroll
                        for (int u = 0; u < 32; ++u) y[u] = scale1 == 0.f ? y[u] : fmaf(z[u], scale1, y[u]);
                    }
                    if (!exists) continue;
                    if (!it.whole) {
#pragma unroll
                        for (int u = 0; u < 32; u += 8) st_global_hint8(p.ws.o + prow * D + c0 + u, *reinterpret_cast<const float(*)[8]>(&y[u]), keep);
                        continue;
                    }
                    for (int x = 0; x < p.src.n; ++x)
                        for (int c = 0; c < p.src.nc[x]; ++c) {
                            const size_t q = orow * p.src.nc[x] + c;
                            const float hm = p.src.m[x][q];
                            if (hm == NEG_INF) continue;           // (its o row is not read)
                            const float w = fast_exp2((hm - top) * 1.4426950408889634f) * unit;
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
                if (!it.wide) {                                    // both streams' sums are read: either may begin anew
                    tc_fence_before_sync();
                    ok = join_sync();
                    if (!ok) break;
                }
            }
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(&ctl.item_empty[j]);
        }
    }
    __syncthreads();
    if (*abort_flag) {                                             // (nobody raises it any more: all threads agree)
        if (lane == 0) {
            if (warp == TREE_K_WARP || warp == TREE_V_WARP) ctl.issued[warp - TREE_K_WARP] = issued;
            if (warp == TREE_V_WARP) ctl.edge_open = edge_open ? (int)(edges & 1u) : -1;
            if (warp == TREE_ITEM_WARP) ctl.q_issued = q_issued;
        }
        __syncthreads();
        // unwinding: copies into this CTA's shared memory may still be on their way.  A warp per slot of the ring, one for the edge
        // barrier and one for the queries, so that the waits' limits do not add up
        if (lane == 0) {
            int none = 0;
            if (warp < S) {
                const int n = ring_last_tile(warp, S, ctl.issued[0], ctl.issued[1]);
                if (n >= 0) pfx_wait(&ctl.full[warp], (uint32_t)(n / S) & 1u, &none);
            }
            if (warp == TREE_MMA_WARP && ctl.edge_open >= 0) pfx_wait(&ctl.edge, (uint32_t)ctl.edge_open, &none);
            if (warp == TREE_ITEM_WARP && ctl.q_issued > 0) pfx_wait(&ctl.q_full, (uint32_t)(ctl.q_issued - 1) & 1u, &none);
        }
        if (tid == 0 && p.status) atomicOr(p.status, HG_DEV_WAIT_TIMEOUT);
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    if (warp == TREE_MMA_WARP) tmem_dealloc(tmem, 512);
}

// Joins the pieces of the units that the ends of the CTAs' stretches cut, and the host's partials.  Grid (CTAs of the kernel in
// front, splits of a unit's rows), a warp per row.
constexpr int TREE_MERGE_THREADS = 256, TREE_MERGE_SPLITS = 16;

template <int D, bool BF16>
__global__ void __launch_bounds__(TREE_MERGE_THREADS) tree_merge_kernel(const __grid_constant__ TreeParams p) {
    constexpr int W = D / 32;                                      // components per lane
    constexpr float LOG2E = 1.4426950408889634f;
    const float NEG_INF = __int_as_float(0xff800000);
    cudaTriggerProgrammaticLaunchCompletion();
    cudaGridDependencySynchronize();
    if (p.status && (*reinterpret_cast<volatile int32_t*>(p.status) & HG_DEV_WAIT_TIMEOUT)) return;
    const int4 cut = *reinterpret_cast<const int4*>(&p.ws.cut[blockIdx.x]);       // row0, nodes, h, last
    if (cut.y <= 0) return;
    const int lane = threadIdx.x & 31, first = blockIdx.x, pieces = cut.w - first + 1, stream_rows = p.nodes * p.G;
    for (int x = blockIdx.y * (TREE_MERGE_THREADS / 32) + (threadIdx.x >> 5); x < cut.y * p.G; x += gridDim.y * (TREE_MERGE_THREADS / 32)) {
        const int node = fast_div(x, p.div_G), s = x >= stream_rows ? 1 : 0;
        const size_t orow = (size_t)(cut.x + node) * p.Hq + cut.z * p.G + (x - node * p.G);
        const int r = s * TREE_TILE + x - s * stream_rows;
        auto slot_of = [&](int e) { return e == 0 ? 2 * first + 1 : 2 * (first + e); };
        float top = NEG_INF;
        for (int e = lane; e < pieces; e += 32)
            if (p.ws.valid[slot_of(e)]) top = fmaxf(top, p.ws.m[(size_t)slot_of(e) * 256 + r]);
        for (int y = 0; y < p.src.n; ++y)
            for (int c = lane; c < p.src.nc[y]; c += 32) top = fmaxf(top, p.src.m[y][orow * p.src.nc[y] + c]);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        float l = 0.f, acc[W];
#pragma unroll
        for (int u = 0; u < W; ++u) acc[u] = 0.f;
        auto add = [&](float m, float pl, const float* o) {
            if (m == NEG_INF) return;                              // (its o row is not read)
            const float w = fast_exp2((m - top) * LOG2E);
            l = fmaf(pl, w, l);
            if constexpr (W == 4) {
                const float4 v = *reinterpret_cast<const float4*>(o + lane * 4);
                acc[0] = fmaf(v.x, w, acc[0]); acc[1] = fmaf(v.y, w, acc[1]); acc[2] = fmaf(v.z, w, acc[2]); acc[3] = fmaf(v.w, w, acc[3]);
            } else {
                const float2 v = *reinterpret_cast<const float2*>(o + lane * 2);
                acc[0] = fmaf(v.x, w, acc[0]); acc[1] = fmaf(v.y, w, acc[1]);
            }
        };
#pragma unroll 4
        for (int e = 0; e < pieces; ++e) {
            const int slot = slot_of(e);
            const size_t q = (size_t)slot * 256 + r;
            if (p.ws.valid[slot]) add(p.ws.m[q], p.ws.l[q], p.ws.o + q * D);
        }
        for (int y = 0; y < p.src.n; ++y)
            for (int c = 0; c < p.src.nc[y]; ++c) {
                const size_t q = orow * p.src.nc[y] + c;
                add(p.src.m[y][q], p.src.l[y][q], p.src.o[y] + q * D);
            }
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
