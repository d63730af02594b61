// Softmax partials over a prefix that several sequences share, computed once for all of them (sm_100a).
//
// Group g of sequences reads the tokens [begin_g, end_g) of ONE block-table row.  For a KV head the queries of the
// group's members, G per member, are the rows of a matrix Q (R = members x G rows), and per chunk of tokens
//     S = Q K^T,   m = row max of scale S,   P = e^{scale S - m},   l = row sum of P,   o = P V
// is what hg_attn_partial computes for one sequence at a time, with K and V read once instead of once per member.
// Both products run on tcgen05.mma with their accumulators in tensor memory; P is carried as hi + lo 16-bit terms (two
// products; three for bf16 with 64 components), so the arithmetic is 1.5 times (twice) that of the formulas: up to about 164 rows
// per KV head (123) the stream of K and V from HBM is the bound at the measured rates, above that the tensor cores.
//
// One CTA per SM, persistent.  It runs two STREAMS, each with 128 rows: a tile of 128 tokens is S (128 x 128 fp32 in
// tensor memory), turned by the stream's four softmax warps (a thread owns a row) into P in the same columns (32 columns
// of S give 16 of hi and 16 of lo terms), which is the A operand of P V.  While one stream's warps do exponentials, the
// tensor cores work for the other.  A work item is
//   wide    (group, chunk, KV head, 256 rows; the streams share every K and V tile), for more than 128 rows;
//   narrow  (group, two chunks, KV head, up to 128 rows; the streams share Q and take a chunk each).
// So few rows never leave a stream idle, and no stream's result has to be combined with the other's.
//
// Roles: warps 0-7 softmax and epilogue; 8 and 9 load K and V tiles (TMA, a page of 16 to 128 tokens and 64 components
// a box, a ring of tiles that alternates K and V); 10 issues the products; 11 decodes the work items and gathers the
// members; 12-15 gather the query rows.  Every wait is bounded.
//
// Bounds, measured (K and V larger than the L2).  128 sequences, 64/8 heads of 128, 65 536 tokens, bf16, chunks of 2432: 316 us,
// 1.24 of the time of its products at the measured 1613 TFLOP/s (1.85 of the formulas', without lo terms); a tile takes 4100
// cycles where its products (2 of S, 4 of P V) take 3100: a stream's S - row - weights - P V chain is longer than that, and the other stream covers only a part of it (the
// exponentials of both need 2048 cycles of the special-function units).  32 sequences, 131 072 tokens: 176 us.  16
// sequences, 56/56 heads, 16 384 tokens (16 rows a KV head): 87 us for 470 MB, 5.4 TB/s.  4 sequences, 512 tokens: 9.3 us.
// Tiles of 64 tokens with two S buffers a stream, so that the next S never waits for P: 361 instead of 316 us.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "hg_device.cuh"
#include "hg_partial.cuh"
#include "hg_ring.h"
#include "hg_tcgen05.cuh"

namespace hg {

struct PrefixParams {
    const int32_t* block_table;      // [B][max_pages], or NULL: identity paging
    const int32_t* seq_group;        // [B]
    const int32_t* group_row;        // [NG]
    const int32_t* group_begin;      // [NG]
    const int32_t* group_end;        // [NG]
    float* o_part;                   // [B][Hq][NC][D]
    float* m_part;                   // [B][Hq][NC]
    float* l_part;
    int32_t* status;
    int32_t* zero;                   // two words to clear on the way (the work counter of the launch that follows), or NULL
    // the sequences' own tokens, as further items of the same launch (own = 0: not part of it)
    const int32_t* seq_lens;         // [B]
    const int32_t* tok_begin;        // [B]
    const int32_t* tok_end;          // [B]
    float* own_o;                    // [B][Hq][own_NC][D]
    float* own_m;
    float* own_l;
    int own, own_NC, own_C;
    int32_t* cut;                    // [B], or NULL: receives where own slices end that stop with the last of cut_NC chunks of cut_C
    int cut_C, cut_NC;               // tokens (the launch that follows works on longer chunks)
    int B, Hq, Hkv, G, NG, NC, C;
    int page_size, page_shift, max_pages, num_pages;
    int sparse_empty, test_stall;
    float scale, scale_log2;
    FastDiv div_G;
};

// The slice of a group (or a sequence's own one), clamped to its block-table row, and its chunks.
struct GroupSlice { int row, begin, end, nc; bool bad; };

__device__ __forceinline__ GroupSlice own_slice(const PrefixParams& p, int b) {
    GroupSlice s;
    s.row = b;
    s.begin = max(p.tok_begin[b], 0);
    s.end = min(p.tok_end[b], p.seq_lens[b]);
    s.bad = false;
    const long long room = (long long)p.max_pages << p.page_shift;
    if (s.end > room && s.end > s.begin) { s.end = (int)room; s.bad = true; }
    s.nc = s.end > s.begin ? min((s.end - 1) / p.own_C - s.begin / p.own_C + 1, p.own_NC) : 0;
    return s;
}

__device__ __forceinline__ GroupSlice group_slice(const PrefixParams& p, int g) {
    GroupSlice s;
    s.row = p.group_row[g];
    s.begin = max(p.group_begin[g], 0);
    s.end = p.group_end[g];
    s.bad = false;
    const long long room = (long long)p.max_pages << p.page_shift;
    if (s.end > room) { s.end = (int)room; s.bad = true; }
    if (s.end > s.begin && (s.row < 0 || s.row >= p.B)) { s.end = s.begin; s.bad = true; }
    s.nc = s.end > s.begin ? min((s.end - 1) / p.C - s.begin / p.C + 1, p.NC) : 0;
    return s;
}

constexpr int PFX_TILE = 128;                 // tokens per tile, rows per stream
constexpr int PFX_THREADS = 512;
constexpr int PFX_K_WARP = 8, PFX_V_WARP = 9, PFX_MMA_WARP = 10, PFX_ITEM_WARP = 11, PFX_Q_WARP = 12;
constexpr int PFX_REGS_SOFTMAX = 200, PFX_REGS_OTHER = 56;     // 256 threads each: together the 128 x 512 of the launch
constexpr int PFX_MAX_SLOTS = 10;
constexpr int PFX_MAX_GROUPS = 512;
constexpr uint32_t PFX_S_COL = 0, PFX_O_COL = 256;      // tensor memory: S / P of the streams, 128 columns each, then their O
constexpr uint32_t PFX_THIRD_COL = 64;                  // behind O where that has 64 columns: third terms of P

template <int D> __host__ __device__ constexpr int pfx_tile_bytes() { return PFX_TILE * D * 2; }
template <int D> __host__ __device__ constexpr int pfx_slots() { return D == 128 ? 5 : 10; }

// One work item, published by the item warp.
struct PfxItem {
    int valid;                       // 0: no more items
    int own;                         // a sequence's own tokens, not a group's
    int row, h;                      // block-table row, KV head
    int wide;
    int chunk;                       // chunk slot of stream 0 (stream 1: the same, or the next one)
    int r0, rows;                    // first row of the group, rows in this item
    int m0;                          // number of the first member in `members`
    int lo0, lo1, hi0, hi1;          // the streams' tokens
    int tiles0, tiles1;
    __device__ __forceinline__ int lo(int s) const { return s ? lo1 : lo0; }
    __device__ __forceinline__ int hi(int s) const { return s ? hi1 : hi0; }
    __device__ __forceinline__ int tiles(int s) const { return s ? tiles1 : tiles0; }
};

struct PfxCtl {
    uint64_t full[PFX_MAX_SLOTS], empty[PFX_MAX_SLOTS];
    uint64_t s_full[2], p_full[2][4], o_full[2];      // p_full: the quarters of a tile's tokens
    uint64_t edge;
    uint64_t q_full, q_free, drain;
    uint64_t item_full[2], item_empty[2];
    PfxItem item[2];
    uint32_t tmem;
    int abort;
    uint8_t bad[16];                 // per tile, in load order: 16-token pieces of the tile whose page was refused
    uint8_t stream_bad[2];           // the same for the tile a stream's softmax warps are about to read
    uint16_t members[2][256];        // sequences of the item's rows, in ascending order
    uint32_t group_n[PFX_MAX_GROUPS / 2];      // members per group, two 16-bit numbers a word (a batch has less than 2^16 sequences)
    int issued[2], q_issued[4];      // tiles, and items' queries, that the loader warps requested (for the unwinding)
};

template <int D> constexpr size_t pfx_smem_bytes() {
    return (size_t)(2 + pfx_slots<D>()) * pfx_tile_bytes<D>() + sizeof(PfxCtl);
}

// First token of a stream's tile i, and the number of tile (stream s, i) in the order in which tiles are loaded.
__device__ __forceinline__ int pfx_tile_token(const PfxItem& it, int s, int i) { return (it.lo(s) & ~(PFX_TILE - 1)) + i * PFX_TILE; }
__device__ __forceinline__ int pfx_tile_index(const PfxItem& it, int s, int i) {
    if (it.wide) return i;
    return s == 0 ? i + min(i, it.tiles(1)) : min(i + 1, it.tiles(0)) + i;
}
__device__ __forceinline__ int pfx_total_tiles(const PfxItem& it) { return it.wide ? it.tiles(0) : it.tiles(0) + it.tiles(1); }

// Two weights -> packed hi terms (rounded) and packed lo terms (what that left, rounded): at most 2^-17 (bf16) or 2^-22
// (fp16, or 2^-25 outright: its smallest steps) of a weight is lost.
template <bool BF16>
__device__ __forceinline__ void split2(float2 w, uint32_t& hi, uint32_t& lo) {
    hi = pack2<BF16>(w.x, w.y);
    const float2 rest = fma2(unpack2<BF16>(hi), make_float2(-1.f, -1.f), w);
    lo = pack2<BF16>(rest.x, rest.y);
}

template <bool BF16>
__device__ __forceinline__ uint32_t split_third(float2 w, uint32_t hi, uint32_t lo) {      // what hi and lo left
    const float2 minus = make_float2(-1.f, -1.f);
    const float2 rest = fma2(unpack2<BF16>(lo), minus, fma2(unpack2<BF16>(hi), minus, w));
    return pack2<BF16>(rest.x, rest.y);
}

template <int D, bool BF16>
__global__ void __launch_bounds__(PFX_THREADS, 1) prefix_partial_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                                                                         const __grid_constant__ CUtensorMap tmV,
                                                                         const PrefixParams p) {
    constexpr int S = pfx_slots<D>();
    constexpr int TILE_BYTES = pfx_tile_bytes<D>();
    constexpr int HALVES = D / 64;
    constexpr uint32_t HALF_BYTES = PFX_TILE * 128;
    constexpr uint32_t FMT = BF16 ? 1u : 0u;
    // instruction descriptors: fp32 accumulator, 16-bit A and B, M = 128; S: both K-major, N = 128 tokens; O: B (V) with
    // its components contiguous (N-major), N = D
    constexpr uint32_t IDESC_S = (1u << 4) | (FMT << 7) | (FMT << 10) | ((128u >> 3) << 17) | ((128u >> 4) << 24);
    constexpr uint32_t IDESC_O = (1u << 4) | (FMT << 7) | (FMT << 10) | (1u << 16) | (((uint32_t)D >> 3) << 17) | ((128u >> 4) << 24);
    // bf16 weights lose up to 2^-17 in two terms (1.1e-6 of a result of 2 000 tokens); with 64 components tensor memory has
    // room for a third one beside O, which leaves 2^-24 (with 128 the four tiles of S / P and O fill it)
    constexpr bool THIRD = BF16 && D == 64;
    const float NEG_INF = __int_as_float(0xff800000);

    extern __shared__ __align__(1024) uint8_t pfx_raw[];
    uint8_t* const ring = pfx_raw + 2 * TILE_BYTES;                // Q of the two streams in front
    PfxCtl& ctl = *reinterpret_cast<PfxCtl*>(pfx_raw + (2 + S) * TILE_BYTES);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    volatile int* const abort_flag = &ctl.abort;

    if (tid == 0) {
        prefetch_tensormap(&tmQ);
        prefetch_tensormap(&tmK);
        prefetch_tensormap(&tmV);
        for (int i = 0; i < S; ++i) { mbar_init(&ctl.full[i], 1); mbar_init(&ctl.empty[i], 1); }
        for (int s = 0; s < 2; ++s) {
            mbar_init(&ctl.s_full[s], 2);                          // the products' completion, and the tile's description
            for (int c = 0; c < 4; ++c) mbar_init(&ctl.p_full[s][c], 4);
            mbar_init(&ctl.o_full[s], 1);
            mbar_init(&ctl.item_full[s], 1);
            mbar_init(&ctl.item_empty[s], 8 + 3 + 4);
        }
        mbar_init(&ctl.q_full, 4);
        mbar_init(&ctl.q_free, 1);
        mbar_init(&ctl.drain, 1);
        mbar_init(&ctl.edge, 1);
        ctl.abort = 0;
        fence_barrier_init();
    }
    if (warp == PFX_MMA_WARP) {
        tmem_alloc(&ctl.tmem, 512);
        tmem_relinquish();
    }
    for (int g = tid; g < PFX_MAX_GROUPS / 2; g += PFX_THREADS) ctl.group_n[g] = 0;
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(&ctl.tmem);

    int issued = 0, q_issued = 0;                                  // (loaders) tiles, (Q warps) items requested so far
    uint32_t edges = 0;                                            // (V loader) tiles that went over the edge barrier
    bool edge_open = false;                                        // ... and one that is still on its way
    cudaTriggerProgrammaticLaunchCompletion();
    auto timed_out = [&]() { return p.status && (*reinterpret_cast<volatile int32_t*>(p.status) & HG_DEV_WAIT_TIMEOUT); };
    // 512 threads x 128 registers at the launch: the softmax warps, which hold a whole row of S, take 72 from the others
    if (warp >= 8) {
      reg_shrink<PFX_REGS_OTHER>();
      cudaGridDependencySynchronize();
      GroupSlice first_slice;                                      // (item warp) on its way while the members are counted
      first_slice.nc = 0;
      if (warp == PFX_ITEM_WARP && lane < p.NG) first_slice = group_slice(p, lane);
      for (int b = tid - 256; b < p.B; b += 256) {
          const uint32_t g = (uint32_t)p.seq_group[b];
          if (g < (uint32_t)p.NG) atomicAdd(&ctl.group_n[g >> 1], (g & 1) ? 0x10000u : 1u);
      }
      if (blockIdx.x == 0 && p.zero && tid < 258) p.zero[tid - 256] = 0;
      asm volatile("bar.sync 1, 256;" ::: "memory");
      if (timed_out()) {
          // an earlier call ran into its limit: no work until the caller has cleared the word
      } else if (warp == PFX_ITEM_WARP) {
        // =============================== item warp: decodes work items, one ahead ===============================
        // units: the groups, then (where they are part of the launch) the sequences; 32 at a time in the lanes
        const int group_units = (p.NG + 31) & ~31, units = group_units + (p.own ? p.B : 0);
        int ub = 0;                                                // first of the units in the lanes
        long long base = 0;                                        // items of the units before them
        GroupSlice sl = first_slice;
        int R = 0, wide_tiles = 0, narrow_rows = 0, n_items = 0, before = 0, block_items = 0;
        auto load_units = [&]() {
            n_items = 0;
            R = 0;
            const int u = ub + lane;
            if (ub < group_units) {
                if (ub > 0 && u < p.NG) sl = group_slice(p, u);
                if (u < p.NG) R = (int)((ctl.group_n[u >> 1] >> ((u & 1) * 16)) & 0xffffu) * p.G;
            } else if (u < units) {
                sl = own_slice(p, u - group_units);
                R = p.G;
            }
            if (R > 0) {
                const int rem = R % 256;
                wide_tiles = R / 256 + (rem > 128 ? 1 : 0);
                narrow_rows = rem <= 128 ? rem : 0;
                n_items = p.Hkv * (wide_tiles * sl.nc + (narrow_rows > 0 ? (sl.nc + 1) / 2 : 0));
            }
            int x = n_items;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int y = __shfl_up_sync(0xffffffffu, x, o);
                if (lane >= o) x += y;
            }
            before = x - n_items;
            block_items = __shfl_sync(0xffffffffu, x, 31);
        };
        load_units();
        bool ok = true;
        int k = 0;
        for (long long i = blockIdx.x; ok; i += gridDim.x, ++k) {
            while (ub < units && i >= base + block_items) {
                base += block_items;
                ub += 32;
                if (ub < units) load_units();
            }
            const int j = k & 1;
            if (k >= 2) ok = pfx_warp_wait(&ctl.item_empty[j], (uint32_t)((k - 2) >> 1) & 1u, abort_flag);
            if (!ok) break;
            PfxItem& it = ctl.item[j];
            if (ub >= units) {
                if (lane == 0) { it.valid = 0; mbar_arrive(&ctl.item_full[j]); }
                break;
            }
            const int at = (int)(i - base);
            const bool mine = at >= before && at < before + n_items;
            const int src = __ffs(__ballot_sync(0xffffffffu, mine)) - 1;
            const bool own = ub >= group_units;
            int m0 = 0, members = 0;
            if (mine) {
                int e = at - before;
                const int wides = p.Hkv * wide_tiles * sl.nc, C = own ? p.own_C : p.C;
                it.valid = 1;
                it.own = own;
                it.row = sl.row;
                const int chunk0 = sl.begin / C;
                int c;
                if (e < wides) {                                   // row tiles fastest: CTAs side by side read the same tiles
                    const int t = e % wide_tiles; e /= wide_tiles;
                    it.h = e % p.Hkv; c = e / p.Hkv;
                    it.wide = 1;
                    it.r0 = t * 256;
                    it.rows = min(256, R - it.r0);
                } else {
                    e -= wides;
                    it.h = e % p.Hkv; c = e / p.Hkv * 2;
                    it.wide = 0;
                    it.r0 = R / 256 * 256;
                    it.rows = narrow_rows;
                }
                it.chunk = c;
                for (int s = 0; s < 2; ++s) {
                    const int cs = it.wide ? c : c + s;
                    const int lo = max(sl.begin, (chunk0 + cs) * C);
                    const int hi = cs < sl.nc ? (int)min((long long)sl.end, (long long)(chunk0 + cs + 1) * C) : lo;
                    (s ? it.lo1 : it.lo0) = lo;
                    (s ? it.hi1 : it.hi0) = hi;
                    (s ? it.tiles1 : it.tiles0) = hi > lo ? (hi - (lo & ~(PFX_TILE - 1)) + PFX_TILE - 1) / PFX_TILE : 0;
                }
                m0 = it.r0 / p.G;
                members = (it.r0 + it.rows - 1) / p.G - m0 + 1;
                it.m0 = m0;
                if (own) ctl.members[j][0] = (uint16_t)sl.row;
            }
            if (own) {
                __syncwarp();
                if (lane == 0) mbar_arrive(&ctl.item_full[j]);
                continue;
            }
            m0 = __shfl_sync(0xffffffffu, m0, src);
            members = __shfl_sync(0xffffffffu, members, src);
            const int g = ub + src;
            int seen = 0;                                          // members met so far
            for (int b0 = 0; b0 < p.B && seen < m0 + members; b0 += 128) {
                int sg[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) sg[u] = b0 + u * 32 + lane < p.B ? p.seq_group[b0 + u * 32 + lane] : -1;
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const uint32_t in = __ballot_sync(0xffffffffu, sg[u] == g);
                    const int r = seen + __popc(in & ((1u << lane) - 1u)) - m0;
                    if (sg[u] == g && r >= 0 && r < members) ctl.members[j][r] = (uint16_t)(b0 + u * 32 + lane);
                    seen += __popc(in);
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&ctl.item_full[j]);
        }
      } else if (warp == PFX_K_WARP || warp == PFX_V_WARP) {
        // =============================== loaders: K tiles and V tiles, alternately in the ring ===============================
        const bool is_k = warp == PFX_K_WARP;
        const CUtensorMap* const tm = is_k ? &tmK : &tmV;
        const uint64_t policy = l2_evict_first_policy();
        const int box_rows = min(p.page_size, PFX_TILE), boxes = PFX_TILE / box_rows * HALVES;
        const int piece = lane / HALVES, half = lane % HALVES;     // this lane's box: a page (or part of one) and a half
        bool ok = true;
        int n = 0;                                                 // tiles of earlier items
        for (int k = 0; ok; ++k) {
            const int j = k & 1;
            ok = pfx_warp_wait(&ctl.item_full[j], (uint32_t)(k >> 1) & 1u, abort_flag);
            if (!ok) break;
            const PfxItem it = ctl.item[j];
            __syncwarp();
            if (lane == 0) mbar_arrive(&ctl.item_empty[j]);
            if (!it.valid) break;
            const int total = pfx_total_tiles(it), both = min(it.tiles(0), it.tiles(1));
            // the block-table entry of this lane's box of tile x (in load order), as it comes: nothing looks at it before its
            // tile's turn, so the look-up, two tiles ahead, is not waited for
            struct Box { int lo, hi, t, e; bool want; };
            auto look_up = [&](int x) -> Box {
                int s = 0, i = x;
                if (!it.wide) {
                    if (x < 2 * both) { s = x & 1; i = x >> 1; }
                    else { s = it.tiles(0) > both ? 0 : 1; i = x - both; }
                }
                Box v;
                v.lo = it.lo(s); v.hi = it.hi(s);
                v.t = pfx_tile_token(it, s, i);
                const int t = v.t + piece * box_rows;
                v.want = lane < boxes && x < total && t < v.hi && t + box_rows > v.lo;
                v.e = it.row * p.max_pages + (t >> p.page_shift);
                if (v.want && p.block_table) v.e = p.block_table[(size_t)it.row * p.max_pages + (t >> p.page_shift)];
                return v;
            };
            Box b0 = look_up(0), b1 = look_up(1);
            for (int x = 0; x < total; ++x) {
                const int lo_x = b0.lo, hi_x = b0.hi, t_x = b0.t, row = (b0.t + piece * box_rows) & (p.page_size - 1);
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
                // V rows outside the slice, and of refused pages, hold anything (NaN patterns among it) and meet weights of 0:
                // such a tile lands on a barrier of its own and is handed on when those rows are cleared
                const int c_lo = max(lo_x - t_x, 0), c_hi = min(hi_x - t_x, PFX_TILE);
                const bool edge = !is_k && (c_lo > 0 || c_hi < PFX_TILE || bad);
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
                    for (int u = lane; u < PFX_TILE * HALVES * 8; u += 32) {     // whole 128-byte rows: the swizzle does not matter
                        const int r = (u >> 3) % PFX_TILE, hf = (u >> 3) / PFX_TILE;
                        if (r < c_lo || r >= c_hi || ((bad >> (r >> 4)) & 1u)) sts128_zero(smem_u32(tile) + hf * HALF_BYTES + r * 128 + (u & 7) * 16);
                    }
                    fence_proxy_async();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&ctl.full[slot]);
                }
                issued = n + x + 1;
            }
            n += total;
            if (p.test_stall) break;
        }
      } else if (warp == PFX_MMA_WARP) {
        // =============================== tensor-core warp: one thread issues all products ===============================
        if (elect_one()) {
            bool ok = true;
            int n = 0, prev_n = 0;                                 // tiles before this item, and before the previous one
            uint32_t np[2] = {0, 0};                               // P tiles taken per stream
            bool held = false;                                     // stream 1's last products of the item before are still to come
            PfxItem it, prev;
            const uint64_t q_desc = tc_smem_desc(smem_u32(pfx_raw), 16u, 1024u, 2u);
            const uint64_t k_desc = tc_smem_desc(smem_u32(ring), 16u, 1024u, 2u);
            const uint64_t v_desc = tc_smem_desc(smem_u32(ring), HALF_BYTES, 1024u, 2u);
            auto scores = [&](int s, int i, bool last) {           // S = Q K^T of a stream's tile
                const int x = n + pfx_tile_index(it, s, i), seq = 2 * x, slot = seq % S;
                ok = pfx_wait(&ctl.full[slot], (uint32_t)(seq / S) & 1u, abort_flag);
                if (!ok) return;
                ctl.stream_bad[s] = ctl.bad[x & 15];
                tc_fence_after_sync();
                const uint64_t a = q_desc + (uint32_t)((it.wide ? s : 0) * (TILE_BYTES >> 4)), b = k_desc + (uint32_t)(slot * (TILE_BYTES >> 4));
                const uint32_t acc = tmem + PFX_S_COL + s * 128;
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
            auto values = [&](const PfxItem& im, int n0, int s, int i) {       // O += P V of a stream's tile, quarter by quarter
                const int x = n0 + pfx_tile_index(im, s, i), seq = 2 * x + 1, slot = seq % S;
                ok = pfx_wait(&ctl.full[slot], (uint32_t)(seq / S) & 1u, abort_flag);
                const uint64_t b = v_desc + (uint32_t)(slot * (TILE_BYTES >> 4));
                const uint32_t acc = tmem + PFX_O_COL + s * 128, a = tmem + PFX_S_COL + s * 128;
#pragma unroll
                for (int part = 0; part < 4; ++part) {
                    ok = ok && pfx_wait(&ctl.p_full[s][part], np[s] & 1u, abort_flag);
                    if (!ok) return;
                    tc_fence_after_sync();
#pragma unroll
                    for (int kk = part * 2; kk < part * 2 + 2; ++kk) {         // 16 tokens: 8 columns of hi terms, 16 further on their lo terms
                        const uint32_t ac = a + (kk >> 1) * 32 + (kk & 1) * 8;
                        tc_mma_f16_ts(acc, ac, b + (uint32_t)(kk * 2048 >> 4), IDESC_O, kk ? 1u : (i ? 1u : 0u));
                        tc_mma_f16_ts(acc, ac + 16, b + (uint32_t)(kk * 2048 >> 4), IDESC_O, 1u);
                        if constexpr (THIRD) tc_mma_f16_ts(acc, acc + PFX_THIRD_COL + kk * 8, b + (uint32_t)(kk * 2048 >> 4), IDESC_O, 1u);
                    }
                }
                ++np[s];
                if (!im.wide || s == 1) tc_commit(&ctl.empty[slot]);
                if (i == im.tiles(s) - 1) tc_commit(&ctl.o_full[s]);
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
                int left = it.tiles(0) + it.tiles(1);              // score products still to issue
                if (it.tiles(0) > 0) scores(0, 0, --left == 0);
                if (ok && held) values(prev, prev_n, 1, prev.tiles(1) - 1);
                held = false;
                if (ok && it.tiles(1) > 0) scores(1, 0, --left == 0);
                const int steps = max(it.tiles(0), it.tiles(1));
                for (int i = 0; i < steps && ok; ++i) {
                    if (i < it.tiles(0)) {
                        values(it, n, 0, i);
                        if (ok && i + 1 < it.tiles(0)) scores(0, i + 1, --left == 0);
                    }
                    if (ok && i < it.tiles(1)) {
                        if (i + 1 == steps) { held = true; break; }            // behind the next item's first scores
                        values(it, n, 1, i);
                        if (ok && i + 1 < it.tiles(1)) scores(1, i + 1, --left == 0);
                    }
                }
                prev = it;
                prev_n = n;
                n += pfx_total_tiles(it);
            }
            if (ok && held) values(prev, prev_n, 1, prev.tiles(1) - 1);
            int none = 0;                                          // nothing is in flight when the tensor memory is given back
            tc_commit(&ctl.drain);
            pfx_wait(&ctl.drain, 0u, &none);
        }
        __syncwarp();
      } else {
        // =============================== query rows, gathered into the 128-byte-swizzled A tiles ===============================
        // four rows and one 64-component half per lane, by the TMA unit (with 16-byte asynchronous copies the 256 rows of an
        // item took some 7000 cycles, queued behind the epilogue's stores); rows behind the last repeat it
        const int group = (warp - PFX_Q_WARP) * 16 + lane / HALVES, half = lane % HALVES;
        bool ok = true;
        for (int k = 0; ok; ++k) {
            const int j = k & 1;
            ok = pfx_warp_wait(&ctl.item_full[j], (uint32_t)(k >> 1) & 1u, abort_flag);
            if (!ok || !ctl.item[j].valid) break;
            const int rows = ctl.item[j].rows, r0 = ctl.item[j].r0, m0 = ctl.item[j].m0, h = ctl.item[j].h;
            const bool mine = lane < 16 * HALVES && group * 4 < rows;
            int row[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int q = r0 + min(group * 4 + u, rows - 1), m = fast_div(q, p.div_G);
                row[u] = mine ? ctl.members[j][m - m0] * p.Hq + h * p.G + q - m * p.G : 0;
            }
            const uint32_t bytes = (uint32_t)__popc(__ballot_sync(0xffffffffu, mine)) * 512u;
            if (k >= 1) ok = pfx_warp_wait(&ctl.q_free, (uint32_t)(k - 1) & 1u, abort_flag);
            if (!ok) break;
            if (lane == 0) {
                mbar_arrive_expect_tx(&ctl.q_full, bytes);
                mbar_arrive(&ctl.item_empty[j]);
            }
            if (mine)
                tma_gather4(pfx_raw + (group >> 5) * TILE_BYTES + half * HALF_BYTES + (group & 31) * 512, &tmQ, &ctl.q_full, half * 64,
                            row[0], row[1], row[2], row[3]);
            q_issued = k + 1;
        }
      }
    } else {
        reg_grow<PFX_REGS_SOFTMAX>();
        // =============================== softmax warps: S -> P, epilogue ===============================
        const int s = warp >> 2, w4 = warp & 3;                    // stream, quarter of its rows
        const uint32_t lanes = (uint32_t)(w4 * 32) << 16;
        const uint32_t s_tmem = tmem + PFX_S_COL + s * 128 + lanes, o_tmem = tmem + PFX_O_COL + s * 128 + lanes;
        const float sc = p.scale_log2;
        const uint64_t keep = l2_evict_last_policy();
        // slots that hold nothing: sequences without a group, chunks beyond a slice
        auto write_empty = [&](int b, int nc, int NC, float* m_out, float* l_out, float* o_out) {
            const int none = NC - nc;
            for (int i = lane; i < p.Hq * none; i += 32) {
                const size_t slot = ((size_t)b * p.Hq + i / none) * NC + nc + i % none;
                m_out[slot] = NEG_INF;
                l_out[slot] = 0.f;
            }
            if (p.sparse_empty) return;
            for (int i = 0; i < p.Hq * none; ++i) {
                const size_t slot = ((size_t)b * p.Hq + i / none) * NC + nc + i % none;
                if (lane < D / 4) reinterpret_cast<float4*>(o_out + slot * D)[lane] = make_float4(0.f, 0.f, 0.f, 0.f);
            }
        };
        auto write_empties = [&]() {
        for (int b = blockIdx.x * 8 + warp; b < p.B; b += gridDim.x * 8) {
            const uint32_t g = (uint32_t)p.seq_group[b];
            write_empty(b, g < (uint32_t)p.NG ? group_slice(p, (int)g).nc : 0, p.NC, p.m_part, p.l_part, p.o_part);
            if (p.cut && lane == 0)
                p.cut[b] = (int)min((long long)p.tok_end[b], (max(p.tok_begin[b], 0) / p.cut_C + (long long)p.cut_NC) * p.cut_C);
            if (!p.own) continue;
            const GroupSlice sl = own_slice(p, b);
            if (sl.bad && lane == 0 && p.status) atomicOr(p.status, HG_DEV_RANGE);
            write_empty(b, sl.nc, p.own_NC, p.own_m, p.own_l, p.own_o);
        }
        for (int g = blockIdx.x * 256 + tid; g < p.NG; g += gridDim.x * 256)
            if (p.status && group_slice(p, g).bad) atomicOr(p.status, HG_DEV_RANGE);
        };
        bool ok = true;
        uint32_t ns = 0, no = 0;                                   // tiles and items of this stream so far
        // Round -1 runs a tile's code on whatever stands in tensor memory and hands nothing on, before the wait for the
        // kernel in front of this one: the tile's instructions (some 20 KB) are in the caches when the first S is there
        for (int k = -1; ok; ++k) {
            const int j = k & 1;
            const bool dry = k < 0;
            int lo = 0, hi = PFX_TILE, tiles = 1, rows = PFX_TILE, wide = 0;      // (of the dry round)
            if (!dry) {
                ok = pfx_warp_wait(&ctl.item_full[j], (uint32_t)(k >> 1) & 1u, abort_flag);
                if (!ok) break;
                const PfxItem& it = ctl.item[j];
                if (!it.valid) break;
                lo = it.lo(s); hi = it.hi(s); tiles = it.tiles(s); rows = it.rows; wide = it.wide;
            }
            const int first_row = (wide ? s * PFX_TILE : 0) + w4 * 32;
            const bool live = first_row < rows;                    // some row of this warp exists
            const bool exists = first_row + lane < rows;           // this thread's
            float m_true = NEG_INF, m_ref = NEG_INF, l = 0.f;      // the maximum, and the one the weights refer to (raw logits)
            for (int i = 0; i < tiles; ++i) {
                if (!dry) {
                    ok = pfx_warp_wait(&ctl.s_full[s], ns & 1u, abort_flag);
                    if (!ok) break;
                    ++ns;
                }
                tc_fence_after_sync();
                if (live) {
                    const int t = (lo & ~(PFX_TILE - 1)) + i * PFX_TILE;
                    const int c_lo = max(lo - t, 0), c_hi = min(hi - t, PFX_TILE);
                    const uint32_t bad = *reinterpret_cast<volatile uint8_t*>(&ctl.stream_bad[s]);
                    const bool edge = c_lo > 0 || c_hi < PFX_TILE || bad;
                    float x[PFX_TILE];
#pragma unroll
                    for (int c0 = 0; c0 < PFX_TILE; c0 += 32) tmem_ld_32x32(s_tmem + c0, *reinterpret_cast<uint32_t(*)[32]>(&x[c0]));
                    tmem_ld_wait();
                    if (edge) {                                    // columns outside the slice or of refused pages
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            uint32_t out = ((bad >> (2 * c)) & 1u ? 0xffffu : 0u) | ((bad >> (2 * c + 1)) & 1u ? 0xffff0000u : 0u);
                            const int below = c_lo - c * 32, in = c_hi - c * 32;
                            out |= below >= 32 ? ~0u : (below > 0 ? (1u << below) - 1u : 0u);
                            out |= in <= 0 ? ~0u : (in < 32 ? ~0u << in : 0u);
#pragma unroll
                            for (int u = 0; u < 32; ++u) x[c * 32 + u] = (out >> u) & 1u ? NEG_INF : x[c * 32 + u];
                        }
                    }
                    const float mx = row_max<PFX_TILE>(x);
                    m_true = fmaxf(m_true, mx);
                    // a row's sums follow its maximum only when that has moved by more than 2^8 (then the weights would leave
                    // the 16-bit types' comfortable range); the difference is put right at the end.  Each row decides by
                    // itself, so its result does not depend on its neighbours (rows that do not exist among them)
                    const bool moved = (m_true - m_ref) * sc > 8.f;
                    if (__any_sync(0xffffffffu, moved && exists)) {
                        const float r = !moved ? 1.f : m_ref == NEG_INF ? 0.f : fast_exp2((m_ref - m_true) * sc);
                        if (moved) m_ref = m_true;
                        if (i > 0) {
                            l *= r;
#pragma unroll 1
                            for (int c0 = 0; c0 < D; c0 += 8) {
                                uint32_t y[8];
                                tmem_ld_32x8(o_tmem + c0, y);
                                tmem_ld_wait();
#pragma unroll
                                for (int u = 0; u < 8; ++u) y[u] = __float_as_uint(__uint_as_float(y[u]) * r);
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
                        uint32_t w[32], w3[16];
#pragma unroll
                        for (int u = 0; u < 16; ++u) {
                            float2 e = fma2(make_float2(x[c * 32 + 2 * u], x[c * 32 + 2 * u + 1]), sc2, off2);
                            e.x = fast_exp2(e.x);
                            e.y = fast_exp2(e.y);
                            sum[u & 1] = add2(sum[u & 1], e);
                            split2<BF16>(e, w[u], w[16 + u]);
                            if constexpr (THIRD) w3[u] = split_third<BF16>(e, w[u], w[16 + u]);
                        }
                        if (c > 0) hand_over(c - 1);
                        if (!dry) {
                            tmem_st_32x32(s_tmem + c * 32, w);
                            if constexpr (THIRD) tmem_st_32x16(o_tmem + PFX_THIRD_COL + c * 16, w3);
                        }
                    }
                    hand_over(3);
                    l += (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
                } else {
                    tc_fence_before_sync();
                    __syncwarp();
                    if (lane < 4) mbar_arrive(&ctl.p_full[s][lane]);
                }
            }
            if (dry) {
                cudaGridDependencySynchronize();
                if (timed_out()) break;
                write_empties();
                continue;
            }
            if (ok && tiles > 0) {
                ok = pfx_warp_wait(&ctl.o_full[s], no & 1u, abort_flag);
                if (!ok) break;
                ++no;
                tc_fence_after_sync();
                if (live) {
                    const PfxItem& it = ctl.item[j];
                    const int r = it.r0 + first_row + lane;
                    const int m = r / p.G, head = it.h * p.G + r - m * p.G;
                    const int b = exists ? ctl.members[j][m - it.m0] : 0;
                    const bool own = it.own;
                    const size_t slot = ((size_t)b * p.Hq + head) * (own ? p.own_NC : p.NC) + it.chunk + (wide ? 0 : s);
                    float* const dst = (own ? p.own_o : p.o_part) + slot * D;
                    const float f = m_true == NEG_INF ? 0.f : fast_exp2((m_ref - m_true) * sc);
                    if (exists) {
                        (own ? p.own_m : p.m_part)[slot] = m_true == NEG_INF ? NEG_INF : m_true * p.scale;
                        (own ? p.own_l : p.l_part)[slot] = l * f;
                    }
                    {
#pragma unroll 1
                        for (int h = 0; h < D; h += 64) {
                            uint32_t x[64];
                            tmem_ld_32x32(o_tmem + h, *reinterpret_cast<uint32_t(*)[32]>(&x[0]));
                            tmem_ld_32x32(o_tmem + h + 32, *reinterpret_cast<uint32_t(*)[32]>(&x[32]));
                            tmem_ld_wait();
                            if (exists)
#pragma unroll
                            for (int c0 = 0; c0 < 64; c0 += 8) {
                                float y[8];
#pragma unroll
                                for (int u = 0; u < 8; ++u) y[u] = __uint_as_float(x[c0 + u]) * f;
                                st_global_hint8(dst + h + c0, y, keep);
                            }
                        }
                    }
                }
                tc_fence_before_sync();
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&ctl.item_empty[j]);
        }
    }
    __syncthreads();
    if (*abort_flag) {                                             // (nobody raises it any more: all threads agree)
        if (lane == 0) {
            if (warp == PFX_K_WARP || warp == PFX_V_WARP) ctl.issued[warp - PFX_K_WARP] = issued;
            if (warp >= PFX_Q_WARP) ctl.q_issued[warp - PFX_Q_WARP] = q_issued;
        }
        __syncthreads();
        // unwinding: copies into this CTA's shared memory may still be on their way.  A warp per slot of the ring and one for
        // the queries, so that the waits' limits do not add up
        if (lane == 0) {
            int none = 0;
            const int slot = warp < PFX_K_WARP ? warp : warp - 2;      // (the V loader's warp has the edge barrier)
            if (warp != PFX_K_WARP && warp != PFX_V_WARP && slot < S) {
                const int n = ring_last_tile(slot, S, ctl.issued[0], ctl.issued[1]);
                if (n >= 0) pfx_wait(&ctl.full[slot], (uint32_t)(n / S) & 1u, &none);
            }
            if (warp == PFX_V_WARP && edge_open) pfx_wait(&ctl.edge, edges & 1u, &none);
            if (warp == PFX_Q_WARP) {                                  // (the four warps may have stopped an item apart)
                const int items = max(max(ctl.q_issued[0], ctl.q_issued[1]), max(ctl.q_issued[2], ctl.q_issued[3]));
                if (items > 0) pfx_wait(&ctl.q_full, (uint32_t)(items - 1) & 1u, &none);
            }
        }
        if (tid == 0 && p.status) atomicOr(p.status, HG_DEV_WAIT_TIMEOUT);
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    if (warp == PFX_MMA_WARP) tmem_dealloc(tmem, 512);
}

}  // namespace hg
