// Page management of the paged KV pool (sm_100a): block-table rows that share pages, the pages' reference counts,
// copy on write, compaction, and the copies of page contents these operations ask for.
//
// The only allocator state is ref_count[num_pages]: how many block-table entries (and other holders) use a page.  A page
// is free when its count is 0, and free pages are handed out lowest id first, so every result is a function of the
// arguments alone: no list whose order would depend on timing, no atomic whose order shows.  Table operations are a few
// kilobytes to a few megabytes of integers and bound by latency; copying is bound by HBM.
#pragma once

#include <cooperative_groups.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "hg_poolview.cuh"

namespace hg {

// The kernels below are launched as programmatic dependents of whatever precedes them in the stream: the launch
// itself overlaps the predecessor, nothing is read or written before this returns.  Since a predecessor may still be writing
// what they read, none of their arrays is declared read-only (const with __restrict__): such loads might go through the
// non-coherent path or be moved in front of the wait.
__device__ __forceinline__ void pages_begin() {
    cudaTriggerProgrammaticLaunchCompletion();
    cudaGridDependencySynchronize();
}

// ---- release: one reference less for every listed page ---------------------------------------------------------------

__global__ void __launch_bounds__(256) kv_release_kernel(const int32_t* ids, int n, int32_t* ref, int num_pages, int32_t* status) {
    pages_begin();
    for (unsigned i = blockIdx.x * 256 + threadIdx.x; i < (unsigned)n; i += gridDim.x * 256) {     // (31 bits of entries and a stride)
        const int p = ids[i];
        if (p < 0) continue;
        bool bad = p >= num_pages;
        if (!bad && atomicSub(ref + p, 1) <= 0) { atomicAdd(ref + p, 1); bad = true; }   // released more often than held
        if (bad && status) atomicOr(status, HG_DEV_BAD_PAGE);
    }
}

// ---- cluster-wide scans over the reference counts ----------------------------------------------------------------------

constexpr int PG_THREADS = 1024;
constexpr int PG_WARPS = PG_THREADS / 32;
// The scans go over the counts in groups of 128 whose numbers, one group past the end too, have 31 bits.
constexpr int SCAN_MAX_PAGES = 0x7fffff00;

// Sum over the 32 lanes of the values of lower lanes.
__device__ __forceinline__ int warp_exclusive(int v, int lane, int& total) {
    int x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    total = __shfl_sync(0xffffffffu, x, 31);
    return x - v;
}

// What each CTA of the cluster contributes to the running scan; read by its peers through distributed shared memory.
struct ClusterScan {
    int warp_sum[PG_WARPS];
    int cta_sum;
};

// Exclusive prefix of one value per WARP over all warps of the cluster, in (CTA, warp) order, and the total.
template <int CLUSTER>
__device__ __forceinline__ int cluster_warp_prefix(int v, ClusterScan& s, int rank, int warp, int lane, int& total) {
    namespace cg = cooperative_groups;
    if (lane == 0) s.warp_sum[warp] = v;
    __syncthreads();
    int cta;
    const int mine = warp_exclusive(s.warp_sum[lane], lane, cta);
    int before = __shfl_sync(0xffffffffu, mine, warp);
    total = cta;
    if constexpr (CLUSTER > 1) {
        cg::cluster_group cluster = cg::this_cluster();
        if (threadIdx.x == 0) s.cta_sum = cta;
        cluster.sync();
        total = 0;
#pragma unroll
        for (int r = 0; r < CLUSTER; ++r) {
            const int x = *cluster.map_shared_rank(&s.cta_sum, r);
            if (r < rank) before += x;
            total += x;
        }
    }
    return before;
}

// Orders the cluster's (or the CTA's) global-memory and shared-memory accesses before and after it: the cluster barrier
// releases and acquires at cluster scope, and what CTAs exchange through global memory is written by atomics or plain
// stores and read past the L1 (__ldcg).
template <int CLUSTER>
__device__ __forceinline__ void cluster_sync_all() {
    if constexpr (CLUSTER > 1) cooperative_groups::this_cluster().sync();
    else __syncthreads();
}

// ---- fork: rows of the block table take other rows' pages ----------------------------------------------------------

constexpr int FORK_THREADS = 512;
constexpr int FORK_UNROLL = 4;
constexpr int FORK_SMEM_MAX = 160 * 1024;

struct ForkParams {
    const int32_t* src_row;          // [B]
    int32_t* table;                  // [B][max_pages]
    int32_t* ref;                    // [num_pages]
    int32_t* vec[3];                 // seq_lens, tok_begin, tok_end (NULL: absent, or the same array as one before)
    int32_t* status;
    int B, max_pages, num_pages;
    int cols_shift;                  // log2 of the block-table columns one cluster handles
};

// Columns of the table are independent of one another: a cluster stages its columns of every changed row's new contents in
// shared memory (a share of the rows per CTA), and writes only after all have been read, so rows may be each other's
// sources (a beam step re-orders all rows in place).  Counts move by +1 / -1 per entry; entries that stay the same (the part
// beams have in common) touch no count.  The last cluster moves the per-sequence lengths the same way.
template <int CLUSTER>
__global__ void __launch_bounds__(FORK_THREADS) kv_fork_kernel(const ForkParams p) {
    extern __shared__ int32_t fork_stage[];
    const int tid = threadIdx.x;
    const int rank = (int)blockIdx.x % CLUSTER, tile = (int)blockIdx.x / CLUSTER;
    const int r0 = (int)((long long)p.B * rank / CLUSTER), r1 = (int)((long long)p.B * (rank + 1) / CLUSTER);
    pages_begin();
    if (tile == (int)gridDim.x / CLUSTER - 1) {
        for (int v = 0; v < 3; ++v) {
            if (!p.vec[v]) continue;                       // (uniform)
            for (int b = r0 + tid; b < r1; b += FORK_THREADS) {
                const int s = p.src_row[b];
                if (v == 0 && s >= p.B && p.status) atomicOr(p.status, HG_DEV_RANGE);
                fork_stage[b - r0] = s < 0 ? 0 : p.vec[v][s < p.B ? s : b];
            }
            cluster_sync_all<CLUSTER>();
            for (int b = r0 + tid; b < r1; b += FORK_THREADS) p.vec[v][b] = fork_stage[b - r0];
            __syncthreads();
        }
        return;
    }
    const int cols = 1 << p.cols_shift, c0 = tile << p.cols_shift;
    const int n = (r1 - r0) << p.cols_shift;               // cells of this CTA (n * 4 <= FORK_SMEM_MAX)
    // f(cell number, row, source, column) for this thread's cells, four look-ups of the source rows in flight
    auto for_cells = [&](auto load, auto use) {
        for (int i0 = tid; i0 < n; i0 += FORK_UNROLL * FORK_THREADS) {
            int src[FORK_UNROLL], val[FORK_UNROLL];
#pragma unroll
            for (int u = 0; u < FORK_UNROLL; ++u) {
                const int i = i0 + u * FORK_THREADS, b = r0 + (i >> p.cols_shift), c = c0 + (i & (cols - 1));
                src[u] = i < n && c < p.max_pages ? p.src_row[b] : b;
                if (src[u] >= p.B) src[u] = b;             // unchanged
            }
#pragma unroll
            for (int u = 0; u < FORK_UNROLL; ++u) {
                const int i = i0 + u * FORK_THREADS, b = r0 + (i >> p.cols_shift);
                if (src[u] != b) val[u] = load(b, src[u], c0 + (i & (cols - 1)));
            }
#pragma unroll
            for (int u = 0; u < FORK_UNROLL; ++u) {
                const int i = i0 + u * FORK_THREADS, b = r0 + (i >> p.cols_shift);
                if (src[u] != b) use(i, b, c0 + (i & (cols - 1)), val[u]);
            }
        }
    };
    for_cells([&](int, int s, int c) { return s < 0 ? -1 : p.table[(size_t)s * p.max_pages + c]; },
              [&](int i, int, int, int v) { fork_stage[i] = v; });
    cluster_sync_all<CLUSTER>();
    for_cells([&](int b, int, int c) { return p.table[(size_t)b * p.max_pages + c]; },
              [&](int i, int b, int c, int was) {
                  const int now = fork_stage[i];
                  if (was == now) return;
                  if ((uint32_t)now < (uint32_t)p.num_pages) atomicAdd(p.ref + now, 1);
                  if ((uint32_t)was < (uint32_t)p.num_pages) atomicSub(p.ref + was, 1);
                  p.table[(size_t)b * p.max_pages + c] = now;
              });
}

// The pages a warp looks after: a contiguous range, whole groups of 128 (32 lanes x 4).
struct PageRange { int begin, end; };
template <int CLUSTER>
__device__ __forceinline__ PageRange warp_pages(int num_pages, int rank, int warp) {
    const int groups = (num_pages + 127) / 128;
    const int per = (groups + CLUSTER * PG_WARPS - 1) / (CLUSTER * PG_WARPS);
    const long long b = (long long)(rank * PG_WARPS + warp) * per * 128;
    PageRange r;
    r.begin = (int)(b < num_pages ? b : num_pages);
    r.end = (int)(b + (long long)per * 128 < num_pages ? b + (long long)per * 128 : num_pages);
    return r;
}

// Four counts from p on (a missing one reads as `pad`).  p is a multiple of 4, ref 16-byte aligned.
__device__ __forceinline__ int4 load_refs(const int32_t* ref, int p, int num_pages, int pad) {
    if (p + 3 < num_pages) return __ldcg(reinterpret_cast<const int4*>(ref + p));
    int4 v;
    v.x = p < num_pages ? __ldcg(ref + p) : pad;
    v.y = p + 1 < num_pages ? __ldcg(ref + p + 1) : pad;
    v.z = p + 2 < num_pages ? __ldcg(ref + p + 2) : pad;
    v.w = pad;
    return v;
}

// ---- reserve: pages for the next tokens, copy on write -----------------------------------------------------------------

struct ReserveParams {
    const int32_t* seq_lens;         // [B]
    const int32_t* n_new;            // [B] or NULL: one each
    int32_t* table;
    int32_t* ref;
    int32_t* copy_src;               // [B]
    int32_t* copy_dst;               // [B]
    int32_t* copy_rows;              // [B] or NULL
    int32_t* n_ready;                // [B] or NULL
    int32_t* status;
    int B, max_pages, num_pages, page_shift;
};

constexpr int RESERVE_MAX_BATCH = 16384;
// Free-page ids a CTA of the cluster keeps, and slots one thread can look at: together the pages a call can hand out.
constexpr int RESERVE_IDS_PER_CTA = 32768;
constexpr int RESERVE_MAX_ITER = 32;

// The block-table slots that hold positions [len, len + n_new) of sequence b.
struct SlotRange { int first, count, len, n; bool cut; };
__device__ __forceinline__ SlotRange reserve_slots(const ReserveParams& p, int b) {
    SlotRange r;
    r.len = max(p.seq_lens[b], 0);
    r.n = p.n_new ? p.n_new[b] : 1;
    r.first = r.len >> p.page_shift;
    r.cut = false;
    if (r.n <= 0) { r.n = 0; r.count = 0; return r; }
    const long long room = ((long long)p.max_pages << p.page_shift) - r.len;
    if (r.n > room) { r.cut = true; r.n = (int)(room > 0 ? room : 0); }
    r.count = r.n > 0 ? (int)(((long long)r.len + r.n - 1) >> p.page_shift) - r.first + 1 : 0;
    return r;
}

constexpr int RESERVE_KEEP = 4;      // groups of 128 counts of a warp's range that stay in registers
// Up to this many pages (their counts then fit the registers of one CTA) and slots (one a thread) one CTA does a call alone
// although a cluster was launched, because the host does not know how many slots n_new asks for: 256 slots, 12069
// pages: 8.4 us instead of 12.2; 1090 slots, 6104 pages: 14.5 either way.
constexpr int RESERVE_SOLO_PAGES = RESERVE_KEEP * 128 * PG_WARPS, RESERVE_SOLO_SLOTS = PG_THREADS;

// One cluster does the whole call: its phases (find the shared pages - give up references - find the last writer - rank the
// needs - hand out) depend on one another, and a cluster barrier costs a few hundred nanoseconds where a launch costs
// microseconds.  Every phase is a round trip to the L2 for one slot per thread; so a thread keeps its first slot in
// registers, the counts of its pages of the free scan too, and without a shared page the middle phases are left out.
//
// A page with `refs` references that k sequences of this call are about to write stays with the last of them exactly
// when k = refs (nobody else reads it); all others copy.  That is what serving the sequences one after the other gives.
// In parallel: every writer of a page with more than one reference takes its own off; a count that is still positive says
// that others remain; else the writers leave the largest of their (sequence, slot) numbers there, as -(number + 1).
//
// reserve_phases: everything from the free scan on.  ids: this CTA's share of the free ids, by rank; cum[b]: slots of the
// sequences before b; refs: the first counts of pr, this warp's pages.
template <int CLUSTER>
__device__ __forceinline__ void reserve_phases(const ReserveParams& p, const int wanted, int32_t* const ids, const int32_t* const cum,
                                               const int4 (&refs)[RESERVE_KEEP], const PageRange pr, const int rank,
                                               ClusterScan& scan_a, ClusterScan& scan_b, int& s_carry, int& s_shared) {
    namespace cg = cooperative_groups;
    constexpr int KEEP = RESERVE_KEEP;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    constexpr int LANES = CLUSTER * PG_THREADS;
    const int T = min(wanted, LANES * RESERVE_MAX_ITER);         // later slots are left for another call (n_ready says so)
    const int max_ids = CLUSTER * RESERVE_IDS_PER_CTA;

    // ---- this thread's slots: a contiguous range per warp, consecutive slots on consecutive lanes ----
    const int iters = (T + LANES - 1) / LANES;
    const int first = (rank * PG_WARPS + warp) * iters * 32 + lane;
    auto find_slot = [&](int i, int& b, int& slot) {             // the sequence whose range holds slot number i
        int lo = 0, hi = p.B - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (cum[mid] <= i) lo = mid;
            else hi = mid - 1;
        }
        b = lo;
        slot = (max(p.seq_lens[b], 0) >> p.page_shift) + i - cum[b];
    };
    auto cell = [&](int b, int slot) -> int32_t& { return p.table[(size_t)b * p.max_pages + slot]; };
    int b_0 = 0, slot_0 = 0, e_0 = -1;
    if (first < T) {
        find_slot(first, b_0, slot_0);
        e_0 = cell(b_0, slot_0);
    }
    // f(k, sequence, slot, entry) for every slot of this thread
    auto for_slots = [&](auto f) {
        if (first < T) f(0, b_0, slot_0, e_0);
        for (int k = 1; k < iters; ++k) {
            const int i = first + k * 32;
            if (i >= T) break;
            int b, slot;
            find_slot(i, b, slot);
            f(k, b, slot, cell(b, slot));
        }
    };
    auto number = [&](int b, int slot) { return b * p.max_pages + slot; };
    auto in_pool = [&](int e) { return (uint32_t)e < (uint32_t)p.num_pages; };
    uint32_t need = 0, keep = 0, shared = 0, got = 0;            // one bit per slot
    for_slots([&](int k, int, int, int e) {
        if (!in_pool(e)) return;
        if (__ldcg(p.ref + e) > 1) shared |= 1u << k;
        else keep |= 1u << k;
    });

    // ---- the lowest free ids, by rank, into the CTAs' shared memory ----
    {
        auto free4 = [&](const int4& v) { return (v.x == 0) + (v.y == 0) + (v.z == 0) + (v.w == 0); };
        int mine = 0;
#pragma unroll
        for (int u = 0; u < KEEP; ++u) mine += free4(refs[u]);
        for (int g = pr.begin + KEEP * 128; g < pr.end; g += 128) mine += free4(load_refs(p.ref, g + lane * 4, p.num_pages, 1));
        mine = __reduce_add_sync(0xffffffffu, mine);
        int total;
        int at = cluster_warp_prefix<CLUSTER>(mine, scan_a, rank, warp, lane, total);
        const int limit = min(T, max_ids);
        auto list = [&](const int4& v, int g) {
            const int id = g + lane * 4;
            const int f[4] = {v.x == 0, v.y == 0, v.z == 0, v.w == 0};
            int step;
            int r = at + warp_exclusive(f[0] + f[1] + f[2] + f[3], lane, step);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (f[j] && r < limit) {
                    if constexpr (CLUSTER > 1) cg::this_cluster().map_shared_rank(ids, r & (CLUSTER - 1))[r / CLUSTER] = id + j;
                    else ids[r] = id + j;
                }
                r += f[j];
            }
            at += step;
        };
#pragma unroll
        for (int u = 0; u < KEEP; ++u)
            if (pr.begin + u * 128 < pr.end && at < limit) list(refs[u], pr.begin + u * 128);
        for (int g = pr.begin + KEEP * 128; g < pr.end && at < limit; g += 128) list(load_refs(p.ref, g + lane * 4, p.num_pages, 1), g);
        s_carry = total;                                         // (every thread stores the same value)
    }
    // ---- is any page shared?  (and: the ids are listed, everybody has read the counts) ----
    bool any = __syncthreads_or(shared != 0) != 0;
    const int n_free = min(s_carry, max_ids);
    if constexpr (CLUSTER > 1) {
        if (tid == 0) s_shared = any;
        cg::this_cluster().sync();
        int x = 0;
#pragma unroll
        for (int r = 0; r < CLUSTER; ++r) x |= *cg::this_cluster().map_shared_rank(&s_shared, r);
        any = x != 0;
    }
    if (any) {
        for_slots([&](int k, int, int, int e) { if ((shared >> k) & 1u) atomicSub(p.ref + e, 1); });
        cluster_sync_all<CLUSTER>();
        for_slots([&](int k, int b, int slot, int e) {
            if (((shared >> k) & 1u) && __ldcg(p.ref + e) <= 0) atomicMin(p.ref + e, -(number(b, slot) + 1));
        });
        cluster_sync_all<CLUSTER>();
    }
    int count = 0;
    for_slots([&](int k, int b, int slot, int e) {
        bool n = e < 0;
        if ((shared >> k) & 1u) {
            n = __ldcg(p.ref + e) != -(number(b, slot) + 1);
            if (!n) keep |= 1u << k;
        }
        if (n) { need |= 1u << k; ++count; }
    });
    count = __reduce_add_sync(0xffffffffu, count);
    int needs;
    int at = cluster_warp_prefix<CLUSTER>(count, scan_b, rank, warp, lane, needs);      // (everybody knows who keeps what)
    if (needs > n_free && rank == 0 && tid == 0 && p.status) atomicOr(p.status, HG_DEV_NO_PAGE);
    auto stop_at = [&](int b, int slot) {                         // positions from this slot on are not ready
        if (!p.n_ready) return;
        const long long t = ((long long)slot << p.page_shift) - max(p.seq_lens[b], 0);
        atomicMin(p.n_ready + b, (int)(t > 0 ? t : 0));
    };
    for (int k = 0; k < iters; ++k) {
        const int i = first + k * 32;
        const bool n = (need >> k) & 1u;
        const uint32_t votes = __ballot_sync(0xffffffffu, n);
        const int r = at + __popc(votes & ((1u << lane) - 1u));
        at += __popc(votes);
        if (i >= T) continue;
        int b = b_0, slot = slot_0, e = e_0;
        if (k > 0) {
            find_slot(i, b, slot);
            e = cell(b, slot);
        }
        if (n && r < n_free) {
            got |= 1u << k;
            int id;
            if constexpr (CLUSTER > 1) id = cg::this_cluster().map_shared_rank(ids, r & (CLUSTER - 1))[r / CLUSTER];
            else id = ids[r];
            cell(b, slot) = id;
            p.ref[id] = 1;
            const int len = max(p.seq_lens[b], 0), in_page = len & ((1 << p.page_shift) - 1);
            if (e >= 0 && slot == (len >> p.page_shift) && in_page) {   // the page holds tokens that the sequence keeps
                p.copy_src[b] = e;
                p.copy_dst[b] = id;
                if (p.copy_rows) p.copy_rows[b] = in_page;
            }
        } else if (n) {                                           // no page left: the slot stays as it was
            if (e >= 0) atomicAdd(p.ref + e, 1);
            stop_at(b, slot);
        } else if ((shared >> k) & 1u) {
            atomicAdd(p.ref + e, number(b, slot) + 2);            // the page's new sole owner: back from -(number + 1) to one
        } else if (!((keep >> k) & 1u)) {                         // an entry outside the pool
            if (p.status) atomicOr(p.status, HG_DEV_BAD_PAGE);
            stop_at(b, slot);
        }
    }
    for (int i = T + rank * PG_THREADS + tid; i < wanted; i += LANES) {       // beyond what one call looks at
        int b, slot;
        find_slot(i, b, slot);
        stop_at(b, slot);
    }
    if (needs > n_free) {                                         // (uniform over the cluster)
        cluster_sync_all<CLUSTER>();
        for (int k = 0; k < iters; ++k) {                         // a kept page that a sharer without a copy still reads
            if (!((keep & shared) >> k & 1u)) continue;
            int b, slot;
            find_slot(first + k * 32, b, slot);
            if (__ldcg(p.ref + cell(b, slot)) > 1) stop_at(b, slot);
        }
    }
    if constexpr (CLUSTER > 1) cg::this_cluster().sync();         // peers' shared memory stays until all have read it
}

template <int CLUSTER>
__global__ void __launch_bounds__(PG_THREADS) kv_reserve_kernel(const ReserveParams p) {
    namespace cg = cooperative_groups;
    extern __shared__ int32_t reserve_smem[];
    int32_t* const ids = reserve_smem;                            // this CTA's share of the free ids, by rank
    int32_t* const cum = reserve_smem + RESERVE_IDS_PER_CTA;      // cum[b]: slots of sequences < b
    __shared__ ClusterScan scan_a, scan_b;
    __shared__ int s_warp[PG_WARPS], s_carry, s_shared;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int rank = CLUSTER > 1 ? (int)cg::this_cluster().block_rank() : 0;
    if (tid == 0) s_carry = 0;
    __syncthreads();
    pages_begin();

    // ---- free pages of this warp's range: counted here, listed below (the first 512 counts stay in registers) ----
    int4 refs[RESERVE_KEEP];
    PageRange pr;
    auto load_range = [&](PageRange r) {
        pr = r;
#pragma unroll
        for (int u = 0; u < RESERVE_KEEP; ++u)
            refs[u] = pr.begin + u * 128 < pr.end ? load_refs(p.ref, pr.begin + u * 128 + lane * 4, p.num_pages, 1) : make_int4(1, 1, 1, 1);
    };
    const bool small_pool = CLUSTER > 1 && p.num_pages <= RESERVE_SOLO_PAGES;
    load_range(small_pool ? warp_pages<1>(p.num_pages, 0, warp) : warp_pages<CLUSTER>(p.num_pages, rank, warp));

    // ---- slots per sequence, and what is known without looking at any page ----
    for (int b0 = 0; b0 < p.B; b0 += PG_THREADS) {
        const int b = b0 + tid;
        SlotRange r;
        r.count = 0;
        if (b < p.B) r = reserve_slots(p, b);
        int wt;
        const int ex = warp_exclusive(r.count, lane, wt);
        if (lane == 31) s_warp[warp] = wt;
        __syncthreads();
        int ct;
        const int wx = warp_exclusive(s_warp[lane], lane, ct);
        const int base = s_carry + __shfl_sync(0xffffffffu, wx, warp);
        if (b < p.B) {
            cum[b] = base + ex;
            if (rank == 0) {
                p.copy_src[b] = -1;
                p.copy_dst[b] = -1;
                if (p.copy_rows) p.copy_rows[b] = 0;
                if (p.n_ready) p.n_ready[b] = r.n;
                if (r.cut && p.status) atomicOr(p.status, HG_DEV_RANGE);
            }
        }
        __syncthreads();
        if (tid == 0) s_carry += ct;
        __syncthreads();
    }
    // (B slots' sum fits: max_pages <= 2^31 / B is checked by the host)
    const int wanted = s_carry;
    if constexpr (CLUSTER > 1) {
        if (small_pool && wanted <= RESERVE_SOLO_SLOTS) {          // (every CTA of the cluster comes to the same decision)
            if (rank == 0) reserve_phases<1>(p, wanted, ids, cum, refs, pr, 0, scan_a, scan_b, s_carry, s_shared);
            return;
        }
        if (small_pool) load_range(warp_pages<CLUSTER>(p.num_pages, rank, warp));
    }
    reserve_phases<CLUSTER>(p, wanted, ids, cum, refs, pr, rank, scan_a, scan_b, s_carry, s_shared);
}

// ---- compact: the pages in use move to the low end of the pool ------------------------------------------------------------

struct CompactParams {
    int32_t* ref;
    int32_t* remap;                  // [num_pages]
    int32_t* move_src;               // [max_moves]
    int32_t* move_dst;               // [max_moves]
    int32_t* n_moves;
    int32_t* table;                  // renamed here too if n_table > 0
    int num_pages, max_moves, n_table;
};

// Tables of up to this many entries are renamed by the one CTA that compacts a small pool (400 entries: one launch and some 3 us
// less); a larger one by a kernel of many CTAs.
constexpr int COMPACT_RENAMES = 8192;

// U pages in use.  Holes (free ids below U) are as many as strays (used ids from U on): the k-th lowest hole takes the
// k-th highest stray, so a call that may move only a few pages still shortens the used range from its end.
template <int CLUSTER>
__global__ void __launch_bounds__(PG_THREADS) kv_compact_kernel(const CompactParams p) {
    namespace cg = cooperative_groups;
    __shared__ ClusterScan scan;
    __shared__ int s_below;                                       // pages in use below U
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int rank = CLUSTER > 1 ? (int)cg::this_cluster().block_rank() : 0;
    pages_begin();
    const PageRange pr = warp_pages<CLUSTER>(p.num_pages, rank, warp);
    int mine = 0;
    for (int g = pr.begin; g < pr.end; g += 128) {
        const int4 v = load_refs(p.ref, g + lane * 4, p.num_pages, 0);
        mine += (v.x > 0) + (v.y > 0) + (v.z > 0) + (v.w > 0);
    }
    mine = __reduce_add_sync(0xffffffffu, mine);
    int U;
    const int before = cluster_warp_prefix<CLUSTER>(mine, scan, rank, warp, lane, U);
    // used ids below U: the warp whose range holds U counts; it tells every CTA
    if (U >= pr.begin && U < pr.end) {
        int below = 0;
        for (int g = pr.begin; g < U; g += 128) {
            const int id = g + lane * 4;
            const int4 v = load_refs(p.ref, id, p.num_pages, 0);
            below += (v.x > 0 && id < U) + (v.y > 0 && id + 1 < U) + (v.z > 0 && id + 2 < U) + (v.w > 0 && id + 3 < U);
        }
        below = before + __reduce_add_sync(0xffffffffu, below);
        if (lane == 0) {
            if constexpr (CLUSTER > 1) {
                for (int r = 0; r < CLUSTER; ++r) *cg::this_cluster().map_shared_rank(&s_below, r) = below;
            } else {
                s_below = below;
            }
        }
    } else if (U == p.num_pages && tid == 0) {
        s_below = U;                                              // a full pool: no stray anywhere
    }
    cluster_sync_all<CLUSTER>();
    const int below = s_below, strays = U - below, moves = min(strays, p.max_moves);
    int at = before;                                              // pages in use below this warp's position
    for (int g = pr.begin; g < pr.end; g += 128) {
        const int id0 = g + lane * 4;
        const int4 v = load_refs(p.ref, id0, p.num_pages, 0);
        const bool used4[4] = {v.x > 0, v.y > 0, v.z > 0, v.w > 0};
        int step;
        int used_before = at + warp_exclusive(used4[0] + used4[1] + used4[2] + used4[3], lane, step);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int id = id0 + j;
            if (id < p.num_pages) {
                const int hole = id - used_before, stray = strays - 1 - (used_before - below);
                if (!used4[j] && id < U && hole < moves) p.move_dst[hole] = id;
                if (used4[j] && id >= U && stray < moves) p.move_src[stray] = id;
                p.remap[id] = id;
            }
            used_before += used4[j];
        }
        at += step;
    }
    for (unsigned i = moves + rank * PG_THREADS + tid; i < (unsigned)p.max_moves; i += CLUSTER * PG_THREADS) {
        p.move_src[i] = -1;
        p.move_dst[i] = -1;
    }
    if (rank == 0 && tid == 0) *p.n_moves = moves;
    cluster_sync_all<CLUSTER>();
    for (int i = rank * PG_THREADS + tid; i < moves; i += CLUSTER * PG_THREADS) {   // all pairs are known: move the counts
        const int src = __ldcg(p.move_src + i), dst = __ldcg(p.move_dst + i);
        p.remap[src] = dst;
        p.ref[dst] = __ldcg(p.ref + src);
        p.ref[src] = 0;
    }
    if (CLUSTER > 1 || p.n_table == 0 || moves == 0) return;
    __syncthreads();
    for (int i = tid; i < p.n_table; i += PG_THREADS) {
        const int e = p.table[i];
        if ((uint32_t)e >= (uint32_t)p.num_pages) continue;
        const int to = __ldcg(p.remap + e);
        if (to != e) p.table[i] = to;
    }
}

// Renames the entries of the block table.
__global__ void __launch_bounds__(256) kv_rename_kernel(int32_t* table, size_t n, const int32_t* remap, const int32_t* n_moves, int num_pages) {
    pages_begin();
    if (*n_moves == 0) return;
    const size_t step = (size_t)gridDim.x * 256;
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += step) {
        const int e = table[i];
        if ((uint32_t)e >= (uint32_t)num_pages) continue;
        const int to = remap[e];
        if (to != e) table[i] = to;
    }
}

// ---- copying pages --------------------------------------------------------------------------------------------------------

constexpr int COPY_THREADS = 256;

// A warp per (pair, tensor, KV head): the head's block of a page, 2 to 64 KB, in 16-byte vectors, eight in flight a lane.
// Bound by HBM: 401 MB of 16-token pages in 120 us, read and written (6.7 TB/s; a plain copy here: 6.54).
__global__ void __launch_bounds__(COPY_THREADS) kv_copy_pages_kernel(KvPoolView pv, const int32_t* src, const int32_t* dst,
                                                                      const int32_t* rows, int n, const int32_t* n_dev, int32_t* status) {
    pages_begin();
    const int pairs = n_dev ? max(0, min(*n_dev, n)) : n;
    const int lane = threadIdx.x & 31;
    const int vec_shift = pv.D == 128 ? 4 : 3;                    // 16-byte vectors per row, as a power of two
    const long long units = (long long)pairs * pv.Hkv * 2;
    const long long step = (long long)gridDim.x * (COPY_THREADS / 32);
    for (long long u = (long long)blockIdx.x * (COPY_THREADS / 32) + (threadIdx.x >> 5); u < units; u += step) {
        const int pair = (int)(u / (pv.Hkv * 2)), r = (int)(u - (long long)pair * pv.Hkv * 2);
        const int s = src[pair], d = dst[pair];
        const int nr = rows ? max(0, min(rows[pair], pv.page_size)) : pv.page_size;
        if (s < 0 || d < 0 || nr == 0 || s == d) continue;
        if (s >= pv.num_pages || d >= pv.num_pages) {
            if (lane == 0 && status) atomicOr(status, HG_DEV_BAD_PAGE);
            continue;
        }
        uint16_t* const pool = (r & 1) ? pv.v : pv.k;
        const int64_t head = (int64_t)(r >> 1) * pv.head_stride;
        const uint16_t* const from = pool + (int64_t)s * pv.page_stride + head;
        uint16_t* const to = pool + (int64_t)d * pv.page_stride + head;
        const int nv = nr << vec_shift;
        constexpr int UNROLL = 8;
        for (int base = lane; base < nv; base += 32 * UNROLL) {
            uint4 x[UNROLL];
            int64_t off[UNROLL];
#pragma unroll
            for (int j = 0; j < UNROLL; ++j) {
                const int i = base + 32 * j;
                off[j] = (int64_t)(i >> vec_shift) * pv.tok_stride + (int64_t)(i & ((1 << vec_shift) - 1)) * 8;
                if (i < nv) x[j] = *reinterpret_cast<const uint4*>(from + off[j]);
            }
#pragma unroll
            for (int j = 0; j < UNROLL; ++j)
                if (base + 32 * j < nv) *reinterpret_cast<uint4*>(to + off[j]) = x[j];
        }
    }
}

}  // namespace hg
