// A step's new tokens (sm_100a): which row is which token, rotary positions with the keys' and values' way into the paged
// pool, and the way of the accepted ones to the end of the cache.  Integers, 16-bit vectors and a few sines: bound by launch
// latency when small and by HBM when large.
#pragma once

#include <cooperative_groups.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "hg_device.cuh"
#include "hg_partial.cuh"
#include "hg_poolview.cuh"

namespace hg {

// The kernels below are programmatic dependents of whatever precedes them in the stream: nothing is read or written before
// this returns.  Since a predecessor may still be writing what they read, none of their arrays is declared read-only.
__device__ __forceinline__ void draft_begin() {
    cudaTriggerProgrammaticLaunchCompletion();
    cudaGridDependencySynchronize();
}

// ---- slots: rows, positions, places, masks -----------------------------------------------------------------------------

constexpr int SLOTS_THREADS = 256;
constexpr int SLOTS_SCAN = 2048;           // sequences that every CTA can scan

struct SlotsParams {
    const int32_t* seq_lens;
    const int32_t* n_new;            // or NULL: one each
    const int32_t* n_ready;          // or NULL: all of them
    const int32_t* parent;           // packed, or NULL: chains
    const int32_t* table;            // or NULL: identity paging
    int32_t* cu;
    int32_t* seq;
    int32_t* pos;
    int64_t* slot;
    uint32_t* mask;
    int32_t* status;
    int B, N, words;
    int cut, limit;                  // the most rows of a sequence; with n_ready, the most tokens that have a place
    int per;                         // sequences per CTA
    int page_shift, max_pages, num_pages;
};

// Sum over the block of two numbers (all threads get it).
__device__ __forceinline__ void block_sum2(long long& a, long long& b, long long (*part)[2]) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        a += __shfl_xor_sync(0xffffffffu, a, o);
        b += __shfl_xor_sync(0xffffffffu, b, o);
    }
    __syncthreads();
    if ((threadIdx.x & 31) == 0) { part[threadIdx.x >> 5][0] = a; part[threadIdx.x >> 5][1] = b; }
    __syncthreads();
    a = b = 0;
    for (int w = 0; w < (int)blockDim.x / 32; ++w) { a += part[w][0]; b += part[w][1]; }
}

// Up the tree from token i of the sequence whose rows begin at `first`: the number of its ancestors, and their bits (and its own),
// which come in descending order.  A load a level, one behind the other: random trees are some ln n deep, but a chain given through
// `parent` is n deep (64 sequences of 48 tokens 4.9 us as random trees, 7.5 as such chains; one of 1024 8.4 and 102; 64 of 1024 34 and
// 144).  Without `parent` chains need no walk.
__device__ __forceinline__ int slots_ancestors(const SlotsParams& p, int first, int i, uint32_t* bits, int& trouble) {
    int depth = 0, w = i >> 5, node = i;
    uint32_t word = 1u << (i & 31);
    if (bits) for (int z = p.words - 1; z > w; --z) bits[z] = 0;
    for (;;) {
        const int up = p.parent[first + node];
        if (up >= node) trouble |= HG_DEV_RANGE;
        if (up < 0 || up >= node) break;
        ++depth;
        if (bits && (up >> 5) != w) {
            bits[w] = word;
            for (--w; w > (up >> 5); --w) bits[w] = 0;
            word = 0;
        }
        word |= 1u << (up & 31);
        node = up;
    }
    if (bits) {
        bits[w] = word;
        for (--w; w >= 0; --w) bits[w] = 0;
    }
    return depth;
}

// A token from the sequence's n_ready on (or behind the mask's bits) keeps its row, but has no place and no bits.
// (READY: there is an n_ready.  Asked at run time, the question keeps the four rows of a thread from being looked up together:
// 600 000 rows of 300 sequences 7.8 us instead of 6.9.)
template <bool READY>
__device__ __forceinline__ bool slots_unready(const SlotsParams& p, int b, int i) {
    if constexpr (READY) return i >= min(p.n_ready[b], p.limit);
    return false;
}

// What a row gets: token i of sequence b, whose rows begin at `first` and whose cache has `len` tokens; `entry`: the block-table
// entry of its page, -1 where the table ends.
template <bool READY>
__device__ __forceinline__ void slots_row(const SlotsParams& p, int r, int b, int first, int len, int entry, int& trouble) {
    const int i = r - first;
    int depth = i;
    uint32_t* const bits = p.mask ? p.mask + (size_t)r * p.words : nullptr;
    if (slots_unready<READY>(p, b, i)) {
        depth = 0;
        if (bits) for (int w = 0; w < p.words; ++w) bits[w] = 0;
    } else if (p.parent) depth = slots_ancestors(p, first, i, bits, trouble);
    else if (bits)
        for (int w = 0; w < p.words; ++w) {
            const int last = i - w * 32;
            bits[w] = last >= 31 ? 0xffffffffu : last < 0 ? 0u : (2u << last) - 1u;
        }
    if (p.seq) p.seq[r] = b;
    if (p.pos) p.pos[r] = len + depth;
    if (p.slot) {
        const int in_page = (len + i) & ((1 << p.page_shift) - 1);
        if (entry == -2) trouble |= HG_DEV_BAD_PAGE;
        p.slot[r] = entry < 0 ? -1ll : ((long long)entry << p.page_shift) + in_page;
    }
}
// Block-table entry of token i of a sequence with len cached ones; -1: none, -2: not in the pool.
template <bool READY>
__device__ __forceinline__ int slots_entry(const SlotsParams& p, int b, int len, int i, int& trouble) {
    if (slots_unready<READY>(p, b, i)) return -1;
    const long long page = ((long long)len + i) >> p.page_shift;
    if (page >= p.max_pages) { trouble |= HG_DEV_RANGE; return -1; }
    const long long e = (long long)b * p.max_pages + page;
    const int entry = p.table ? p.table[e] : (int)e;
    return (unsigned)entry < (unsigned)p.num_pages ? entry : -2;
}

// Up to SLOTS_SCAN sequences: every CTA scans all the lengths, which costs less than handing them on, and takes rows in turn, so
// that long and short sequences balance.  Sums are cut at N, which leaves them associative.  QUADS: a thread takes four rows in a
// row (no masks to write, arrays aligned for vectors), else one.  600 000 rows of 300 sequences: 6.4 us; one row a thread 9.5.
template <bool QUADS, bool READY>
__global__ void __launch_bounds__(SLOTS_THREADS) kv_slots_kernel(SlotsParams p) {
    __shared__ unsigned warp_total[SLOTS_THREADS / 32];
    __shared__ int start[SLOTS_SCAN + 1], cached[SLOTS_SCAN];
    draft_begin();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, run = (p.B + SLOTS_THREADS - 1) / SLOTS_THREADS;
    const unsigned N = (unsigned)p.N;
    int trouble = 0;
    unsigned sum = 0;
    for (int b = tid; b < p.B; b += SLOTS_THREADS) {
        cached[b] = max(p.seq_lens[b], 0);
        start[b] = max(p.n_new ? p.n_new[b] : 1, 0);               // (as asked, for now)
    }
    __syncthreads();
    const int b0 = min(p.B, tid * run), b1 = min(p.B, b0 + run);
    for (int b = b0; b < b1; ++b) sum = min(sum + (unsigned)min(start[b], p.cut), N);
    unsigned x = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const unsigned y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x = min(x + y, N);
    }
    if (lane == 31) warp_total[warp] = x;
    unsigned upto = __shfl_up_sync(0xffffffffu, x, 1);
    if (lane == 0) upto = 0;
    __syncthreads();
    for (int w = 0; w < warp; ++w) upto = min(upto + warp_total[w], N);
    for (int b = b0; b < b1; ++b) {
        const int asked = start[b];
        const unsigned next = min(upto + (unsigned)min(asked, p.cut), N);
        start[b] = (int)upto;
        if ((next - upto < (unsigned)asked || (READY && asked > p.limit)) && blockIdx.x == 0) trouble |= HG_DEV_RANGE;
        upto = next;
        if (b == p.B - 1) start[p.B] = (int)next;
    }
    __syncthreads();
    if (blockIdx.x == 0) for (int b = tid; b <= p.B; b += SLOTS_THREADS) p.cu[b] = start[b];
    const int total = start[p.B];
    constexpr int ROWS = QUADS ? 4 : 1;
    for (long long r0 = ((long long)blockIdx.x * SLOTS_THREADS + tid) * ROWS; r0 < p.N; r0 += (long long)gridDim.x * SLOTS_THREADS * ROWS) {
        int k = 0;
        if (r0 < total)
            for (int above = p.B; above - k > 1;) {                // the last sequence that starts at or before the row
                const int mid = (k + above) >> 1;
                if (start[mid] <= (int)r0) k = mid; else above = mid;
            }
        if constexpr (QUADS) {
            __align__(16) int seq[4], pos[4];
            __align__(16) long long slot[4];
            int entry[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                seq[u] = -1; pos[u] = 0; slot[u] = -1;
                if (r0 + u >= total) continue;
                const int r = (int)r0 + u;
                while (start[k + 1] <= r) ++k;
                seq[u] = k;
                pos[u] = cached[k] + (slots_unready<READY>(p, k, r - start[k]) ? 0 : r - start[k]);
                if (p.slot) entry[u] = slots_entry<READY>(p, k, cached[k], r - start[k], trouble);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                if (!p.slot || seq[u] < 0) continue;
                if (entry[u] == -2) trouble |= HG_DEV_BAD_PAGE;
                if (entry[u] >= 0) slot[u] = ((long long)entry[u] << p.page_shift) + (pos[u] & ((1 << p.page_shift) - 1));
            }
            if (r0 + 4 <= p.N) {
                if (p.seq) *reinterpret_cast<int4*>(p.seq + r0) = *reinterpret_cast<const int4*>(seq);
                if (p.pos) *reinterpret_cast<int4*>(p.pos + r0) = *reinterpret_cast<const int4*>(pos);
                if (p.slot) {
                    *reinterpret_cast<longlong2*>(p.slot + r0) = *reinterpret_cast<const longlong2*>(slot);
                    *reinterpret_cast<longlong2*>(p.slot + r0 + 2) = *reinterpret_cast<const longlong2*>(slot + 2);
                }
            } else
                for (int u = 0; r0 + u < p.N; ++u) {
                    if (p.seq) p.seq[r0 + u] = u == 0 ? seq[0] : u == 1 ? seq[1] : seq[2];
                    if (p.pos) p.pos[r0 + u] = u == 0 ? pos[0] : u == 1 ? pos[1] : pos[2];
                    if (p.slot) p.slot[r0 + u] = u == 0 ? slot[0] : u == 1 ? slot[1] : slot[2];
                }
        } else if (r0 < total) {
            const int r = (int)r0, entry = p.slot ? slots_entry<READY>(p, k, cached[k], r - start[k], trouble) : -1;
            slots_row<READY>(p, r, k, start[k], cached[k], entry, trouble);
        } else {                                                   // behind the last token
            if (p.seq) p.seq[r0] = -1;
            if (p.pos) p.pos[r0] = 0;
            if (p.slot) p.slot[r0] = -1;
            if (p.mask) for (int w = 0; w < p.words; ++w) p.mask[(size_t)r0 * p.words + w] = 0;
        }
    }
    if (trouble && p.status) atomicOr(p.status, trouble);
}

// More sequences than that.  Grid (sequence ranges, splits of a range's rows).  A CTA sums the lengths in front of its range
// (reading them takes less than a second launch would: 65 535 lengths are 256 KB from the L2), scans its own 256 at a time and
// fills their rows, a thread a row.
template <bool READY>
__global__ void __launch_bounds__(SLOTS_THREADS) kv_slots_many_kernel(SlotsParams p) {
    __shared__ long long part[SLOTS_THREADS / 32][2];
    __shared__ long long warp_total[SLOTS_THREADS / 32];
    __shared__ int first_row[SLOTS_THREADS], length[SLOTS_THREADS];
    __shared__ int end_row;
    draft_begin();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int s0 = min(p.B, (int)blockIdx.x * p.per), s1 = min(p.B, s0 + p.per);
    auto wanted = [&](int b) { return max(p.n_new ? p.n_new[b] : 1, 0); };
    long long before = 0, all = 0;
    for (int b = tid; b < p.B; b += SLOTS_THREADS) {
        const int n = min(wanted(b), p.cut);
        all += n;
        if (b < s0) before += n;
    }
    block_sum2(before, all, part);
    int trouble = 0;
    for (int q0 = s0; q0 < s1; q0 += SLOTS_THREADS) {
        const int b = q0 + tid;
        const bool mine = b < s1;
        const int asked = mine ? wanted(b) : 0, n = min(asked, p.cut);
        long long x = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, x, o);
            if (lane >= o) x += y;
        }
        if (lane == 31) warp_total[warp] = x;
        __syncthreads();                                           // (the last round's rows are done with first_row too)
        long long start = before + x - n;
        for (int w = 0; w < warp; ++w) start += warp_total[w];
        for (int w = 0; w < SLOTS_THREADS / 32; ++w) before += warp_total[w];
        const int lo = (int)min(start, (long long)p.N), hi = (int)min(start + n, (long long)p.N);
        first_row[tid] = lo;
        length[tid] = mine ? max(p.seq_lens[b], 0) : 0;
        if (tid == SLOTS_THREADS - 1) end_row = hi;
        if (mine && blockIdx.y == 0) {
            p.cu[b] = lo;
            if (b == p.B - 1) p.cu[p.B] = hi;
            if (hi - lo < asked || (READY && asked > p.limit)) trouble |= HG_DEV_RANGE;
        }
        __syncthreads();
        const int n_seqs = min(SLOTS_THREADS, s1 - q0);
        for (long long row = first_row[0] + (long long)blockIdx.y * SLOTS_THREADS + tid; row < end_row; row += (long long)gridDim.y * SLOTS_THREADS) {
            const int r = (int)row;
            int k = 0;                                             // the last sequence that starts at or before the row
            for (int above = n_seqs; above - k > 1;) {
                const int mid = (k + above) >> 1;
                if (first_row[mid] <= r) k = mid; else above = mid;
            }
            const int entry = p.slot ? slots_entry<READY>(p, q0 + k, length[k], r - first_row[k], trouble) : -1;
            slots_row<READY>(p, r, q0 + k, first_row[k], length[k], entry, trouble);
        }
    }
    // rows behind the last token
    const long long ctas = (long long)gridDim.x * gridDim.y, cta = (long long)blockIdx.y * gridDim.x + blockIdx.x;
    for (long long r = min(all, (long long)p.N) + cta * SLOTS_THREADS + tid; r < p.N; r += ctas * SLOTS_THREADS) {
        if (p.seq) p.seq[r] = -1;
        if (p.pos) p.pos[r] = 0;
        if (p.slot) p.slot[r] = -1;
        if (p.mask) for (int w = 0; w < p.words; ++w) p.mask[(size_t)r * p.words + w] = 0;
    }
    if (trouble && p.status) atomicOr(p.status, trouble);
}

// ---- rotary positions, keys and values to their places -------------------------------------------------------------------

constexpr int ROPE_THREADS = 256, ROPE_UNROLL = 2;

struct RopeParams {
    const uint16_t* q;               // or NULL
    const uint16_t* k;               // or NULL: no pool
    const uint16_t* v;
    uint16_t* q_out;
    KvPoolView pv;
    const int32_t* pos;
    const int64_t* slot;
    const double* freq;
    int32_t* status;
    int64_t q_stride, q_out_stride, k_stride, v_stride, places;
    int Hq, Hkv, D, rot;
    float magnitude, sign;           // sign -1: turn back
    int head_units, units;           // of a rotated head, of a row
    FastDiv div_head;
};

// A row's units are 16-byte vectors, or pairs of vectors that turn with each other (HALF), of its query heads, key heads and
// value heads.  Angles are a product of 64 bits whose whole turns are dropped before sine and cosine are taken in fp32: an
// error of at most 2^-24 * pi up to some 10^8 turns; beyond, the product's own roundings count (2^-51 of the angle: 2^-20 for the
// fastest pair at position 2^31).  They are computed once a row and shared by its heads.
//
// Bound by HBM, every byte moved once: 16 384 rows of 40 + 40 heads of 128 take 174 us (1007 MB, 5.8 TB/s, 90 % of a plain copy's
// rate); two units a thread are requested before the angles are computed and 6 to 8 CTAs share an SM.  1024 rows of 64 + 8 heads
// 11.4 us in a loop and 9.5 in a captured graph (42 MB: 6.5); a row's units are split over CTAs where there are few rows, else
// some SMs would have a row more than others (12.4 without).  16 rows: 3.6 us, 2.4 in a graph, which is a launch.
template <bool BF16, bool HALF>
__global__ void __launch_bounds__(ROPE_THREADS) kv_append_rope_kernel(RopeParams p) {
    __shared__ float2 turn[64];      // (cosine, sine) of each pair, times the magnitude
    draft_begin();
    const int tid = threadIdx.x;
    const int64_t n = blockIdx.x;
    const int64_t slot = p.k ? p.slot[n] : -1;
    const bool stored = slot >= 0 && slot < p.places;
    if (p.k && slot >= p.places && tid == 0 && blockIdx.y == 0 && p.status) atomicOr(p.status, HG_DEV_BAD_PAGE);
    const int64_t place = stored ? (slot >> p.pv.page_shift) * p.pv.page_stride + (slot & (p.pv.page_size - 1)) * p.pv.tok_stride : 0;
    struct Unit { const uint16_t* src; uint16_t* dst; int c; bool turned; };       // c: its first component; dst NULL: nothing to do
    auto unit_of = [&](int u) {
        Unit x = {nullptr, nullptr, 0, false};
        if (u >= p.units) return x;
        const int rotated = (p.Hq + p.Hkv) * p.head_units;
        if (u >= rotated) {                                        // values
            const int e = u - rotated, shift = p.D == 128 ? 4 : 3, h = e >> shift;
            x.c = (e - (h << shift)) * 8;
            if (!stored) return x;
            x.src = p.v + n * p.v_stride + h * p.D;
            x.dst = p.pv.v + place + (int64_t)h * p.pv.head_stride;
            return x;
        }
        int h = fast_div(u, p.div_head);
        const int e = u - h * p.head_units, pairs = HALF ? p.rot / 16 : p.rot / 8;
        x.turned = e < pairs;
        x.c = x.turned ? e * 8 : p.rot + (e - pairs) * 8;
        if (h < p.Hq) {
            x.src = p.q + n * p.q_stride + h * p.D;
            x.dst = p.q_out + n * p.q_out_stride + h * p.D;
        } else if (stored) {
            h -= p.Hq;
            x.src = p.k + n * p.k_stride + h * p.D;
            x.dst = p.pv.k + place + (int64_t)h * p.pv.head_stride;
        }
        return x;
    };
    Unit x[ROPE_UNROLL];
    uint4 a[ROPE_UNROLL], b[ROPE_UNROLL];
    auto load = [&](int u0) {
#pragma unroll
        for (int j = 0; j < ROPE_UNROLL; ++j) {
            x[j] = unit_of(u0 + j * ROPE_THREADS);
            if (!x[j].dst) continue;
            a[j] = *reinterpret_cast<const uint4*>(x[j].src + x[j].c);
            if (HALF && x[j].turned) b[j] = *reinterpret_cast<const uint4*>(x[j].src + x[j].c + p.rot / 2);
        }
    };
    const int step = ROPE_UNROLL * ROPE_THREADS, first = (int)blockIdx.y * step + tid;
    load(first);
    if (tid < p.rot / 2) {
        const double turns = (double)p.pos[n] * (p.freq[tid] * 0.15915494309189533577);
        float s, c;
        sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
        turn[tid] = make_float2(c * p.magnitude, s * p.magnitude * p.sign);
    }
    __syncthreads();
    for (int u0 = first; u0 < p.units + tid; u0 += step * gridDim.y) {
        if (u0 != first) load(u0);
#pragma unroll
        for (int j = 0; j < ROPE_UNROLL; ++j) {
            if (!x[j].dst) continue;
            uint32_t* const lo = reinterpret_cast<uint32_t*>(&a[j]);
            uint32_t* const hi = reinterpret_cast<uint32_t*>(&b[j]);
            if (x[j].turned) {
                if constexpr (HALF) {
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const float2 f = unpack2<BF16>(lo[w]), g = unpack2<BF16>(hi[w]);
                        const float2 t0 = turn[x[j].c + 2 * w], t1 = turn[x[j].c + 2 * w + 1];
                        lo[w] = pack2<BF16>(f.x * t0.x - g.x * t0.y, f.y * t1.x - g.y * t1.y);
                        hi[w] = pack2<BF16>(g.x * t0.x + f.x * t0.y, g.y * t1.x + f.y * t1.y);
                    }
                    *reinterpret_cast<uint4*>(x[j].dst + x[j].c + p.rot / 2) = b[j];
                } else {
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const float2 f = unpack2<BF16>(lo[w]), t = turn[x[j].c / 2 + w];
                        lo[w] = pack2<BF16>(f.x * t.x - f.y * t.y, f.y * t.x + f.x * t.y);
                    }
                }
            }
            *reinterpret_cast<uint4*>(x[j].dst + x[j].c) = a[j];
        }
    }
}

// ---- accepted rows ---------------------------------------------------------------------------------------------------------

constexpr int ACCEPT_THREADS = 256, ACCEPT_UNROLL = 4, ACCEPT_MAX_PATH = 1024;

struct AcceptParams {
    KvPoolView pv;
    const int32_t* path;
    const int32_t* n_accept;
    const int32_t* seq_lens;
    int32_t* new_lens;
    int32_t* status;
    int max_path;
};

// A cluster per sequence.  A thread moves one 16-byte column of a head's rows, token after token: row j comes from row
// path[j] >= j, and the paths ascend, so that a row is read before it is overwritten and no thread meets another's.
// Bound by latency: length, path, table entries and rows follow one another (8 sequences, paths up to 5: 3.7 us, 2.6 in a captured
// graph); 128 sequences, 40 heads, paths up to 16: 11 us, 8.5 in a graph (42 MB: 6.5).
__global__ void __launch_bounds__(ACCEPT_THREADS) kv_accept_kernel(AcceptParams p) {
    namespace cg = cooperative_groups;
    __shared__ int64_t from[ACCEPT_MAX_PATH], to[ACCEPT_MAX_PATH];
    __shared__ int kept;
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = (int)cluster.block_rank(), ranks = (int)cluster.num_blocks(), b = blockIdx.x / ranks, tid = threadIdx.x;
    if (tid == 0) kept = p.max_path;
    __syncthreads();
    draft_begin();
    const KvPoolView& pv = p.pv;
    const int len = max(p.seq_lens[b], 0), n = min(p.n_accept[b], p.max_path);
    int trouble = 0;
    auto entry = [&](long long t) {                                // of position t: a page, or, negative, what is wrong with it
        const long long page = t >> pv.page_shift;
        if (page >= pv.max_pages) return -HG_DEV_RANGE;
        const long long e = (long long)b * pv.max_pages + page;
        const int id = pv.block_table ? pv.block_table[e] : (int)e;
        return (unsigned)id < (unsigned)pv.num_pages ? id : -HG_DEV_BAD_PAGE;
    };
    int last = p.max_path;                                         // this thread's first bad step
    for (int j = tid; j < n; j += ACCEPT_THREADS) {
        const int x = p.path[(size_t)b * p.max_path + j], above = j > 0 ? p.path[(size_t)b * p.max_path + j - 1] : -1;
        const bool ascends = x > above && x >= j;
        const long long f = (long long)len + (ascends ? x : j), t = (long long)len + j;
        const int fe = entry(f), te = entry(t), wrong = !ascends ? HG_DEV_RANGE : fe < 0 ? -fe : te < 0 ? -te : 0;
        from[j] = fe * pv.page_stride + (f & (pv.page_size - 1)) * pv.tok_stride;
        to[j] = te * pv.page_stride + (t & (pv.page_size - 1)) * pv.tok_stride;
        if (wrong && j < last) { last = j; trouble = wrong; }
    }
    if (last < p.max_path) atomicMin(&kept, last);
    __syncthreads();
    const int keep = max(0, min(n, kept));
    if (trouble && last == keep && p.status) atomicOr(p.status, trouble);
    if (p.new_lens == p.seq_lens) cluster.sync();                  // every CTA has read the length before it is overwritten
    if (p.new_lens && rank == 0 && tid == 0) p.new_lens[b] = len + keep;
    const int vecs = pv.D / 8, columns = pv.Hkv * vecs;
    for (int c = rank * ACCEPT_THREADS + tid; c < 2 * columns; c += ranks * ACCEPT_THREADS) {
        const int e = c < columns ? c : c - columns, h = e / vecs;
        uint16_t* const col = (c < columns ? pv.k : pv.v) + (int64_t)h * pv.head_stride + (e - h * vecs) * 8;
        for (int j0 = 0; j0 < keep; j0 += ACCEPT_UNROLL) {
            uint4 x[ACCEPT_UNROLL];
#pragma unroll
            for (int u = 0; u < ACCEPT_UNROLL; ++u)
                if (j0 + u < keep) x[u] = *reinterpret_cast<const uint4*>(col + from[j0 + u]);
#pragma unroll
            for (int u = 0; u < ACCEPT_UNROLL; ++u)
                if (j0 + u < keep && from[j0 + u] != to[j0 + u]) *reinterpret_cast<uint4*>(col + to[j0 + u]) = x[u];
        }
    }
}

}  // namespace hg
