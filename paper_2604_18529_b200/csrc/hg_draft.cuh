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

struct SlotsParams {
    const int32_t* seq_lens;
    const int32_t* n_new;            // or NULL: one each
    const int32_t* parent;           // packed, or NULL: chains
    const int32_t* table;            // or NULL: identity paging
    int32_t* cu;
    int32_t* seq;
    int32_t* pos;
    int64_t* slot;
    uint32_t* mask;
    int32_t* status;
    int B, N, words, cut;            // cut: the most tokens of a sequence
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

// Grid (sequence ranges, splits of a range's rows).  A CTA sums the lengths in front of its range (reading them takes less
// than a second launch would: 65 535 lengths are 256 KB from the L2), scans its own 256 at a time and fills their rows, a
// thread a row.
__global__ void __launch_bounds__(SLOTS_THREADS) kv_slots_kernel(SlotsParams p) {
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
            if (hi - lo < asked) trouble |= HG_DEV_RANGE;
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
            const int i = r - first_row[k];
            int depth = i;
            uint32_t* const bits = p.mask ? p.mask + (size_t)r * p.words : nullptr;
            if (p.parent) {                                        // up the tree; ancestors come in descending order
                depth = 0;
                int w = i >> 5, node = i;
                uint32_t word = 1u << (i & 31);
                if (bits) for (int z = p.words - 1; z > w; --z) bits[z] = 0;
                for (;;) {
                    const int up = p.parent[first_row[k] + node];
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
            } else if (bits) {
                for (int w = 0; w < p.words; ++w) {
                    const int last = i - w * 32;
                    bits[w] = last >= 31 ? 0xffffffffu : last < 0 ? 0u : (2u << last) - 1u;
                }
            }
            if (p.seq) p.seq[r] = q0 + k;
            if (p.pos) p.pos[r] = length[k] + depth;
            if (p.slot) {
                const long long t = (long long)length[k] + i, page = t >> p.page_shift;
                long long at = -1;
                if (page >= p.max_pages) trouble |= HG_DEV_RANGE;
                else {
                    const long long e = (long long)(q0 + k) * p.max_pages + page, id = p.table ? p.table[e] : e;
                    if (id < 0 || id >= p.num_pages) trouble |= HG_DEV_BAD_PAGE;
                    else at = (id << p.page_shift) + (t & ((1 << p.page_shift) - 1));
                }
                p.slot[r] = at;
            }
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
// error of at most 2^-24 * pi whatever the position.  They are computed once a row and shared by its heads.
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

constexpr int ACCEPT_THREADS = 256, ACCEPT_UNROLL = 8, ACCEPT_MAX_PATH = 1024;

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
    auto place = [&](long long t, int64_t& at) {                   // of position t: 0, or what is wrong with it
        const long long page = t >> pv.page_shift;
        if (page >= pv.max_pages) return HG_DEV_RANGE;
        const long long e = (long long)b * pv.max_pages + page;
        const long long id = pv.block_table ? pv.block_table[e] : e;
        if (id < 0 || id >= pv.num_pages) return HG_DEV_BAD_PAGE;
        at = id * pv.page_stride + (t & (pv.page_size - 1)) * pv.tok_stride;
        return 0;
    };
    int last = p.max_path;                                         // this thread's first bad step
    for (int j = tid; j < n; j += ACCEPT_THREADS) {
        const int x = p.path[(size_t)b * p.max_path + j], above = j > 0 ? p.path[(size_t)b * p.max_path + j - 1] : -1;
        int wrong = x > above && x >= j ? 0 : HG_DEV_RANGE;
        int64_t f = 0, t = 0;
        if (!wrong) wrong = place((long long)len + x, f);
        if (!wrong) wrong = place((long long)len + j, t);
        from[j] = f;
        to[j] = t;
        if (wrong && j < last) { last = j; trouble = wrong; }
    }
    if (last < p.max_path) atomicMin(&kept, last);
    __syncthreads();
    const int keep = max(0, min(n, kept));
    if (trouble && last == keep && p.status) atomicOr(p.status, trouble);
    cluster.sync();                                                // every CTA has read the length, which may be overwritten
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
