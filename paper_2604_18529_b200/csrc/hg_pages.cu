// Host side of the page operations declared in include/hybridgen_attn.h: argument validation and launches.
#include "hybridgen_attn.h"

#include <cuda_runtime.h>
#include <string.h>

#include <atomic>

#include "hg_hostutil.h"
#include "hg_pages.cuh"

namespace hg {

// Launches with the programmatic-serialisation attribute (every kernel here waits for its predecessor before its first
// access), as one cluster of `cluster` CTAs where that is more than 1.
template <typename... P, typename... A>
static hg_status launch_pages(void (*kern)(P...), unsigned grid, unsigned threads, size_t smem, int cluster, void* stream, A... args) {
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof cfg);
    cfg.gridDim = dim3(grid); cfg.blockDim = dim3(threads); cfg.dynamicSmemBytes = smem;
    cfg.stream = static_cast<cudaStream_t>(stream);
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    int na = 1;
    if (cluster > 1) {
        attr[na].id = cudaLaunchAttributeClusterDimension;
        attr[na].val.clusterDim.x = (unsigned)cluster; attr[na].val.clusterDim.y = 1; attr[na].val.clusterDim.z = 1;
        ++na;
    }
    cfg.attrs = attr; cfg.numAttrs = (unsigned)na;
    if (cudaLaunchKernelEx(&cfg, kern, args...) != cudaSuccess) { cudaGetLastError(); return HG_ERR_CUDA; }
    return HG_OK;
}

// Once per kernel and device: the opt-in to `most` bytes of dynamic shared memory.  `done` is the kernel's own (a bit per
// device; racing threads set the same attribute).
static hg_status opt_in(const void* kern, size_t most, std::atomic<uint64_t>& done) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) { cudaGetLastError(); return HG_ERR_CUDA; }
    if ((done.load(std::memory_order_acquire) >> dev) & 1u) return HG_OK;
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most) != cudaSuccess) { cudaGetLastError(); return HG_ERR_CUDA; }
    done.fetch_or(1ull << dev, std::memory_order_release);
    return HG_OK;
}

// Pool and table; the operations that change the table need one (with identity paging a row owns its pages for good).
static hg_status check_table(const hg_attn_desc* d) {
    hg_status st = check_pool(d);
    if (st != HG_OK) return st;
    if (!d->block_table) return HG_ERR_INVALID_ARG;
    if ((int64_t)d->batch * d->max_pages > 0x7ffffff0ll) return HG_ERR_UNSUPPORTED;      // a slot's number has 31 bits
    return HG_OK;
}

// Two arrays of `bytes` each that share memory.
static bool overlap(const void* a, const void* b, size_t bytes) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return a && b && (x < y ? y - x : x - y) < bytes;
}

static int sm_count() {
    static std::atomic<int> known[kMaxDevices];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) { cudaGetLastError(); return 0; }
    int sms = known[dev].load(std::memory_order_relaxed);
    if (sms == 0) {
        if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) { cudaGetLastError(); return 0; }
        known[dev].store(sms, std::memory_order_relaxed);
    }
    return sms;
}

}  // namespace hg

using namespace hg;

extern "C" {

hg_status hg_kv_fork(const int32_t* src_row, int32_t* ref_count, int32_t* seq_lens, int32_t* tok_begin, int32_t* tok_end,
                     void* stream, const hg_attn_desc* desc) {
    hg_status st = check_table(desc);
    if (st != HG_OK) return st;
    if (!src_row || !ref_count || !seq_lens) return HG_ERR_INVALID_ARG;
    ForkParams p;
    p.src_row = src_row; p.table = const_cast<int32_t*>(desc->block_table); p.ref = ref_count;
    // one array may stand for several (seq_lens for tok_end, where the GPU holds all tokens): it is moved once.  Arrays that
    // overlap in part, and a src_row that the call would write while it reads it, are refused.
    int32_t* const vec[3] = {seq_lens, tok_begin, tok_end};
    const size_t bytes = (size_t)desc->batch * sizeof(int32_t);
    for (int i = 0; i < 3; ++i) {
        p.vec[i] = vec[i];
        if (overlap(src_row, vec[i], bytes)) return HG_ERR_INVALID_ARG;
        for (int j = 0; j < i; ++j) {
            if (vec[j] == vec[i]) p.vec[i] = nullptr;
            else if (overlap(vec[j], vec[i], bytes)) return HG_ERR_INVALID_ARG;
        }
    }
    p.status = desc->status; p.B = desc->batch; p.max_pages = desc->max_pages; p.num_pages = desc->num_pages;
    // a cluster of 8 CTAs shares a tile's rows once there is work for it (1024 rows of 64 entries: 4.1 us instead of 10.2; 256
    // rows of 502: 5.7 instead of 4.2); 32 columns (128-byte row pieces) a tile where that leaves two CTAs for every SM, down
    // to 8 (one 32-byte sector) for short tables, and fewer only where the rows of the batch fill the shared memory
    const int cluster = p.B >= 512 ? 8 : 1;
    const size_t rows = ((size_t)p.B + cluster - 1) / cluster;
    int shift = 5;
    while (shift > 3 && (p.max_pages >> shift) * cluster < 296) --shift;
    while (shift > 0 && (rows << shift) * 4 > FORK_SMEM_MAX) --shift;
    p.cols_shift = shift;
    const unsigned tiles = (unsigned)((p.max_pages + (1 << shift) - 1) >> shift);
    const size_t smem = (rows << shift) * 4;
    static std::atomic<uint64_t> done1, done8;
    st = cluster == 8 ? opt_in(reinterpret_cast<const void*>(kv_fork_kernel<8>), FORK_SMEM_MAX, done8)
                      : opt_in(reinterpret_cast<const void*>(kv_fork_kernel<1>), FORK_SMEM_MAX, done1);
    if (st != HG_OK) return st;
    return cluster == 8 ? launch_pages(kv_fork_kernel<8>, (tiles + 1) * 8, FORK_THREADS, smem, 8, stream, p)
                        : launch_pages(kv_fork_kernel<1>, tiles + 1, FORK_THREADS, smem, 1, stream, p);
}

hg_status hg_kv_release(const int32_t* page_ids, int32_t n, int32_t* ref_count, void* stream, const hg_attn_desc* desc) {
    hg_status st = check_pool(desc);
    if (st != HG_OK) return st;
    if (!page_ids || !ref_count || n < 0) return HG_ERR_INVALID_ARG;
    if (n == 0) return HG_OK;
    const unsigned grid = (unsigned)((n + 255) / 256);
    return launch_pages(kv_release_kernel, grid < 1024 ? grid : 1024, 256, 0, 1, stream, page_ids, (int)n, ref_count,
                        (int)desc->num_pages, desc->status);
}

hg_status hg_kv_reserve(const int32_t* seq_lens, const int32_t* n_new, int32_t* ref_count, int32_t* copy_src, int32_t* copy_dst,
                        int32_t* copy_rows, int32_t* n_ready, void* stream, const hg_attn_desc* desc) {
    hg_status st = check_table(desc);
    if (st != HG_OK) return st;
    if (!seq_lens || !ref_count || !copy_src || !copy_dst || !aligned16(ref_count)) return HG_ERR_INVALID_ARG;
    if (desc->batch > RESERVE_MAX_BATCH || desc->num_pages > SCAN_MAX_PAGES) return HG_ERR_UNSUPPORTED;
    const size_t bytes = (size_t)desc->batch * sizeof(int32_t);
    const int32_t* const written[4] = {n_ready, copy_src, copy_dst, copy_rows};                 // while others still read these two
    for (const int32_t* w : written)
        if (overlap(w, n_new, bytes) || overlap(w, seq_lens, bytes)) return HG_ERR_INVALID_ARG;
    ReserveParams p;
    p.seq_lens = seq_lens; p.n_new = n_new; p.table = const_cast<int32_t*>(desc->block_table); p.ref = ref_count;
    p.copy_src = copy_src; p.copy_dst = copy_dst; p.copy_rows = copy_rows; p.n_ready = n_ready; p.status = desc->status;
    p.B = desc->batch; p.max_pages = desc->max_pages; p.num_pages = desc->num_pages; p.page_shift = ilog2_exact(desc->page_size);
    const size_t smem = ((size_t)RESERVE_IDS_PER_CTA + desc->batch) * 4;
    static std::atomic<uint64_t> done1, done8;
    constexpr size_t most = ((size_t)RESERVE_IDS_PER_CTA + RESERVE_MAX_BATCH) * 4;
    st = opt_in(reinterpret_cast<const void*>(kv_reserve_kernel<1>), most, done1);
    if (st == HG_OK) st = opt_in(reinterpret_cast<const void*>(kv_reserve_kernel<8>), most, done8);
    if (st != HG_OK) return st;
    // a small pool and table: one CTA (its barriers are cheaper than the cluster's, and it can look at every slot there is)
    if (desc->num_pages <= 8192 && (int64_t)desc->batch * desc->max_pages <= PG_THREADS * RESERVE_MAX_ITER)
        return launch_pages(kv_reserve_kernel<1>, 1, PG_THREADS, smem, 1, stream, p);
    return launch_pages(kv_reserve_kernel<8>, 8, PG_THREADS, smem, 8, stream, p);
}

hg_status hg_kv_compact(int32_t* ref_count, int32_t* remap, int32_t* move_src, int32_t* move_dst, int32_t max_moves,
                        int32_t* n_moves, void* stream, const hg_attn_desc* desc) {
    hg_status st = check_table(desc);
    if (st != HG_OK) return st;
    if (!ref_count || !remap || !move_src || !move_dst || !n_moves || max_moves < 1 || !aligned16(ref_count)) return HG_ERR_INVALID_ARG;
    if (desc->num_pages > SCAN_MAX_PAGES) return HG_ERR_UNSUPPORTED;
    const int sms = sm_count();
    if (sms < 1) return HG_ERR_CUDA;
    CompactParams p;
    p.ref = ref_count; p.remap = remap; p.move_src = move_src; p.move_dst = move_dst; p.n_moves = n_moves;
    p.num_pages = desc->num_pages; p.max_moves = max_moves;
    const size_t n = (size_t)desc->batch * desc->max_pages;
    const bool one = desc->num_pages <= 8192, renames = one && n <= COMPACT_RENAMES;
    p.table = const_cast<int32_t*>(desc->block_table); p.n_table = renames ? (int)n : 0;
    st = one ? launch_pages(kv_compact_kernel<1>, 1, PG_THREADS, 0, 1, stream, p) : launch_pages(kv_compact_kernel<8>, 8, PG_THREADS, 0, 8, stream, p);
    if (st != HG_OK || renames) return st;
    const size_t want = (n + 1023) / 1024, most = (size_t)sms * 8;
    return launch_pages(kv_rename_kernel, (unsigned)(want < most ? want : most), 256, 0, 1, stream, const_cast<int32_t*>(desc->block_table), n,
                        const_cast<const int32_t*>(remap), const_cast<const int32_t*>(n_moves), (int)desc->num_pages);
}

hg_status hg_kv_copy_pages(const int32_t* src, const int32_t* dst, const int32_t* rows, int32_t n, const int32_t* n_dev, void* k_cache,
                           void* v_cache, void* stream, const hg_attn_desc* desc) {
    hg_status st = check_pool(desc);
    if (st != HG_OK) return st;
    if (!src || !dst || !k_cache || !v_cache || n < 0) return HG_ERR_INVALID_ARG;
    if (!aligned16(k_cache) || !aligned16(v_cache)) return HG_ERR_INVALID_ARG;
    if (n == 0) return HG_OK;
    const int sms = sm_count();
    if (sms < 1) return HG_ERR_CUDA;
    const long long units = (long long)n * desc->num_kv_heads * 2, ctas = (units + COPY_THREADS / 32 - 1) / (COPY_THREADS / 32);
    const long long most = (long long)sms * (2048 / COPY_THREADS);
    return launch_pages(kv_copy_pages_kernel, (unsigned)(ctas < most ? ctas : most), COPY_THREADS, 0, 1, stream,
                        pool_view(desc, k_cache, v_cache), src, dst, rows, (int)n, n_dev, desc->status);
}

}  // extern "C"
