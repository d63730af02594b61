// Host side of the attention of a step's new tokens declared in include/hybridgen_attn.h: argument validation and launches.
#include "hybridgen_attn.h"

#include <cuda.h>
#include <cuda_runtime.h>
#include <math.h>
#include <string.h>

#include <atomic>

#include "hg_hostutil.h"
#include "hg_tree.cuh"

namespace hg {

static hg_status check_tree(const hg_attn_desc* d, const hg_tree_desc* t) {
    hg_status st = check_pool(d);
    if (st != HG_OK) return st;
    if (!t || t->struct_size < sizeof(hg_tree_desc)) return HG_ERR_INVALID_ARG;
    if (t->max_nodes < 1 || t->num_rows < 1 || !t->cu_nodes) return HG_ERR_INVALID_ARG;
    if (t->mask && t->mask_words < (t->max_nodes + 31) / 32) return HG_ERR_INVALID_ARG;
    if ((t->q_stride & 7) || (t->q_stride != 0 && t->q_stride < (int64_t)d->num_q_heads * d->head_dim)) return HG_ERR_INVALID_ARG;
    if (t->max_nodes > HG_MAX_TREE_NODES || d->num_q_heads / d->num_kv_heads > 128) return HG_ERR_UNSUPPORTED;
    if ((int64_t)d->max_pages * d->page_size > 0x7fffff00ll) return HG_ERR_UNSUPPORTED;      // token positions have 31 bits,
    if ((int64_t)t->num_rows * d->num_q_heads > 0x7fffffffll) return HG_ERR_UNSUPPORTED;      // and so have rows of out
    return HG_OK;
}

// The queries as a tensor {64 components of a head, head, row}: a box is one half of the components of a KV head's G query heads,
// for the new tokens of a stream.
static hg_status make_query_map(const hg_attn_desc* d, const TreeParams& p, int64_t q_stride, const void* q, CUtensorMap* tq) {
    EncodeTiledFn enc = encode_fn();
    if (!enc) return HG_ERR_CUDA;
    cuuint64_t dims[3] = {(cuuint64_t)d->head_dim, (cuuint64_t)d->num_q_heads, (cuuint64_t)p.N};
    cuuint64_t strides[2] = {(cuuint64_t)d->head_dim * 2u, (cuuint64_t)q_stride * 2u};
    cuuint32_t box[3] = {64, (cuuint32_t)p.G, (cuuint32_t)p.nodes};
    cuuint32_t estr[3] = {1, 1, 1};
    if (enc(tq, d->dtype == HG_DTYPE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void*>(q), dims, strides, box,
            estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
        return HG_ERR_UNSUPPORTED;
    return HG_OK;
}

// Workspace: the cut units' descriptions and flags, then their partials, two slots of 256 rows a CTA.
constexpr int HG_TREE_CTAS = 160;    // the most CTAs (the device has 148 SMs; the workspace is sized without asking it)
struct TreePlan { size_t valid, o, m, l, total; };
static TreePlan plan_tree(int head_dim, int ctas) {
    TreePlan w;
    size_t off = up256((size_t)ctas * sizeof(TreeCut));
    w.valid = off; off += up256((size_t)ctas * 2 * sizeof(int32_t));
    w.o = off; off += (size_t)ctas * 2 * 256 * head_dim * sizeof(float);
    w.m = off; off += (size_t)ctas * 2 * 256 * sizeof(float);
    w.l = off; off += (size_t)ctas * 2 * 256 * sizeof(float);
    w.total = off;
    return w;
}

template <int D, bool BF16, int ROWS>
static hg_status launch_tree(const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv, const TreeParams& p, int ctas, cudaStream_t st, bool pdl) {
    static std::atomic<uint64_t> done;                     // a bit per device: the shared-memory opt-in is in force
    auto kern = tree_kernel<D, BF16, ROWS>;
    constexpr size_t smem = tree_smem_bytes<D, ROWS>();
    static_assert(smem <= 227 * 1024, "shared memory of one SM");
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) { cudaGetLastError(); return HG_ERR_CUDA; }
    if (!((done.load(std::memory_order_acquire) >> dev) & 1u)) {
        if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) { cudaGetLastError(); return HG_ERR_CUDA; }
        done.fetch_or(1ull << dev, std::memory_order_release);
    }
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof cfg);
    cfg.gridDim = dim3((unsigned)ctas); cfg.blockDim = dim3(tree_threads<ROWS>()); cfg.dynamicSmemBytes = smem; cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr; cfg.numAttrs = pdl ? 1 : 0;
    if (cudaLaunchKernelEx(&cfg, kern, tq, tk, tv, p) != cudaSuccess) { cudaGetLastError(); return HG_ERR_CUDA; }
    // (a row of a cut unit for a warp; with many rows two)
    cfg.gridDim = dim3((unsigned)ctas, ROWS ? ROWS / 8 : 16); cfg.blockDim = dim3(TREE_MERGE_THREADS); cfg.dynamicSmemBytes = 0;
    if (cudaLaunchKernelEx(&cfg, tree_merge_kernel<D, BF16>, p) != cudaSuccess) { cudaGetLastError(); return HG_ERR_CUDA; }
    return HG_OK;
}

template <int D, bool BF16>
static hg_status launch_tree_rows(int rows, const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv, const TreeParams& p, int ctas, cudaStream_t st, bool pdl) {
    switch (rows) {
        case 16: return launch_tree<D, BF16, 16>(tq, tk, tv, p, ctas, st, pdl);
        case 32: return launch_tree<D, BF16, 32>(tq, tk, tv, p, ctas, st, pdl);
        default: return launch_tree<D, BF16, 0>(tq, tk, tv, p, ctas, st, pdl);
    }
}

static int device_sms() {
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

size_t hg_attn_tree_workspace_bytes(const hg_attn_desc* desc, const hg_tree_desc* tree) {
    if (check_tree(desc, tree) != HG_OK) return 0;
    return plan_tree(desc->head_dim, HG_TREE_CTAS).total;
}

hg_status hg_attn_decode_tree(const void* q, const void* k_cache, const void* v_cache, const int32_t* seq_lens,
                              const int32_t* tok_begin, const hg_partial_src* host_partials, int32_t n_host_src, void* out, float* lse,
                              void* workspace, size_t workspace_bytes, void* stream, const hg_attn_desc* desc,
                              const hg_tree_desc* tree) {
    hg_status st = check_tree(desc, tree);
    if (st != HG_OK) return st;
    if (!q || !k_cache || !v_cache || !seq_lens || !out) return HG_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(out)) return HG_ERR_INVALID_ARG;
    if (n_host_src < 0 || n_host_src > HG_MAX_MERGE_SRC || (n_host_src && !host_partials)) return HG_ERR_INVALID_ARG;
    for (int i = 0; i < n_host_src; ++i)
        if (!host_partials[i].o || !host_partials[i].m || !host_partials[i].l || host_partials[i].nc < 1 || !aligned16(host_partials[i].o))
            return HG_ERR_INVALID_ARG;
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return HG_ERR_INVALID_ARG;
    if (workspace_bytes < hg_attn_tree_workspace_bytes(desc, tree)) return HG_ERR_WORKSPACE;
    const int64_t q_width = (int64_t)desc->num_q_heads * desc->head_dim;       // (rows of out are written while others' q is still read)
    if (rows_overlap(q, tree->q_stride ? tree->q_stride : q_width, q_width, out, q_width, q_width, tree->num_rows)) return HG_ERR_INVALID_ARG;
    TreeParams p;
    memset(&p, 0, sizeof p);
    p.v = static_cast<const uint16_t*>(v_cache);
    p.page_stride = desc->page_stride; p.head_stride = desc->head_stride; p.tok_stride = desc->tok_stride;
    p.block_table = desc->block_table; p.seq_lens = seq_lens; p.tok_begin = tok_begin; p.cu = tree->cu_nodes; p.mask = tree->mask;
    p.out = static_cast<uint16_t*>(out); p.lse = lse; p.status = desc->status;
    p.src.n = n_host_src;
    for (int i = 0; i < n_host_src; ++i) {
        p.src.o[i] = host_partials[i].o; p.src.m[i] = host_partials[i].m; p.src.l[i] = host_partials[i].l; p.src.nc[i] = host_partials[i].nc;
    }
    p.B = desc->batch; p.Hq = desc->num_q_heads; p.Hkv = desc->num_kv_heads; p.G = p.Hq / p.Hkv;
    p.N = tree->num_rows; p.max_nodes = tree->max_nodes; p.words = tree->mask_words;
    const int most = tree->max_nodes < 128 ? tree->max_nodes * p.G : 128, rows = most <= 16 ? 16 : most <= 32 ? 32 : 0;
    p.nodes = (rows ? rows : 128) / p.G;
    p.page_size = desc->page_size; p.page_shift = ilog2_exact(desc->page_size); p.max_pages = desc->max_pages; p.num_pages = desc->num_pages;
    p.scale = desc->scale > 0.f ? desc->scale : 1.0f / sqrtf((float)desc->head_dim);
    p.div_G = make_fast_div((uint32_t)p.G);
    p.div_wide = make_fast_div((uint32_t)(2 * p.nodes));
    p.scale_log2 = p.scale * 1.4426950408889634f;
    p.reread = tree->max_nodes > 2 * p.nodes;
    p.test_stall = (desc->flags & HG_FLAG_TEST_STALL) ? 1 : 0;
    const int sms = device_sms(), ctas = sms < HG_TREE_CTAS ? sms : HG_TREE_CTAS;
    if (sms < 1) return HG_ERR_CUDA;
    p.inv_ctas = ctas > 1 ? ~0ull / (unsigned)ctas + 1ull : 0ull;      // (one CTA: its stretch begins at 0)
    const TreePlan w = plan_tree(desc->head_dim, HG_TREE_CTAS);
    char* ws = static_cast<char*>(workspace);
    p.ws.cut = reinterpret_cast<TreeCut*>(ws); p.ws.valid = reinterpret_cast<int32_t*>(ws + w.valid);
    p.ws.o = reinterpret_cast<float*>(ws + w.o); p.ws.m = reinterpret_cast<float*>(ws + w.m); p.ws.l = reinterpret_cast<float*>(ws + w.l);
    CUtensorMap tq, tk, tv;
    st = make_query_map(desc, p, tree->q_stride ? tree->q_stride : q_width, q, &tq);
    if (st != HG_OK) return st;
    st = make_tile_maps(desc, k_cache, v_cache, TREE_TILE, &tk, &tv);
    if (st != HG_OK) return st;
    cudaStream_t cs = static_cast<cudaStream_t>(stream);
    const bool bf16 = desc->dtype == HG_DTYPE_BF16, pdl = !desc_tune(desc).off(HG_TUNE_NO_PDL);
    if (desc->head_dim == 128) return bf16 ? launch_tree_rows<128, true>(rows, tq, tk, tv, p, ctas, cs, pdl) : launch_tree_rows<128, false>(rows, tq, tk, tv, p, ctas, cs, pdl);
    return bf16 ? launch_tree_rows<64, true>(rows, tq, tk, tv, p, ctas, cs, pdl) : launch_tree_rows<64, false>(rows, tq, tk, tv, p, ctas, cs, pdl);
}

}  // extern "C"
