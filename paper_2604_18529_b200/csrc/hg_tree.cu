// Host side of the attention of a step's new tokens declared in include/hybridgen_attn.h: argument validation and launches.
#include "hybridgen_attn.h"

#include <cuda_runtime.h>
#include <math.h>
#include <string.h>

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

}  // namespace hg

using namespace hg;

extern "C" {

size_t hg_attn_tree_workspace_bytes(const hg_attn_desc* desc, const hg_tree_desc* tree) {
    if (check_tree(desc, tree) != HG_OK) return 0;
    return 256;
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
    TreeParams p;
    memset(&p, 0, sizeof p);
    p.q = static_cast<const uint16_t*>(q); p.k = static_cast<const uint16_t*>(k_cache); p.v = static_cast<const uint16_t*>(v_cache);
    p.block_table = desc->block_table; p.seq_lens = seq_lens; p.tok_begin = tok_begin; p.cu = tree->cu_nodes; p.mask = tree->mask;
    p.out = static_cast<uint16_t*>(out); p.lse = lse; p.status = desc->status;
    p.src.n = n_host_src;
    for (int i = 0; i < n_host_src; ++i) {
        p.src.o[i] = host_partials[i].o; p.src.m[i] = host_partials[i].m; p.src.l[i] = host_partials[i].l; p.src.nc[i] = host_partials[i].nc;
    }
    p.B = desc->batch; p.Hq = desc->num_q_heads; p.Hkv = desc->num_kv_heads; p.G = p.Hq / p.Hkv;
    p.N = tree->num_rows; p.max_nodes = tree->max_nodes; p.words = tree->mask_words;
    p.q_stride = tree->q_stride ? tree->q_stride : (int64_t)p.Hq * desc->head_dim;
    p.page_stride = desc->page_stride; p.head_stride = desc->head_stride; p.tok_stride = desc->tok_stride;
    p.page_size = desc->page_size; p.page_shift = ilog2_exact(desc->page_size); p.max_pages = desc->max_pages; p.num_pages = desc->num_pages;
    p.scale = desc->scale > 0.f ? desc->scale : 1.0f / sqrtf((float)desc->head_dim);
    p.div_G = make_fast_div((uint32_t)p.G);
    const unsigned grid = (unsigned)(((int64_t)p.N * p.Hq + 3) / 4);
    cudaStream_t cs = static_cast<cudaStream_t>(stream);
    const bool bf16 = desc->dtype == HG_DTYPE_BF16;
    if (desc->head_dim == 128) bf16 ? tree_kernel<128, true><<<grid, 128, 0, cs>>>(p) : tree_kernel<128, false><<<grid, 128, 0, cs>>>(p);
    else bf16 ? tree_kernel<64, true><<<grid, 128, 0, cs>>>(p) : tree_kernel<64, false><<<grid, 128, 0, cs>>>(p);
    return cudaGetLastError() == cudaSuccess ? HG_OK : HG_ERR_CUDA;
}

}  // extern "C"
