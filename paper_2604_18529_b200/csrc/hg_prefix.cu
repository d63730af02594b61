// Host side of the shared-prefix entry points declared in include/hybridgen_attn.h: argument validation, launches,
// and the decode step that joins the shared and the own partials.
#include "hybridgen_attn.h"

#include <cuda.h>
#include <cuda_runtime.h>
#include <math.h>
#include <string.h>

#include "hg_hostutil.h"
#include "hg_prefix.cuh"

namespace hg {

static hg_status check_prefix(const hg_attn_desc* d, const hg_prefix_desc* x) {
    hg_status st = check_desc(d, true);
    if (st != HG_OK) return st;
    if (!x || x->struct_size < sizeof(hg_prefix_desc)) return HG_ERR_INVALID_ARG;
    if (x->num_groups < 1 || x->chunk_tokens < 1 || x->num_chunks < 1) return HG_ERR_INVALID_ARG;
    if (!x->seq_group || !x->group_row || !x->group_begin || !x->group_end) return HG_ERR_INVALID_ARG;
    if (x->num_groups > HG_MAX_GROUPS) return HG_ERR_UNSUPPORTED;
    if (x->chunk_tokens % 128 || x->chunk_tokens % d->page_size) return HG_ERR_UNSUPPORTED;
    if ((int64_t)d->max_pages * d->page_size > 0x7fffff00ll) return HG_ERR_UNSUPPORTED;       // token positions have 31 bits
    return HG_OK;
}

template <int D, bool BF16>
static hg_status launch_prefix(const PrefixParams& p, cudaStream_t st) {
    const int row_blocks = (int)(((long long)p.B * p.G + PFX_ROWS - 1) / PFX_ROWS);
    prefix_partial_kernel<D, BF16><<<dim3((unsigned)p.NC, (unsigned)(p.Hkv * row_blocks), (unsigned)(p.NG + 1)), PFX_THREADS, 0, st>>>(p, row_blocks);
    return cudaGetLastError() == cudaSuccess ? HG_OK : HG_ERR_CUDA;
}

static hg_status run_prefix(const void* q, const void* k, const void* v, float* o_part, float* m_part, float* l_part, void* stream,
                            const hg_attn_desc* d, const hg_prefix_desc* x) {
    PrefixParams p;
    memset(&p, 0, sizeof p);
    p.q = static_cast<const uint16_t*>(q); p.k = static_cast<const uint16_t*>(k); p.v = static_cast<const uint16_t*>(v);
    p.block_table = d->block_table; p.seq_group = x->seq_group; p.group_row = x->group_row;
    p.group_begin = x->group_begin; p.group_end = x->group_end;
    p.o_part = o_part; p.m_part = m_part; p.l_part = l_part; p.status = d->status;
    p.page_stride = d->page_stride; p.head_stride = d->head_stride; p.tok_stride = d->tok_stride;
    p.B = d->batch; p.Hq = d->num_q_heads; p.Hkv = d->num_kv_heads; p.G = p.Hq / p.Hkv;
    p.NG = x->num_groups; p.NC = x->num_chunks; p.C = x->chunk_tokens;
    p.page_size = d->page_size; p.page_shift = ilog2_exact(d->page_size); p.max_pages = d->max_pages; p.num_pages = d->num_pages;
    p.sparse_empty = (d->flags & HG_FLAG_SPARSE_EMPTY) ? 1 : 0;
    p.scale = d->scale > 0.f ? d->scale : 1.0f / sqrtf((float)d->head_dim);
    cudaStream_t cs = static_cast<cudaStream_t>(stream);
    if (d->head_dim == 128) return d->dtype == HG_DTYPE_BF16 ? launch_prefix<128, true>(p, cs) : launch_prefix<128, false>(p, cs);
    return d->dtype == HG_DTYPE_BF16 ? launch_prefix<64, true>(p, cs) : launch_prefix<64, false>(p, cs);
}

// Workspace of the joined step: the shared partials in front, behind them what hg_attn_decode's partial half needs.
struct SharedWorkspace { size_t po, pm, pl, o, m, l, sched, total; };

static SharedWorkspace plan_shared(const hg_attn_desc* d, const hg_prefix_desc* x) {
    SharedWorkspace w;
    const size_t rows = (size_t)d->batch * d->num_q_heads;
    size_t off = 0;
    w.po = off; off += up256(rows * x->num_chunks * d->head_dim * sizeof(float));
    w.pm = off; off += up256(rows * x->num_chunks * sizeof(float));
    w.pl = off; off += up256(rows * x->num_chunks * sizeof(float));
    w.o = off; off += up256(rows * d->num_chunks * d->head_dim * sizeof(float));
    w.m = off; off += up256(rows * d->num_chunks * sizeof(float));
    w.l = off; off += up256(rows * d->num_chunks * sizeof(float));
    w.sched = off; off += 256;
    w.total = off;
    return w;
}

}  // namespace hg

using namespace hg;

extern "C" {

hg_status hg_attn_prefix_partial(const void* q, const void* k_cache, const void* v_cache, float* o_part, float* m_part, float* l_part,
                                 void* stream, const hg_attn_desc* desc, const hg_prefix_desc* prefix) {
    hg_status st = check_prefix(desc, prefix);
    if (st != HG_OK) return st;
    if (!q || !k_cache || !v_cache || !o_part || !m_part || !l_part) return HG_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(o_part)) return HG_ERR_INVALID_ARG;
    return run_prefix(q, k_cache, v_cache, o_part, m_part, l_part, stream, desc, prefix);
}

int32_t hg_attn_prefix_suggest_chunk(int64_t shared_tokens, int32_t num_groups, int32_t num_members, int32_t num_q_heads,
                                     int32_t num_kv_heads, int32_t page_size) {
    if (shared_tokens < 0 || num_groups < 1 || num_members < 0 || num_kv_heads < 1 || num_q_heads < 1 || num_q_heads % num_kv_heads) return 0;
    const int shift = ilog2_exact(page_size);
    if (shift < 4 || shift > 8) return 0;
    return 256;
}

size_t hg_attn_shared_workspace_bytes(const hg_attn_desc* desc, const hg_prefix_desc* prefix) {
    if (check_prefix(desc, prefix) != HG_OK) return 0;
    return plan_shared(desc, prefix).total;
}

hg_status hg_attn_decode_shared(const void* q, const void* k_cache, const void* v_cache, const int32_t* seq_lens,
                                const int32_t* tok_begin, const int32_t* tok_end, const hg_partial_src* host_partials,
                                int32_t n_host_src, float* out, float* lse, void* workspace, size_t workspace_bytes, void* stream,
                                const hg_attn_desc* desc, const hg_prefix_desc* prefix) {
    hg_status st = check_prefix(desc, prefix);
    if (st != HG_OK) return st;
    if (!q || !k_cache || !v_cache || !seq_lens || !tok_begin || !tok_end || !out) return HG_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(k_cache) || !aligned16(v_cache)) return HG_ERR_INVALID_ARG;
    if (n_host_src < 0 || n_host_src > HG_MAX_MERGE_SRC - 2 || (n_host_src && !host_partials)) return HG_ERR_INVALID_ARG;
    for (int i = 0; i < n_host_src; ++i)
        if (!host_partials[i].o || !host_partials[i].m || !host_partials[i].l || host_partials[i].nc < 1 || !aligned16(host_partials[i].o))
            return HG_ERR_INVALID_ARG;
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return HG_ERR_INVALID_ARG;
    const SharedWorkspace w = plan_shared(desc, prefix);
    if (workspace_bytes < w.total) return HG_ERR_WORKSPACE;
    char* ws = static_cast<char*>(workspace);
    auto at = [&](size_t off) { return reinterpret_cast<float*>(ws + off); };
    hg_attn_desc dd;
    memset(&dd, 0, sizeof dd);
    memcpy(&dd, desc, desc->struct_size < sizeof dd ? desc->struct_size : sizeof dd);
    dd.struct_size = sizeof dd;
    dd.flags |= HG_FLAG_SPARSE_EMPTY;                                  // the partials are private to this call and its merge
    dd.sched_counter = reinterpret_cast<int32_t*>(ws + w.sched);
    st = run_prefix(q, k_cache, v_cache, at(w.po), at(w.pm), at(w.pl), stream, &dd, prefix);
    if (st != HG_OK) return st;
    st = hg_attn_partial(q, k_cache, v_cache, seq_lens, tok_begin, tok_end, at(w.o), at(w.m), at(w.l), stream, &dd);
    if (st != HG_OK) return st;
    hg_partial_src src[HG_MAX_MERGE_SRC];
    src[0].o = at(w.po); src[0].m = at(w.pm); src[0].l = at(w.pl); src[0].nc = prefix->num_chunks; src[0].reserved = 0;
    src[1].o = at(w.o); src[1].m = at(w.m); src[1].l = at(w.l); src[1].nc = desc->num_chunks; src[1].reserved = 0;
    for (int i = 0; i < n_host_src; ++i) src[2 + i] = host_partials[i];
    return hg_attn_merge(src, 2 + n_host_src, out, lse, stream, &dd);
}

}  // extern "C"
