// Host side of the shared-prefix entry points declared in include/hybridgen_attn.h: argument validation, launches,
// and the decode step that joins the shared and the own partials.
#include "hybridgen_attn.h"

#include <cuda.h>
#include <cuda_runtime.h>
#include <math.h>
#include <string.h>

#include <atomic>

#include "hg_hostutil.h"
#include "hg_prefix.cuh"

namespace hg {

// `own`: the description's own chunk fields are used too
static hg_status check_prefix(const hg_attn_desc* d, const hg_prefix_desc* x, bool own) {
    hg_status st = own ? check_desc(d, true) : check_pool(d);
    if (st != HG_OK) return st;
    if (!x || x->struct_size < sizeof(hg_prefix_desc)) return HG_ERR_INVALID_ARG;
    if (x->num_groups < 1 || x->chunk_tokens < 1 || x->num_chunks < 1) return HG_ERR_INVALID_ARG;
    if (!x->seq_group || !x->group_row || !x->group_begin || !x->group_end) return HG_ERR_INVALID_ARG;
    if (x->num_groups > HG_MAX_GROUPS) return HG_ERR_UNSUPPORTED;
    if (x->chunk_tokens % 128 || x->chunk_tokens % d->page_size) return HG_ERR_UNSUPPORTED;
    if ((int64_t)d->max_pages * d->page_size > 0x7fffff00ll) return HG_ERR_UNSUPPORTED;       // token positions have 31 bits,
    const int64_t rows = (int64_t)d->batch * d->num_q_heads;                                   // and so have partials of a
    if (rows * x->num_chunks > 0x7fffffffll) return HG_ERR_UNSUPPORTED;                        // call and items of a group
    if ((rows / 128 + 2ll * d->num_kv_heads) * x->num_chunks > 0x7fffffffll) return HG_ERR_UNSUPPORTED;
    return HG_OK;
}

// The queries are a matrix of B * Hq rows, read by rows.
static hg_status make_prefix_maps(const hg_attn_desc* d, const void* q, const void* k, const void* v, CUtensorMap* tq, CUtensorMap* tk, CUtensorMap* tv) {
    hg_status st = make_tile_maps(d, k, v, PFX_TILE, tk, tv);
    if (st != HG_OK) return st;
    EncodeTiledFn enc = encode_fn();
    cuuint32_t estr[2] = {1, 1};
    const CUtensorMapDataType dt = d->dtype == HG_DTYPE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    cuuint64_t qdims[2] = {(cuuint64_t)d->head_dim, (cuuint64_t)d->batch * d->num_q_heads}, qstride[1] = {(cuuint64_t)d->head_dim * 2u};
    cuuint32_t qbox[2] = {64, 1};
    if (enc(tq, dt, 2, const_cast<void*>(q), qdims, qstride, qbox, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
        return HG_ERR_UNSUPPORTED;
    return HG_OK;
}

template <int D, bool BF16>
static hg_status launch_prefix(const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv, const PrefixParams& p, cudaStream_t st, bool pdl) {
    static std::atomic<int> sms_of[kMaxDevices];           // set once the device's shared-memory opt-in is in force; zero-initialised
    auto kern = prefix_partial_kernel<D, BF16>;
    constexpr size_t smem = pfx_smem_bytes<D>();
    static_assert(smem <= 227 * 1024, "shared memory of one SM");
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) { cudaGetLastError(); return HG_ERR_CUDA; }
    int sms = sms_of[dev].load(std::memory_order_acquire);
    if (sms == 0) {
        if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess ||
            cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || sms < 1) {
            cudaGetLastError();
            return HG_ERR_CUDA;
        }
        sms_of[dev].store(sms, std::memory_order_release);   // racing threads store the same value
    }
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof cfg);
    cfg.gridDim = dim3((unsigned)sms); cfg.blockDim = dim3(PFX_THREADS); cfg.dynamicSmemBytes = smem; cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr; cfg.numAttrs = pdl ? 1 : 0;
    if (cudaLaunchKernelEx(&cfg, kern, tq, tk, tv, p) != cudaSuccess) { cudaGetLastError(); return HG_ERR_CUDA; }
    return HG_OK;
}

// The own slices of a joined step: further items of the shared launch, or only cut (where `cut` is given) for the launch behind it.
struct OwnSlices {
    const int32_t *seq_lens, *tok_begin, *tok_end;
    float *o, *m, *l;
    bool items;
    int32_t* cut;
    int cut_C, cut_NC;
};

static hg_status run_prefix(const void* q, const void* k, const void* v, float* o_part, float* m_part, float* l_part, int32_t* zero,
                            const OwnSlices* own, void* stream, const hg_attn_desc* d, const hg_prefix_desc* x) {
    PrefixParams p;
    memset(&p, 0, sizeof p);
    CUtensorMap tq, tk, tv;
    hg_status st = make_prefix_maps(d, q, k, v, &tq, &tk, &tv);
    if (st != HG_OK) return st;
    p.block_table = d->block_table; p.seq_group = x->seq_group; p.group_row = x->group_row;
    p.group_begin = x->group_begin; p.group_end = x->group_end;
    p.o_part = o_part; p.m_part = m_part; p.l_part = l_part; p.status = d->status; p.zero = zero;
    if (own) {
        p.own = own->items; p.own_NC = d->num_chunks; p.own_C = d->chunk_tokens;
        p.cut = own->cut; p.cut_C = own->cut_C; p.cut_NC = own->cut_NC;
        p.seq_lens = own->seq_lens; p.tok_begin = own->tok_begin; p.tok_end = own->tok_end;
        p.own_o = own->o; p.own_m = own->m; p.own_l = own->l;
    }
    p.B = d->batch; p.Hq = d->num_q_heads; p.Hkv = d->num_kv_heads; p.G = p.Hq / p.Hkv;
    p.NG = x->num_groups; p.NC = x->num_chunks; p.C = x->chunk_tokens;
    p.page_size = d->page_size; p.page_shift = ilog2_exact(d->page_size); p.max_pages = d->max_pages; p.num_pages = d->num_pages;
    p.sparse_empty = (d->flags & HG_FLAG_SPARSE_EMPTY) ? 1 : 0;
    p.test_stall = (d->flags & HG_FLAG_TEST_STALL) ? 1 : 0;
    p.scale = d->scale > 0.f ? d->scale : 1.0f / sqrtf((float)d->head_dim);
    p.scale_log2 = p.scale * 1.4426950408889634f;
    p.div_G = make_fast_div((uint32_t)p.G);
    cudaStream_t cs = static_cast<cudaStream_t>(stream);
    const bool bf16 = d->dtype == HG_DTYPE_BF16, pdl = !desc_tune(d).off(HG_TUNE_NO_PDL);
    if (d->head_dim == 128) return bf16 ? launch_prefix<128, true>(tq, tk, tv, p, cs, pdl) : launch_prefix<128, false>(tq, tk, tv, p, cs, pdl);
    return bf16 ? launch_prefix<64, true>(tq, tk, tv, p, cs, pdl) : launch_prefix<64, false>(tq, tk, tv, p, cs, pdl);
}

// Whether a step's own slices run as items of the shared launch instead of in hg_attn_partial's: when there are so few that
// they find SMs of their own.  (Steps in a loop.  4 sequences, 8 KV heads, 512 shared and 32 own tokens: 13.1 us instead of 21.2.
// An item costs its SM some 4 us whatever it holds, where hg_attn_partial streams the next one meanwhile: 64 sequences, 8 heads
// of 64, 2048 + 100 tokens: 34 us instead of 28; 16 sequences, 56 heads, 16384 + 500: 156 instead of 139; 96 sequences in 12
// groups, 8 KV heads: 199 instead of 161.)
static bool own_in_shared_launch(const hg_attn_desc* d) {
    return (int64_t)d->batch * d->num_kv_heads * ((d->num_chunks + 1) / 2) <= 128;
}

// Workspace of the joined step: the shared partials in front, behind them what hg_attn_decode's partial half needs.
struct SharedWorkspace { size_t po, pm, pl, o, m, l, sched, cut, total; };

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
    w.cut = off; off += up256((size_t)d->batch * sizeof(int32_t));
    w.total = off;
    return w;
}

}  // namespace hg

using namespace hg;

extern "C" {

hg_status hg_attn_prefix_partial(const void* q, const void* k_cache, const void* v_cache, float* o_part, float* m_part, float* l_part,
                                 void* stream, const hg_attn_desc* desc, const hg_prefix_desc* prefix) {
    hg_status st = check_prefix(desc, prefix, false);
    if (st != HG_OK) return st;
    if (!q || !k_cache || !v_cache || !o_part || !m_part || !l_part) return HG_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(k_cache) || !aligned16(v_cache) || (reinterpret_cast<uintptr_t>(o_part) & 31u)) return HG_ERR_INVALID_ARG;
    return run_prefix(q, k_cache, v_cache, o_part, m_part, l_part, nullptr, nullptr, stream, desc, prefix);
}

int32_t hg_attn_prefix_suggest_chunk(int64_t shared_tokens, int32_t num_groups, int32_t num_members, int32_t num_q_heads,
                                     int32_t num_kv_heads, int32_t page_size) {
    if (shared_tokens < 0 || num_groups < 1 || num_members < 0 || num_kv_heads < 1 || num_q_heads < 1 || num_q_heads % num_kv_heads) return 0;
    const int shift = ilog2_exact(page_size);
    if (shift < 4 || shift > 8) return 0;
    // Work items are dealt out in turn, one at a time to each of 148 SMs, so the number of items should fill whole rounds;
    // against many short items stand their epilogues and the merge, which reads every chunk's partials.  The costs, in
    // microseconds, are those measured at 128 components: 2 per step of an item (128 tokens for two row tiles), 2.5 per item,
    // 1e-4 per partial row in the merge.  Several groups count as if all were of the average size, but since they are not,
    // the last round is taken to be one item longer than the average.
    // A chunk is not longer than 2560 tokens (1024 where few rows make short ones cheap): the tensor cores cut their sums off
    // where fp32 arithmetic rounds, so a chunk's error grows with its length (measured: 2.3e-9 of the result per token, 1.7e-5
    // at 7296 tokens), while the merge of the chunks rounds.  (Steps in a loop.  131072 tokens, 32 sequences of 64/8 heads:
    // 213 us at 2432 tokens, 200 at 7296; 65536 tokens, 128 sequences: 446 at 1792, 418 at 2432, 373 at 7296.)
    const int64_t unit = page_size > PFX_TILE ? page_size / PFX_TILE : 1;
    int64_t tiles = (shared_tokens / num_groups + PFX_TILE - 1) / PFX_TILE;
    if (tiles < 1) tiles = 1;
    const int64_t rows = ((int64_t)num_members + num_groups - 1) / num_groups * (num_q_heads / num_kv_heads), rem = rows % 256;
    const int64_t wide = rows / 256 + (rem > 128 ? 1 : 0), narrow = rem > 0 && rem <= 128 ? 1 : 0;
    const int64_t longest = wide > 0 ? 20 : 8;
    int64_t best = 0;
    double best_cost = 0;
    for (int64_t c = unit; c <= longest; c += unit) {
        const int64_t nc = (tiles + c - 1) / c;
        const int64_t items = num_groups * (int64_t)num_kv_heads * (wide * nc + narrow * ((nc + 1) / 2));
        const double rounds = num_groups == 1 ? (double)((items + 147) / 148) : (double)items / 148.0 + 1.0;
        const double cost = rounds * (2.0 * (double)c + 2.5) + 1e-4 * (double)nc * num_members * num_q_heads;
        if (best == 0 || cost < best_cost) { best = c; best_cost = cost; }
    }
    return (int32_t)(best * PFX_TILE);
}

size_t hg_attn_shared_workspace_bytes(const hg_attn_desc* desc, const hg_prefix_desc* prefix) {
    if (check_prefix(desc, prefix, true) != HG_OK) return 0;
    return plan_shared(desc, prefix).total;
}

hg_status hg_attn_decode_shared(const void* q, const void* k_cache, const void* v_cache, const int32_t* seq_lens,
                                const int32_t* tok_begin, const int32_t* tok_end, const hg_partial_src* host_partials,
                                int32_t n_host_src, float* out, float* lse, void* workspace, size_t workspace_bytes, void* stream,
                                const hg_attn_desc* desc, const hg_prefix_desc* prefix) {
    hg_status st = check_prefix(desc, prefix, true);
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
    // The chunks of the own slices are private to this call: where there are many, 256 tokens are better than fewer (with
    // 4000 to 5400 chunk slots of 128 tokens hg_attn_partial takes 26, 32 and 36 us instead of 31, 37 and 40).  A slice is
    // still cut where the caller's chunk slots end: the shared kernel writes the ends that hg_attn_partial reads.
    const int coarse = 256;
    int32_t* cut = nullptr;
    const int64_t slots = ((int64_t)dd.num_chunks * dd.chunk_tokens + coarse - 1) / coarse + 1;
    if (dd.chunk_tokens < coarse && slots <= dd.num_chunks && (int64_t)dd.batch * dd.num_kv_heads * dd.num_chunks >= 1024) {
        cut = reinterpret_cast<int32_t*>(ws + w.cut);
        dd.chunk_tokens = coarse;
        dd.num_chunks = (int32_t)slots;
    }
    const bool one_launch = !cut && own_in_shared_launch(&dd);
    const OwnSlices own = {seq_lens, tok_begin, tok_end, at(w.o), at(w.m), at(w.l), one_launch, cut, desc->chunk_tokens, desc->num_chunks};
    // where the own partials get a launch of their own, the shared kernel clears their work counter on its way, so that no
    // clearing stands between the two
    st = run_prefix(q, k_cache, v_cache, at(w.po), at(w.pm), at(w.pl), one_launch ? nullptr : dd.sched_counter, &own, stream, &dd, prefix);
    if (st != HG_OK) return st;
    if (!one_launch) {
        dd.flags |= HG_FLAG_COUNTER_CLEAN;
        st = hg_attn_partial(q, k_cache, v_cache, seq_lens, tok_begin, cut ? cut : tok_end, at(w.o), at(w.m), at(w.l), stream, &dd);
        if (st != HG_OK) return st;
    }
    hg_partial_src src[HG_MAX_MERGE_SRC];
    src[0].o = at(w.po); src[0].m = at(w.pm); src[0].l = at(w.pl); src[0].nc = prefix->num_chunks; src[0].reserved = 0;
    src[1].o = at(w.o); src[1].m = at(w.m); src[1].l = at(w.l); src[1].nc = dd.num_chunks; src[1].reserved = 0;
    for (int i = 0; i < n_host_src; ++i) src[2 + i] = host_partials[i];
    return hg_attn_merge(src, 2 + n_host_src, out, lse, stream, &dd);
}

}  // extern "C"
