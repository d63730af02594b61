// Host side of the operators on a step's new tokens declared in include/hybridgen_attn.h: argument validation, launches, and
// the frequencies of rotary positions.
#include "hybridgen_attn.h"

#include <cuda_runtime.h>
#include <math.h>
#include <string.h>

#include "hg_draft.cuh"
#include "hg_hostutil.h"

namespace hg {

// Launches with the programmatic-serialisation attribute (every kernel here waits for its predecessor before its first access).
template <typename P>
static hg_status launch_draft(void (*kern)(P), dim3 grid, unsigned threads, int cluster, void* stream, const P& p) {
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof cfg);
    cfg.gridDim = grid; cfg.blockDim = dim3(threads);
    cfg.stream = static_cast<cudaStream_t>(stream);
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    int na = 1;
    if (cluster > 0) {
        attr[na].id = cudaLaunchAttributeClusterDimension;
        attr[na].val.clusterDim.x = (unsigned)cluster; attr[na].val.clusterDim.y = 1; attr[na].val.clusterDim.z = 1;
        ++na;
    }
    cfg.attrs = attr; cfg.numAttrs = (unsigned)na;
    if (cudaLaunchKernelEx(&cfg, kern, p) != cudaSuccess) { cudaGetLastError(); return HG_ERR_CUDA; }
    return HG_OK;
}

static hg_status check_rope(const hg_rope_desc* r, int head_dim) {
    if (!r || r->struct_size < sizeof(hg_rope_desc)) return HG_ERR_INVALID_ARG;
    if (r->num_rows < 1 || r->rot_dim < 2 || r->rot_dim > head_dim || !r->freq) return HG_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(r->freq) & 7u) return HG_ERR_INVALID_ARG;
    if (r->layout != HG_ROPE_HALF && r->layout != HG_ROPE_INTERLEAVED) return HG_ERR_INVALID_ARG;
    if (!isfinite(r->magnitude) || (r->flags & ~HG_ROPE_INVERSE)) return HG_ERR_INVALID_ARG;
    if ((r->q_stride | r->q_out_stride | r->k_stride | r->v_stride) & 7) return HG_ERR_INVALID_ARG;
    if (r->rot_dim % 16) return HG_ERR_UNSUPPORTED;
    return HG_OK;
}

// Row stride of an array of `heads` heads, or -1.
static int64_t row_stride(int64_t given, int heads, int head_dim) {
    const int64_t least = (int64_t)heads * head_dim;
    return given == 0 ? least : given < least ? -1 : given;
}

static hg_status run_rope(RopeParams& p, int heads, int kv_heads, int head_dim, bool bf16, const hg_rope_desc* r, void* stream) {
    p.freq = r->freq;
    p.Hq = heads; p.Hkv = kv_heads; p.D = head_dim; p.rot = r->rot_dim;
    p.magnitude = r->magnitude == 0.f ? 1.f : r->magnitude;
    p.sign = r->flags & HG_ROPE_INVERSE ? -1.f : 1.f;
    const bool half = r->layout == HG_ROPE_HALF;
    p.head_units = half ? r->rot_dim / 16 + (head_dim - r->rot_dim) / 8 : head_dim / 8;
    p.units = (heads + kv_heads) * p.head_units + kv_heads * (head_dim / 8);
    p.div_head = make_fast_div((uint32_t)p.head_units);
    // a row's units go to several CTAs where there are few rows
    const int step = ROPE_THREADS * ROPE_UNROLL, chunks = (p.units + step - 1) / step;
    const dim3 grid((unsigned)r->num_rows, (unsigned)(r->num_rows >= 2048 ? 1 : chunks < 65535 ? chunks : 65535));
    if (half) return bf16 ? launch_draft(kv_append_rope_kernel<true, true>, grid, ROPE_THREADS, 0, stream, p)
                          : launch_draft(kv_append_rope_kernel<false, true>, grid, ROPE_THREADS, 0, stream, p);
    return bf16 ? launch_draft(kv_append_rope_kernel<true, false>, grid, ROPE_THREADS, 0, stream, p)
                : launch_draft(kv_append_rope_kernel<false, false>, grid, ROPE_THREADS, 0, stream, p);
}

}  // namespace hg

using namespace hg;

extern "C" {

hg_status hg_kv_slots(const int32_t* seq_lens, const int32_t* n_new, const int32_t* parent, int32_t num_rows, int32_t* cu_new,
                      int32_t* tok_seq, int32_t* tok_pos, int64_t* tok_slot, uint32_t* mask, int32_t mask_words, void* stream,
                      const hg_attn_desc* desc) {
    return hg_kv_slots_ready(seq_lens, n_new, nullptr, parent, num_rows, cu_new, tok_seq, tok_pos, tok_slot, mask, mask_words, stream, desc);
}

hg_status hg_kv_slots_ready(const int32_t* seq_lens, const int32_t* n_new, const int32_t* n_ready, const int32_t* parent, int32_t num_rows,
                            int32_t* cu_new, int32_t* tok_seq, int32_t* tok_pos, int64_t* tok_slot, uint32_t* mask, int32_t mask_words,
                            void* stream, const hg_attn_desc* desc) {
    hg_status st = check_pool(desc);
    if (st != HG_OK) return st;
    if (!seq_lens || !cu_new || num_rows < 1 || (mask && mask_words < 1)) return HG_ERR_INVALID_ARG;
    if (mask && mask_words > HG_MAX_TREE_NODES / 32) return HG_ERR_UNSUPPORTED;
    if (reinterpret_cast<uintptr_t>(tok_slot) & 7u) return HG_ERR_INVALID_ARG;
    const size_t N = (size_t)num_rows, B = (size_t)desc->batch;
    const void* const out[5] = {cu_new, tok_seq, tok_pos, tok_slot, mask};
    const size_t out_bytes[5] = {(B + 1) * 4, N * 4, N * 4, N * 8, mask ? N * mask_words * 4 : 0};
    const void* const in[5] = {seq_lens, n_new, n_ready, parent, desc->block_table};
    const size_t in_bytes[5] = {B * 4, B * 4, B * 4, N * 4, B * desc->max_pages * 4};
    for (int i = 0; i < 5; ++i) {
        for (int j = 0; j < i; ++j) if (overlap(out[i], out_bytes[i], out[j], out_bytes[j])) return HG_ERR_INVALID_ARG;
        for (int j = 0; j < 5; ++j) if (overlap(out[i], out_bytes[i], in[j], in_bytes[j])) return HG_ERR_INVALID_ARG;
    }
    SlotsParams p;
    p.seq_lens = seq_lens; p.n_new = n_new; p.n_ready = n_ready; p.parent = parent; p.table = desc->block_table;
    p.cu = cu_new; p.seq = tok_seq; p.pos = tok_pos; p.slot = tok_slot; p.mask = mask; p.status = desc->status;
    p.B = desc->batch; p.N = num_rows; p.words = mask ? mask_words : 0;
    p.limit = !parent && !mask ? 0x7fffffff : mask && mask_words * 32 < HG_MAX_TREE_NODES ? mask_words * 32 : HG_MAX_TREE_NODES;
    p.cut = n_ready ? 0x7fffffff : p.limit;            // (with n_ready no sequence loses a row, and nothing behind it moves)
    p.page_shift = ilog2_exact(desc->page_size); p.max_pages = desc->max_pages; p.num_pages = desc->num_pages;
    if (desc->batch <= SLOTS_SCAN) {
        const bool quads = !parent && !mask && aligned16(tok_seq) && aligned16(tok_pos) && aligned16(tok_slot);
        const long long per_cta = SLOTS_THREADS * (quads ? 4 : 1), ctas = ((long long)num_rows + per_cta - 1) / per_cta;
        const dim3 grid((unsigned)(ctas < 888 ? ctas : 888));      // (what 148 SMs hold at a time)
        if (n_ready) return quads ? launch_draft(kv_slots_kernel<true, true>, grid, SLOTS_THREADS, 0, stream, p)
                                  : launch_draft(kv_slots_kernel<false, true>, grid, SLOTS_THREADS, 0, stream, p);
        return quads ? launch_draft(kv_slots_kernel<true, false>, grid, SLOTS_THREADS, 0, stream, p)
                     : launch_draft(kv_slots_kernel<false, false>, grid, SLOTS_THREADS, 0, stream, p);
    }
    // ranges of sequences, and splits of their rows
    const int ranges = desc->batch < 592 ? desc->batch : 592;
    p.per = (desc->batch + ranges - 1) / ranges;
    const long long per_range = ((long long)num_rows + ranges - 1) / ranges, splits = (per_range + 511) / 512, most = 1184 / ranges;
    return launch_draft(n_ready ? kv_slots_many_kernel<true> : kv_slots_many_kernel<false>, dim3((unsigned)ranges, (unsigned)(splits < most ? splits : most)),
                        SLOTS_THREADS, 0, stream, p);
}

hg_status hg_rope(const void* x, void* y, const int32_t* pos, int32_t num_heads, int32_t head_dim, int32_t dtype, void* stream,
                  const hg_rope_desc* rope) {
    if (num_heads < 1 || head_dim < 1 || (dtype != HG_DTYPE_F16 && dtype != HG_DTYPE_BF16)) return HG_ERR_INVALID_ARG;
    if (head_dim != 64 && head_dim != 128) return HG_ERR_UNSUPPORTED;
    hg_status st = check_rope(rope, head_dim);
    if (st != HG_OK) return st;
    if (num_heads > 65535) return HG_ERR_UNSUPPORTED;
    if (!x || !y || !pos || !aligned16(x) || !aligned16(y)) return HG_ERR_INVALID_ARG;
    RopeParams p;
    memset(&p, 0, sizeof p);
    p.q_stride = row_stride(rope->q_stride, num_heads, head_dim);
    p.q_out_stride = row_stride(rope->q_out_stride, num_heads, head_dim);
    if (p.q_stride < 0 || p.q_out_stride < 0) return HG_ERR_INVALID_ARG;
    const int64_t width = (int64_t)num_heads * head_dim, n = rope->num_rows;
    if (!(x == y && p.q_stride == p.q_out_stride) && rows_overlap(x, p.q_stride, width, y, p.q_out_stride, width, n)) return HG_ERR_INVALID_ARG;
    p.q = static_cast<const uint16_t*>(x); p.q_out = static_cast<uint16_t*>(y); p.pos = pos;
    return run_rope(p, num_heads, 0, head_dim, dtype == HG_DTYPE_BF16, rope, stream);
}

hg_status hg_kv_append_rope(const void* q, const void* k_new, const void* v_new, const int32_t* pos, const int64_t* slot, void* q_out,
                            void* k_cache, void* v_cache, void* stream, const hg_attn_desc* desc, const hg_rope_desc* rope) {
    hg_status st = check_pool(desc);
    if (st != HG_OK) return st;
    st = check_rope(rope, desc->head_dim);
    if (st != HG_OK) return st;
    if (desc->num_q_heads > 65535) return HG_ERR_UNSUPPORTED;
    if (!k_new || !v_new || !pos || !slot || !k_cache || !v_cache || !q != !q_out) return HG_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(q_out) || !aligned16(k_new) || !aligned16(v_new) || !aligned16(k_cache) || !aligned16(v_cache) ||
        (reinterpret_cast<uintptr_t>(slot) & 7u)) return HG_ERR_INVALID_ARG;
    const int Hq = desc->num_q_heads, Hkv = desc->num_kv_heads, D = desc->head_dim;
    RopeParams p;
    memset(&p, 0, sizeof p);
    p.q_stride = row_stride(rope->q_stride, Hq, D);
    p.q_out_stride = row_stride(rope->q_out_stride, Hq, D);
    p.k_stride = row_stride(rope->k_stride, Hkv, D);
    p.v_stride = row_stride(rope->v_stride, Hkv, D);
    if (p.q_stride < 0 || p.q_out_stride < 0 || p.k_stride < 0 || p.v_stride < 0) return HG_ERR_INVALID_ARG;
    const int64_t width = (int64_t)Hq * D, kv_width = (int64_t)Hkv * D, n = rope->num_rows;
    if (q && ((!(q == q_out && p.q_stride == p.q_out_stride) && rows_overlap(q, p.q_stride, width, q_out, p.q_out_stride, width, n)) ||
              rows_overlap(k_new, p.k_stride, kv_width, q_out, p.q_out_stride, width, n) ||
              rows_overlap(v_new, p.v_stride, kv_width, q_out, p.q_out_stride, width, n))) return HG_ERR_INVALID_ARG;
    p.q = static_cast<const uint16_t*>(q); p.q_out = static_cast<uint16_t*>(q_out);
    p.k = static_cast<const uint16_t*>(k_new); p.v = static_cast<const uint16_t*>(v_new);
    p.pv = pool_view(desc, k_cache, v_cache);
    p.pos = pos; p.slot = slot; p.status = desc->status;
    p.places = (int64_t)desc->num_pages * desc->page_size;
    return run_rope(p, q ? Hq : 0, Hkv, D, desc->dtype == HG_DTYPE_BF16, rope, stream);
}

hg_status hg_rope_frequencies(int32_t rot_dim, const hg_rope_scaling* s, double* freq, float* magnitude) {
    if (!s || s->struct_size < sizeof(hg_rope_scaling) || !freq || rot_dim < 2 || rot_dim % 2) return HG_ERR_INVALID_ARG;
    if (s->kind < HG_ROPE_SCALE_NONE || s->kind > HG_ROPE_SCALE_INDEX || !(s->theta > 1.0) || !isfinite(s->theta)) return HG_ERR_INVALID_ARG;
    if (s->kind != HG_ROPE_SCALE_NONE && (!(s->factor >= 1.0) || !isfinite(s->factor))) return HG_ERR_INVALID_ARG;
    const bool blend = s->kind == HG_ROPE_SCALE_TURNS || s->kind == HG_ROPE_SCALE_INDEX;
    if (blend && (!(s->low > 0.0) || !(s->high > s->low) || !isfinite(s->high) || !(s->context > 0.0) || !isfinite(s->context))) return HG_ERR_INVALID_ARG;
    const double two_pi = 6.283185307179586477, n = rot_dim;
    const int pairs = rot_dim / 2;
    double theta = s->theta;
    if (s->kind == HG_ROPE_SCALE_BASE && rot_dim > 2) theta *= pow(s->factor, n / (n - 2.0));
    // the index at which a pair makes so many turns within the context: context theta^(-2 i / n) = 2 pi turns
    auto index_of = [&](double turns) { return n * log(s->context / (two_pi * turns)) / (2.0 * log(s->theta)); };
    double first = 0, last = 0;
    if (s->kind == HG_ROPE_SCALE_INDEX) {
        first = fmin(fmax(floor(index_of(s->high)), 0.0), n - 1.0);
        last = fmin(fmax(ceil(index_of(s->low)), 0.0), n - 1.0);
        if (last <= first) last = first + 0.001;       // a step
    }
    for (int i = 0; i < pairs; ++i) {
        const double f = pow(theta, -2.0 * i / n);
        double kept = 1.0;                             // 1: as it is, 0: divided by the factor
        if (s->kind == HG_ROPE_SCALE_LINEAR) kept = 0.0;
        if (s->kind == HG_ROPE_SCALE_TURNS) kept = (s->context * f / two_pi - s->low) / (s->high - s->low);
        if (s->kind == HG_ROPE_SCALE_INDEX) kept = 1.0 - (i - first) / (last - first);
        kept = fmin(fmax(kept, 0.0), 1.0);
        freq[i] = kept == 1.0 ? f : f * kept + f / s->factor * (1.0 - kept);
    }
    if (magnitude) *magnitude = s->kind == HG_ROPE_SCALE_INDEX ? (float)(1.0 + 0.1 * log(s->factor)) : 1.f;
    return HG_OK;
}

hg_status hg_kv_accept(const int32_t* path, const int32_t* n_accept, int32_t max_path, const int32_t* seq_lens, int32_t* new_lens,
                       void* k_cache, void* v_cache, void* stream, const hg_attn_desc* desc) {
    hg_status st = check_pool(desc);
    if (st != HG_OK) return st;
    if (!path || !n_accept || !seq_lens || !k_cache || !v_cache || max_path < 1) return HG_ERR_INVALID_ARG;
    if (!aligned16(k_cache) || !aligned16(v_cache)) return HG_ERR_INVALID_ARG;
    if (max_path > ACCEPT_MAX_PATH) return HG_ERR_UNSUPPORTED;
    const size_t B = (size_t)desc->batch * 4;
    if (overlap(new_lens, B, n_accept, B) || overlap(new_lens, B, path, B * max_path) ||
        overlap(new_lens, B, desc->block_table, B * desc->max_pages) || (new_lens != seq_lens && overlap(new_lens, B, seq_lens, B)))
        return HG_ERR_INVALID_ARG;
    AcceptParams p;
    p.pv = pool_view(desc, k_cache, v_cache);
    p.path = path; p.n_accept = n_accept; p.seq_lens = seq_lens; p.new_lens = new_lens; p.status = desc->status; p.max_path = max_path;
    // a column for every thread, up to the portable size of a cluster
    int cluster = 1;
    while (cluster < 8 && cluster * ACCEPT_THREADS < 2 * desc->num_kv_heads * desc->head_dim / 8) cluster *= 2;
    return launch_draft(kv_accept_kernel, dim3((unsigned)desc->batch * cluster), ACCEPT_THREADS, cluster, stream, p);
}

}  // extern "C"
