// Host-side helpers shared by the translation units of the C ABI: argument validation, the driver's tensor-map
// encoder, the optional tuning fields of a description.
#pragma once

#include "hybridgen_attn.h"

#include <cuda.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stddef.h>
#include <string.h>

#include "hg_poolview.cuh"
#include "hg_partial.cuh"

namespace hg {

constexpr int kMaxDevices = 64;

// ---- validation ------------------------------------------------------------------------------------

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// The optional trailing field, for callers compiled against a shorter struct.
inline int32_t* desc_sched(const hg_attn_desc* d) {
    return d->struct_size >= offsetof(hg_attn_desc, sched_counter) + sizeof(int32_t*) ? d->sched_counter : nullptr;
}

// Multiplier and shift that divide a number below 2^31 by d (see FastDiv).
inline FastDiv make_fast_div(uint32_t d) {
    FastDiv f = {0u, 0u};
    if (d <= 1) return f;
    uint32_t s = 0;
    while ((1ull << s) < d) ++s;                                   // ceil(log2 d) >= 1
    f.mul = (uint32_t)(((1ull << (31 + s)) + d - 1) / d);          // < 2^32 because d > 2^(s-1)
    f.shift = s - 1;
    return f;
}

inline int ilog2_exact(int v) {
    for (int s = 0; s < 31; ++s)
        if ((1 << s) == v) return s;
    return -1;
}

// Checks the fields every entry point relies on.  `need_kv` also checks the KV addressing.
inline hg_status check_desc(const hg_attn_desc* d, bool need_kv) {
    if (!d || d->struct_size < offsetof(hg_attn_desc, sched_counter)) return HG_ERR_INVALID_ARG;
    if (d->batch < 1 || d->batch > 65535) return HG_ERR_INVALID_ARG;
    if (d->num_kv_heads < 1 || d->num_q_heads < 1 || d->num_q_heads % d->num_kv_heads) return HG_ERR_INVALID_ARG;
    if (d->head_dim <= 0 || d->head_dim % 8) return HG_ERR_INVALID_ARG;
    if (d->head_dim != 64 && d->head_dim != 128) return HG_ERR_UNSUPPORTED;
    if (!need_kv) return HG_OK;
    if (d->dtype != HG_DTYPE_F16 && d->dtype != HG_DTYPE_BF16) return HG_ERR_INVALID_ARG;
    if (d->page_size < 1 || d->num_pages < 1 || d->max_pages < 1) return HG_ERR_INVALID_ARG;
    if (d->page_stride < 0 || d->head_stride < 0 || d->tok_stride < d->head_dim) return HG_ERR_INVALID_ARG;
    if ((d->page_stride | d->head_stride | d->tok_stride) & 7) return HG_ERR_INVALID_ARG;   // 16-byte multiples
    if (d->chunk_tokens < 1 || d->num_chunks < 1) return HG_ERR_INVALID_ARG;
    if (!(d->scale >= 0.f) || isinf(d->scale)) return HG_ERR_INVALID_ARG;
    const int shift = ilog2_exact(d->page_size);
    if (shift < 4 || shift > 8) return HG_ERR_UNSUPPORTED;                                   // 16 .. 256
    if (d->chunk_tokens % TILE_T || d->chunk_tokens % d->page_size || d->chunk_tokens > 65536)
        return HG_ERR_UNSUPPORTED;
    if (d->chunk_tokens / d->page_size > MAX_CHUNK_PAGES) return HG_ERR_UNSUPPORTED;
    if (desc_sched(d) && (reinterpret_cast<uintptr_t>(desc_sched(d)) & 7u)) return HG_ERR_INVALID_ARG;
    if ((int64_t)d->num_kv_heads * ((d->num_q_heads / d->num_kv_heads + 7) / 8) > 65535) return HG_ERR_UNSUPPORTED;
    if (!d->block_table && (int64_t)d->batch * d->max_pages > d->num_pages) return HG_ERR_INVALID_ARG;
    return HG_OK;
}

// Two arrays that share memory.
inline bool overlap(const void* a, size_t a_bytes, const void* b, size_t b_bytes) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return a && b && a_bytes && b_bytes && x < y + b_bytes && y < x + a_bytes;
}
// Two packed tensors of n rows, `width` 16-bit elements wide and `stride` apart, that share memory.  Rows of the same stride may lie
// between one another (parts of a fused projection's output).
inline bool rows_overlap(const void* a, int64_t a_stride, int64_t a_width, const void* b, int64_t b_stride, int64_t b_width, int64_t n) {
    if (!overlap(a, (size_t)((n - 1) * a_stride + a_width) * 2, b, (size_t)((n - 1) * b_stride + b_width) * 2)) return false;
    if (a_stride != b_stride || n == 1) return true;
    const int64_t apart = (int64_t)(reinterpret_cast<uintptr_t>(b) - reinterpret_cast<uintptr_t>(a)) / 2, d = (apart % b_stride + b_stride) % b_stride;
    return d < a_width || d + b_width > b_stride;
}

// ---- tensor maps -------------------------------------------------------------------------------------

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline EncodeTiledFn encode_fn() {
    static EncodeTiledFn fn = []() -> EncodeTiledFn {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess)
            return nullptr;
        return reinterpret_cast<EncodeTiledFn>(f);
    }();
    return fn;
}

// The pool as in hg_attn_partial, {d within a 64-element half, token in page, half, head, page}, but ONE half a box: the
// tensor cores want the token rows of a tile's half at one stride, whatever the page size.
inline hg_status make_tile_maps(const hg_attn_desc* d, const void* k, const void* v, int tile, CUtensorMap* tk, CUtensorMap* tv) {
    EncodeTiledFn enc = encode_fn();
    if (!enc) return HG_ERR_CUDA;
    cuuint64_t dims[5] = {64, (cuuint64_t)d->page_size, (cuuint64_t)(d->head_dim / 64), (cuuint64_t)d->num_kv_heads, (cuuint64_t)d->num_pages};
    cuuint64_t strides[4] = {(cuuint64_t)d->tok_stride * 2u, 128u, (cuuint64_t)d->head_stride * 2u, (cuuint64_t)d->page_stride * 2u};
    if (d->num_kv_heads == 1) strides[2] = strides[0];     // unused dimensions still need a legal stride
    if (d->num_pages == 1) strides[3] = strides[0];
    cuuint32_t box[5] = {64, (cuuint32_t)(d->page_size < tile ? d->page_size : tile), 1, 1, 1};
    cuuint32_t estr[5] = {1, 1, 1, 1, 1};
    const CUtensorMapDataType dt = d->dtype == HG_DTYPE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    const void* base[2] = {k, v};
    CUtensorMap* out[2] = {tk, tv};
    for (int i = 0; i < 2; ++i)
        if (enc(out[i], dt, 5, const_cast<void*>(base[i]), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
            return HG_ERR_UNSUPPORTED;   // a stride pattern the TMA unit cannot express
    return HG_OK;
}

// The optional tuning fields (all defaults when the caller's struct ends before them).
struct Tune {
    uint32_t bits;
    int stages, ctas_per_sm;
    bool off(uint32_t bit) const { return (bits & bit) != 0; }
};

inline Tune desc_tune(const hg_attn_desc* d) {
    Tune t = {0u, 0, 0};
    if (d->struct_size >= offsetof(hg_attn_desc, tune_ctas_per_sm) + sizeof(int32_t)) {
        t.bits = d->tune; t.stages = d->tune_stages; t.ctas_per_sm = d->tune_ctas_per_sm;
    }
    return t;
}

inline size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

// The KV addressing fields only (chunking is irrelevant to residency operations).
inline hg_status check_pool(const hg_attn_desc* d) {
    if (!d || d->struct_size < offsetof(hg_attn_desc, sched_counter)) return HG_ERR_INVALID_ARG;
    hg_attn_desc t;
    memset(&t, 0, sizeof t);
    memcpy(&t, d, d->struct_size < sizeof t ? d->struct_size : sizeof t);
    t.chunk_tokens = t.page_size > TILE_T ? t.page_size : TILE_T;
    t.num_chunks = 1;
    t.sched_counter = nullptr;
    t.struct_size = sizeof t;
    return check_desc(&t, true);
}

inline KvPoolView pool_view(const hg_attn_desc* d, const void* k, const void* v) {
    KvPoolView pv;
    pv.k = static_cast<uint16_t*>(const_cast<void*>(k));
    pv.v = static_cast<uint16_t*>(const_cast<void*>(v));
    pv.block_table = d->block_table;
    pv.page_stride = d->page_stride; pv.head_stride = d->head_stride; pv.tok_stride = d->tok_stride;
    pv.B = d->batch; pv.Hkv = d->num_kv_heads; pv.D = d->head_dim; pv.page_size = d->page_size;
    pv.page_shift = ilog2_exact(d->page_size); pv.max_pages = d->max_pages; pv.num_pages = d->num_pages;
    return pv;
}

}  // namespace hg
