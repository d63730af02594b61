// Attention of a step's new tokens over the cache and, masked, over one another (sm_100a).
//
// Token i of sequence b sees the cached positions [begin, len) and the new tokens j, at positions len + j, whose bit its mask
// row has.  Per query head: s = scale <q, k>, m = max s, l = sum e^{s - m}, out = sum e^{s - m} v / l, lse = m + ln l.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "hg_device.cuh"
#include "hg_partial.cuh"

namespace hg {

struct TreeSources {
    const float* o[HG_MAX_MERGE_SRC];
    const float* m[HG_MAX_MERGE_SRC];
    const float* l[HG_MAX_MERGE_SRC];
    int nc[HG_MAX_MERGE_SRC];
    int n;
};

struct TreeParams {
    const uint16_t* q;
    const uint16_t* k;
    const uint16_t* v;
    const int32_t* block_table;
    const int32_t* seq_lens;
    const int32_t* tok_begin;        // or NULL
    const int32_t* cu;
    const uint32_t* mask;            // or NULL: chains
    uint16_t* out;
    float* lse;
    int32_t* status;
    TreeSources src;
    int64_t q_stride, page_stride, head_stride, tok_stride;
    int B, Hq, Hkv, G, N, max_nodes, words;
    int page_size, page_shift, max_pages, num_pages;
    float scale;
    FastDiv div_G;
};

// Simple form: a warp per row and head, token after token.
template <int D, bool BF16>
__global__ void __launch_bounds__(128) tree_kernel(TreeParams p) {
    constexpr int W = D / 64;        // 32-bit words per lane
    const int lane = threadIdx.x & 31;
    const long long id = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
    const int row = (int)(id / p.Hq), h = (int)(id % p.Hq);
    if (row >= p.N || row >= p.cu[p.B] || row < p.cu[0]) return;
    int b = 0;
    for (int above = p.B; above - b > 1;) {
        const int mid = (b + above) >> 1;
        if (p.cu[mid] <= row) b = mid; else above = mid;
    }
    const int i = row - p.cu[b];
    int n = p.cu[b + 1] - p.cu[b], trouble = 0;
    if (n > p.max_nodes) { n = p.max_nodes; trouble = HG_DEV_RANGE; }
    if (i < n) {
        const long long room = (long long)p.max_pages << p.page_shift;
        long long len = max(p.seq_lens[b], 0), end = len + n;
        const int begin = (int)min(len, (long long)max(p.tok_begin ? p.tok_begin[b] : 0, 0));
        if (end > room) { end = room; trouble = HG_DEV_RANGE; }
        const uint16_t* qr = p.q + row * p.q_stride + h * D + lane * 2 * W;
        float2 q[W], o[W];
        for (int w = 0; w < W; ++w) { q[w] = unpack2<BF16>(reinterpret_cast<const uint32_t*>(qr)[w]); o[w] = make_float2(0.f, 0.f); }
        float m = __int_as_float(0xff800000), l = 0.f;
        auto join = [&](float m2, float l2, const float2 (&o2)[W]) {
            if (m2 == __int_as_float(0xff800000)) return;
            const float top = fmaxf(m, m2), a = expf(m - top), c = expf(m2 - top);
            m = top;
            l = l * a + l2 * c;
            for (int w = 0; w < W; ++w) { o[w].x = o[w].x * a + o2[w].x * c; o[w].y = o[w].y * a + o2[w].y * c; }
        };
        for (long long t = begin; t < end; ++t) {
            const long long j = t - len;
            if (j >= 0 && !(p.mask ? (p.mask[(size_t)row * p.words + (j >> 5)] >> (j & 31)) & 1u : j <= i)) continue;
            const long long e = (long long)b * p.max_pages + (t >> p.page_shift), page = p.block_table ? p.block_table[e] : e;
            if (page < 0 || page >= p.num_pages) { trouble |= HG_DEV_BAD_PAGE; continue; }
            const int64_t at = page * p.page_stride + (h / p.G) * p.head_stride + (t & (p.page_size - 1)) * p.tok_stride + lane * 2 * W;
            float s = 0.f;
            float2 v[W];
            for (int w = 0; w < W; ++w) {
                const float2 k = unpack2<BF16>(reinterpret_cast<const uint32_t*>(p.k + at)[w]);
                v[w] = unpack2<BF16>(reinterpret_cast<const uint32_t*>(p.v + at)[w]);
                s += q[w].x * k.x + q[w].y * k.y;
            }
            for (int x = 16; x > 0; x >>= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
            join(s * p.scale, 1.f, v);
        }
        for (int x = 0; x < p.src.n; ++x)
            for (int c = 0; c < p.src.nc[x]; ++c) {
                const size_t at = ((size_t)row * p.Hq + h) * p.src.nc[x] + c;
                float2 o2[W];
                for (int w = 0; w < W; ++w) o2[w] = p.src.m[x][at] == __int_as_float(0xff800000) ? make_float2(0.f, 0.f) :
                    reinterpret_cast<const float2*>(p.src.o[x] + at * D + lane * 2 * W)[w];
                join(p.src.m[x][at], p.src.l[x][at], o2);
            }
        for (int w = 0; w < W; ++w)
            reinterpret_cast<uint32_t*>(p.out + ((size_t)row * p.Hq + h) * D + lane * 2 * W)[w] =
                l == 0.f ? 0u : pack2<BF16>(o[w].x / l, o[w].y / l);
        if (p.lse && lane == 0) p.lse[(size_t)row * p.Hq + h] = l == 0.f ? __int_as_float(0xff800000) : m + logf(l);
    }
    if (trouble && lane == 0 && p.status) atomicOr(p.status, trouble);
}

}  // namespace hg
