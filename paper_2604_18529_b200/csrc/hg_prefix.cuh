// Softmax partials over a prefix that several sequences share, computed once for all of them (sm_100a).
//
// Group g of sequences reads the tokens [begin_g, end_g) of ONE block-table row.  For a KV head the queries of the
// group's members, G per member, are the rows of a matrix Q (R = members x G rows), and per chunk of tokens
//     S = Q K^T,   m = row max of scale S,   P = e^{scale S - m},   l = row sum of P,   o = P V
// is what hg_attn_partial computes for one sequence at a time, with K and V read once instead of once per member.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "hg_device.cuh"

namespace hg {

struct PrefixParams {
    const uint16_t* q;               // [B][Hq][D]
    const uint16_t* k;
    const uint16_t* v;
    const int32_t* block_table;      // [B][max_pages], or NULL: identity paging
    const int32_t* seq_group;        // [B]
    const int32_t* group_row;        // [NG]
    const int32_t* group_begin;      // [NG]
    const int32_t* group_end;        // [NG]
    float* o_part;                   // [B][Hq][NC][D]
    float* m_part;                   // [B][Hq][NC]
    float* l_part;
    int32_t* status;
    int64_t page_stride, head_stride, tok_stride;
    int B, Hq, Hkv, G, NG, NC, C;
    int page_size, page_shift, max_pages, num_pages;
    int sparse_empty;
    float scale;
};

// The slice of a group, clamped to its block-table row, and its chunks.
struct GroupSlice { int row, begin, end, chunk0, nc; bool bad; };

__device__ __forceinline__ GroupSlice group_slice(const PrefixParams& p, int g) {
    GroupSlice s;
    s.row = p.group_row[g];
    s.begin = max(p.group_begin[g], 0);
    s.end = p.group_end[g];
    s.bad = false;
    const long long room = (long long)p.max_pages << p.page_shift;
    if (s.end > room) { s.end = (int)room; s.bad = true; }
    if (s.end > s.begin && (s.row < 0 || s.row >= p.B)) { s.end = s.begin; s.bad = true; }
    s.chunk0 = s.begin / p.C;
    s.nc = s.end > s.begin ? min((s.end - 1) / p.C - s.chunk0 + 1, p.NC) : 0;
    return s;
}

constexpr int PFX_ROWS = 32, PFX_TOK = 16, PFX_THREADS = 256;

// One CTA per (chunk, KV head and block of 32 rows, group); group NG stands for the sequences without one.
template <int D, bool BF16>
__global__ void __launch_bounds__(PFX_THREADS) prefix_partial_kernel(const PrefixParams p, int row_blocks) {
    const float NEG_INF = __int_as_float(0xff800000);
    __shared__ float qs[PFX_ROWS][D + 1], ks[PFX_TOK][D + 1], vs[PFX_TOK][D], ss[PFX_ROWS][PFX_TOK + 1];
    __shared__ int rows[PFX_ROWS], phys[PFX_TOK];
    const int tid = threadIdx.x, g = blockIdx.z, c = blockIdx.x, h = blockIdx.y / row_blocks, rb = blockIdx.y % row_blocks;
    if (tid < PFX_ROWS) {
        // row r of the group: head r % G of its member number r / G
        const int r = rb * PFX_ROWS + tid, want = r / p.G;
        int found = -1, n = 0;
        for (int b = 0; b < p.B; ++b) {
            const int sg = p.seq_group[b];
            const bool in = g < p.NG ? sg == g : (sg < 0 || sg >= p.NG);
            if (in && n++ == want) found = b;
        }
        rows[tid] = found < 0 ? -1 : found * p.Hq + h * p.G + r % p.G;
    }
    __syncthreads();
    if (rows[0] < 0) return;
    GroupSlice sl;
    sl.nc = 0;
    if (g < p.NG) {
        sl = group_slice(p, g);
        if (sl.bad && tid == 0 && p.status) atomicOr(p.status, HG_DEV_RANGE);
    }
    if (c >= sl.nc) {
        for (int r = 0; r < PFX_ROWS && rows[r] >= 0; ++r) {
            const size_t slot = (size_t)rows[r] * p.NC + c;
            if (tid == 0) { p.m_part[slot] = NEG_INF; p.l_part[slot] = 0.f; }
            if (!p.sparse_empty && tid < D) p.o_part[slot * D + tid] = 0.f;
        }
        return;
    }
    const int t_lo = max(sl.begin, (sl.chunk0 + c) * p.C), t_hi = min(sl.end, (sl.chunk0 + c + 1) * p.C);
    for (int i = tid; i < PFX_ROWS * D; i += PFX_THREADS) {
        const int r = i / D, d = i % D;
        float x = 0.f;
        if (rows[r] >= 0) {
            const uint16_t w = p.q[(size_t)rows[r] * D + d];
            x = unpack2<BF16>((uint32_t)w).x;
        }
        qs[r][d] = x;
    }
    const int row = tid / 8, part = tid % 8;                       // eight threads per row
    constexpr int PER = D / 8;
    float acc[PER], m = NEG_INF, l = 0.f;
    for (int i = 0; i < PER; ++i) acc[i] = 0.f;
    for (int t0 = t_lo; t0 < t_hi; t0 += PFX_TOK) {
        const int n = min(PFX_TOK, t_hi - t0);
        __syncthreads();
        if (tid < n) {
            const int pg = (t0 + tid) >> p.page_shift;
            int e = p.block_table ? p.block_table[(size_t)sl.row * p.max_pages + pg] : sl.row * p.max_pages + pg;
            if (e < 0 || e >= p.num_pages) { e = -1; if (p.status) atomicOr(p.status, HG_DEV_BAD_PAGE); }
            phys[tid] = e;
        }
        __syncthreads();
        for (int i = tid; i < n * D; i += PFX_THREADS) {
            const int t = i / D, d = i % D;
            float a = 0.f, b = 0.f;
            if (phys[t] >= 0) {
                const int64_t off = (int64_t)phys[t] * p.page_stride + (int64_t)h * p.head_stride +
                                    (int64_t)((t0 + t) & (p.page_size - 1)) * p.tok_stride + d;
                a = unpack2<BF16>((uint32_t)p.k[off]).x;
                b = unpack2<BF16>((uint32_t)p.v[off]).x;
            }
            ks[t][d] = a;
            vs[t][d] = b;
        }
        __syncthreads();
        float mx = NEG_INF;
        for (int t = part; t < n; t += 8) {
            float s = 0.f;
            for (int d = 0; d < D; ++d) s = fmaf(qs[row][d], ks[t][d], s);
            s = phys[t] >= 0 ? s * p.scale : NEG_INF;
            ss[row][t] = s;
            mx = fmaxf(mx, s);
        }
        for (int o = 1; o < 8; o <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
        __syncwarp();
        if (mx > m) {
            const float r = expf(m - mx);
            l *= r;
            for (int i = 0; i < PER; ++i) acc[i] *= r;
            m = mx;
        }
        if (m != NEG_INF)
            for (int t = 0; t < n; ++t) {
                const float w = expf(ss[row][t] - m);
                l += w;
                for (int i = 0; i < PER; ++i) acc[i] = fmaf(w, vs[t][i * 8 + part], acc[i]);
            }
    }
    if (rows[row] < 0) return;
    const size_t slot = (size_t)rows[row] * p.NC + c;
    if (part == 0) { p.m_part[slot] = m; p.l_part[slot] = l; }
    for (int i = 0; i < PER; ++i) p.o_part[slot * D + i * 8 + part] = acc[i];
}

}  // namespace hg
