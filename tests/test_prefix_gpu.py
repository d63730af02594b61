"""Attention over shared prefixes on the GPU against a plain softmax in 64 bits.

Tolerances.  q and k have components of order 1, so |q| |k| / sqrt(D) is about 14 * 15 / 11.3 = 18.6 at D = 128; a sum of D
products in fp32 has D roundings of at most 2^-24 of that, independent ones: sqrt(128) * 2^-24 * 18.6 * 4 (four standard
deviations) = 5e-5, doubled for an accumulator that truncates: a logit is off by at most 1e-4 (8e-4 where keys are eight
times as large).  The same bound holds for the log-sum-exp.  Weights, normalised, are off by twice that, relatively; their
own rounding (hi + lo terms: 2^-17) is below it, and so is the fp32 sum of weights; half of the weights' errors have the
other sign, and a convex combination of V rows moves by at most the weights' error times max |V|: 1e-4 * max |V|.
"""
import numpy as np
import pytest
import torch

import paper_2604_18529_b200 as pkg
from paper_2604_18529_b200 import binding as hg

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F16, BF16 = torch.float16, torch.bfloat16


def ints(a):
    return torch.tensor(a, dtype=torch.int32, device=DEV)


class Batch:
    """Sequences in groups: row b of the block table lists its group's whole pages, then pages of its own."""

    def __init__(self, group, shared, own, Hq=8, Hkv=2, D=128, P=16, dtype=F16, chunk=256, begin=None, layout="HND", seed=0, spare=3,
                 tables=None, outliers=False, flags=0):
        B, NG = len(group), len(shared)
        self.B, self.NG, self.Hq, self.Hkv, self.D, self.P, self.chunk = B, NG, Hq, Hkv, D, P, chunk
        self.group, self.shared, self.begin = group, shared, begin or [0] * NG
        rep = [group.index(g) if g in group else 0 for g in range(NG)]
        start = [shared[g] if 0 <= g < NG else 0 for g in group]
        self.total = [s + n for s, n in zip(start, own)]
        S = max([-(-t // P) for t in self.total] + [1])
        pages, table, shared_pages = 0, np.full((B, S), -1, dtype=np.int32), {}
        for b, g in enumerate(group):
            m = 0
            if 0 <= g < NG:
                if g not in shared_pages:
                    shared_pages[g] = list(range(pages, pages + shared[g] // P))
                    pages += shared[g] // P
                m = shared[g] // P
                table[b, :m] = shared_pages[g]
            n = -(-self.total[b] // P) - m
            table[b, m:m + n] = range(pages, pages + n)
            pages += n
        n = pages + spare
        perm = np.random.RandomState(seed).permutation(n).astype(np.int32)
        table = np.where(table >= 0, perm[table], -1)
        gen = torch.Generator(device=DEV)
        gen.manual_seed(seed)
        shape = (n, Hkv, P, D) if layout == "HND" else (n, P, Hkv, D)
        k, v = [torch.randn(shape, generator=gen, device=DEV).to(dtype) for _ in range(2)]
        self.q = torch.randn((B, Hq, D), generator=gen, device=DEV).to(dtype)
        if outliers:
            for x in (k, v):
                x.view(-1, D)[::97] *= 8
        if layout == "NHD":
            k, v = k.transpose(1, 2), v.transpose(1, 2)
        self.k, self.v = k, v
        used = set()                                    # rows nobody reads hold NaN: nothing may come of them
        for b, g in enumerate(group):
            for t in range(start[b], self.total[b]):
                used.add((int(table[b, t // P]), t % P))
        for g in range(NG):
            for t in range(self.begin[g], shared[g] if g in group else 0):
                used.add((int(table[rep[g], t // P]), t % P))
        mask = torch.ones((n, P), dtype=torch.bool)
        if used:
            mask[tuple(torch.tensor(sorted(used)).T)] = False
        for x in (self.k, self.v):
            x.masked_fill_(mask.to(DEV)[:, None, :, None], float("nan"))
        self.table, self.status = torch.from_numpy(table).to(DEV), ints([0])
        self.rep, self.tol = rep, 8e-4 if outliers else 1e-4
        self.seq_lens, self.tok_begin, self.tok_end = ints(self.total), ints(start), ints(self.total)
        self.prefix = self.groups(chunk)
        own_chunk = max(64, P)
        self.desc = hg.attn_desc(batch=B, num_q_heads=Hq, num_kv_heads=Hkv, head_dim=D, dtype=dtype, page_size=P, num_pages=n,
                                 page_stride=self.k.stride(0), head_stride=self.k.stride(1), tok_stride=self.k.stride(2),
                                 block_table=self.table, max_pages=S, chunk_tokens=own_chunk, num_chunks=max(own + [0]) // own_chunk + 2,
                                 status=self.status, flags=flags)
        self.NC = self.prefix.num_chunks

    def groups(self, chunk, extra=0):
        nc = max([-(-n // chunk) - b // chunk for n, b in zip(self.shared, self.begin)] + [1]) + extra
        return hg.prefix_desc(seq_group=ints(self.group), group_row=ints(self.rep), group_begin=ints(self.begin),
                              group_end=ints([n if g in self.group else 0 for g, n in enumerate(self.shared)]), chunk_tokens=chunk, num_chunks=nc)

    def rows64(self, pool, row, lo, hi):
        """Token rows [lo, hi) of a block-table row in 64 bits: [Hkv][hi - lo][D]"""
        t = torch.arange(lo, hi, device=DEV)
        page = self.table[row].long()[t // self.P].clamp(0, pool.shape[0] - 1)      # (left-out pages: any, they are dropped)
        return pool[page, :, t % self.P].double().transpose(0, 1)

    def logits64(self, b, row, lo, hi):
        q = self.q[b].double().reshape(self.Hkv, -1, self.D)
        return (q @ self.rows64(self.k, row, lo, hi).transpose(1, 2) * self.D ** -0.5).reshape(self.Hq, hi - lo)

    def values64(self, row, lo, hi):
        return self.rows64(self.v, row, lo, hi).repeat_interleave(self.Hq // self.Hkv, 0)

    def step64(self, drop=()):
        """Out and lse of every sequence; ``drop``: token positions of a shared slice to leave out."""
        out, lse = [], []
        for b, g in enumerate(self.group):
            at = int(self.tok_begin[b])
            s, v = [self.logits64(b, b, at, self.total[b])], [self.values64(b, at, self.total[b])]
            if 0 <= g < self.NG:
                lo, hi = self.begin[g], self.shared[g]
                x = self.logits64(b, self.rep[g], lo, hi)
                y = self.values64(self.rep[g], lo, hi)
                keep = [t - lo for t in range(lo, hi) if t not in drop]
                s.append(x[:, keep])
                v.append(y[:, keep])
            s, v = torch.cat(s, 1), torch.cat(v, 1)
            if s.shape[1] == 0:
                out.append(torch.zeros(self.Hq, self.D, dtype=torch.float64, device=DEV))
                lse.append(torch.full((self.Hq,), float("-inf"), dtype=torch.float64, device=DEV))
                continue
            lse.append(torch.logsumexp(s, 1))
            out.append((torch.softmax(s, 1)[:, None] @ v)[:, 0])
        return torch.stack(out), torch.stack(lse)

    def partial(self, prefix=None, q=None, fill=float("nan")):
        prefix = prefix or self.prefix
        o = torch.full((self.B, self.Hq, prefix.num_chunks, self.D), fill, device=DEV)
        m, l = (torch.full((self.B, self.Hq, prefix.num_chunks), fill, device=DEV) for _ in range(2))
        pkg.hg_attn_prefix_partial(self.q if q is None else q, self.k, self.v, o, m, l, self.desc, prefix)
        return o, m, l

    def step(self, host=(), prefix=None):
        prefix = prefix or self.prefix
        out, lse = torch.full((self.B, self.Hq, self.D), float("nan"), device=DEV), torch.full((self.B, self.Hq), float("nan"), device=DEV)
        ws = torch.empty(pkg.hg_attn_shared_workspace_bytes(self.desc, prefix), dtype=torch.uint8, device=DEV)
        ws.fill_(0xff)
        pkg.hg_attn_decode_shared(self.q, self.k, self.v, self.seq_lens, self.tok_begin, self.tok_end, list(host), out, lse, ws, self.desc,
                                  prefix)
        return out, lse

    def biggest_v(self):
        return float(torch.nan_to_num(self.v.float(), 0.0).abs().max())


def close(batch, got, want, what=""):
    out, lse = got[0].double(), got[1].double()
    assert not out.isnan().any() and not lse.isnan().any(), what
    finite = want[1].isfinite()
    assert torch.equal(lse.isfinite(), finite), what
    assert (out - want[0]).abs().max() <= batch.tol * max(1.0, batch.biggest_v()), (what, float((out - want[0]).abs().max()))
    if finite.any():
        assert (lse[finite] - want[1][finite]).abs().max() <= batch.tol, what


def check_step(batch, status=0, drop=(), **kw):
    close(batch, batch.step(**kw), batch.step64(drop))
    assert int(batch.status) == status


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(4, 4), (8, 2), (16, 2), (7, 1), (24, 1)])
def test_types_heads_and_head_groups(dtype, D, Hq, Hkv):
    check_step(Batch([0, 0, 1, -1, 0, 1], [300, 77], [5, 40, 1, 90, 0, 17], Hq, Hkv, D, 16, dtype, seed=Hq))


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 255, 256, 257, 383, 700, 1025])
def test_prefix_lengths(n):
    check_step(Batch([0, 0, 0], [n], [3, 1, 20], seed=n))


@pytest.mark.parametrize("members", [1, 2, 7, 8, 15, 16, 17, 31, 32, 33, 40, 63, 64, 65, 70, 100])
def test_numbers_of_members(members):
    """1 .. 400 rows per KV head: part of a row tile, whole ones, several."""
    check_step(Batch([0] * members, [333], [members % 5] * members, 8, 2, 64, 16, seed=members))
    check_step(Batch([0] * members, [333], [members % 5] * members, 3, 3, 128, 32, BF16, seed=members))


@pytest.mark.parametrize("layout", ["HND", "NHD"])
@pytest.mark.parametrize("P", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("D", [64, 128])
def test_page_sizes_and_layouts(P, layout, D):
    check_step(Batch([0, 1, 0, 1, 1], [517, 260], [30, 1, 200, 0, 65], 8, 4, D, P, BF16, 256, layout=layout, seed=P))
    check_step(Batch([0] * 40, [2 * P + 1], [1] * 40, 16, 2, D, P, F16, 256, layout=layout, seed=P + 1))


@pytest.mark.parametrize("chunk,begin", [(128, 0), (128, 1), (256, 130), (512, 511), (512, 512), (2048, 700), (128, 1199), (128, 1200)])
def test_chunk_grids_and_slices_that_begin_late(chunk, begin):
    """Chunks sit on absolute multiples of chunk_tokens; an empty slice is an empty source."""
    b = Batch([0, 0, 0, 0, 0], [1200], [4, 30, 0, 1, 2], 8, 1, 128, 16, F16, chunk, begin=[begin], seed=chunk + begin)
    check_step(b)
    o, m, l = b.partial(b.groups(chunk, extra=2))
    for c in range(m.shape[2]):
        lo, hi = max(begin, (begin // chunk + c) * chunk), min(1200, (begin // chunk + c + 1) * chunk)
        if lo >= hi:
            assert torch.equal(m[:, :, c], torch.full_like(m[:, :, c], float("-inf"))) and not l[:, :, c].any() and not o[:, :, c].any()
            continue
        for s in range(5):
            x = b.logits64(s, 0, lo, hi)
            assert (m[s, :, c].double() - x.amax(1)).abs().max() <= b.tol, (c, s)
            w = (x - m[s, :, c].double()[:, None]).exp()
            assert ((l[s, :, c].double() - w.sum(1)) / w.sum(1)).abs().max() <= 1e-4
            want = (w[:, None] @ b.values64(0, lo, hi))[:, 0] / w.sum(1)[:, None]
            assert (o[s, :, c].double() / l[s, :, c].double()[:, None] - want).abs().max() <= 1e-4 * b.biggest_v()


def test_many_groups_of_all_sizes_and_sequences_without_one():
    r = np.random.RandomState(3)
    group = r.randint(-1, 41, 150).tolist() + [40, 39]
    shared = r.randint(1, 600, 41).tolist()
    shared[5] = 0
    check_step(Batch(group, shared, r.randint(0, 100, 152).tolist(), 8, 2, 64, 16, BF16, 128, seed=9))


def test_most_groups_and_a_large_batch():
    n = hg.HG_MAX_GROUPS
    r = np.random.RandomState(4)
    group = list(range(n)) + r.randint(0, n, 700 - n).tolist()
    check_step(Batch(group, r.randint(1, 200, n).tolist(), [1] * 700, 2, 1, 64, 16, F16, 128, seed=10))


def test_group_numbers_outside_the_range_share_nothing():
    check_step(Batch([0, -7, 1, 5, 0], [100, 30], [5, 6, 7, 8, 0], seed=2))


def test_all_sequences_without_a_group_and_nothing_at_all():
    b = Batch([-1, -1, -1], [10], [50, 0, 7], seed=2)
    check_step(b)
    o, m, l = b.partial()
    assert torch.equal(m, torch.full_like(m, float("-inf"))) and not l.any() and not o.any()


def test_sparse_empty_leaves_the_rows_of_empty_slots():
    b = Batch([0, -1], [100], [5, 5], chunk=128, seed=2, flags=hg.HG_FLAG_SPARSE_EMPTY)
    o, m, l = b.partial(b.groups(128, extra=1), fill=3.0)
    assert (o[1] == 3).all() and (o[0, :, 1] == 3).all() and (l[1] == 0).all() and torch.isinf(m[1]).all() and (o[0, :, 0] != 3).any()


def test_long_prefix_and_outliers():
    """Maxima that move late and by much: the running rescale."""
    check_step(Batch([0] * 9 + [1], [20000, 9000], [10] * 10, 16, 2, 128, 64, BF16, 2048, outliers=True, seed=6))
    check_step(Batch([0] * 40, [5000], [1] * 40, 16, 2, 64, 16, F16, 1024, outliers=True, seed=7))


def test_rising_logits():
    """Every token's logit above the last one's: the maximum moves in every tile, by more than any threshold."""
    b = Batch([0] * 20, [1500], [0] * 20, 8, 1, 128, 16, F16, 2048, seed=8)
    t = torch.arange(1500, device=DEV)
    at = b.table[0].long()[t // 16]
    b.q.fill_(0)
    b.q[..., 0] = 11.3125
    b.k[at, :, t % 16] = 0
    b.k[at, :, t % 16, 0] = (t.float() / 8)[:, None].to(F16)
    check_step(b)


def test_unmapped_and_bad_pages_inside_the_slice_are_left_out():
    for P, members in ((16, 3), (16, 40), (64, 40), (128, 3), (256, 40)):
        n = 5 * P + 300
        b = Batch([0] * members, [n], [1] * members, 8, 1, 128, P, F16, 256 * (P // 256 or 1), seed=P + members)
        drop = set()
        for slot, e in ((1, -1), (3, 10 ** 6)):
            b.table[0, slot] = e                        # (row 0 is the group's representative)
            drop |= set(range(slot * P, (slot + 1) * P))
        check_step(b, hg.HG_DEV_BAD_PAGE, drop)
        # a whole tile, a whole chunk
        b.status.zero_()
        b.table[0, : n // P] = -1
        check_step(b, hg.HG_DEV_BAD_PAGE, set(range(n // P * P)))


def test_slices_past_the_table_are_cut():
    b = Batch([0, 0], [100], [28, 12], P=16, seed=1)
    b.prefix._keep[3].fill_(10 ** 6)
    b.tok_begin.copy_(b.tok_end)                        # nothing of their own: the slice covers row 0's 128 positions
    out, lse = b.step()
    for s in range(2):
        x = b.logits64(s, 0, 0, 128)
        assert (out[s].double() - (torch.softmax(x, 1)[:, None] @ b.values64(0, 0, 128))[:, 0]).abs().max() <= b.tol * b.biggest_v()
    assert int(b.status) == hg.HG_DEV_RANGE
    b.status.zero_()
    b.prefix._keep[1].fill_(2)                          # a row that is not there: an empty group
    out, lse = b.step()
    assert torch.isinf(lse).all() and not out.any() and int(b.status) == hg.HG_DEV_RANGE


def test_own_scale():
    b = Batch([0, 0], [200], [9, 1], D=64, seed=1)
    b.desc.scale = 0.25
    out, lse = b.step()
    for s in range(2):
        x = torch.cat([b.logits64(s, 0, 0, 200), b.logits64(s, s, 200, b.total[s])], 1) * 2
        assert (lse[s].double() - torch.logsumexp(x, 1)).abs().max() <= 1e-4


def test_host_partials_join_and_identity_paging():
    """A further source, and a cache without a block table (rows of the table are rows of pages)."""
    b = Batch([0, 0, 0], [90], [7, 8, 1], 8, 2, 64, 16, seed=3)
    m = torch.randn(3, 8, 1, device=DEV)
    o, l = torch.randn(3, 8, 1, 64, device=DEV), torch.rand(3, 8, 1, device=DEV) + 0.5
    out, lse = b.step(host=[(o, m, l)])
    want_out, want_lse = b.step64()
    w = (m[..., 0].double() + l[..., 0].double().log())
    both = torch.logaddexp(want_lse, w)
    want = want_out * (want_lse - both).exp()[..., None] + o[:, :, 0].double() / l.double() * (w - both).exp()[..., None]
    close(b, (out, lse), (want, both))
    c = Batch([0], [250], [0], 8, 2, 64, 16, seed=4)
    order = c.table[0].long()
    c.k, c.v = c.k[order].contiguous(), c.v[order].contiguous()
    want = c.k, c.v
    c.desc.block_table, c.desc.num_pages = None, len(order)
    c.table.copy_(torch.arange(len(order), dtype=torch.int32)[None])
    check_step(c)


def test_same_bits_as_often_as_it_runs_and_for_any_neighbours():
    b = Batch([0] * 45 + [1, -1], [3000, 500], [9] * 47, 16, 2, 128, 16, BF16, 512, seed=12)
    first = b.step()
    for _ in range(5):
        again = b.step()
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    # a row's partials do not depend on what stands in the other rows
    q = b.q.clone()
    one = b.partial()
    b.q[1:44] *= 30
    two = b.partial()
    for x, y in zip(one, two):
        assert torch.equal(x[0], y[0]) and torch.equal(x[44:], y[44:])
    b.q.copy_(q)


def test_a_wait_that_runs_out_is_reported():
    """The loader never fills a tile: the call returns with a status bit, the next ones skip their work until it is cleared."""
    b = Batch([0, 0, 0], [300], [1, 2, 3], seed=15)
    b.desc.flags = hg.HG_FLAG_TEST_STALL
    b.partial()
    torch.cuda.synchronize()
    assert int(b.status) == hg.HG_DEV_WAIT_TIMEOUT
    b.desc.flags = 0
    o, m, l = b.partial()
    torch.cuda.synchronize()
    assert o.isnan().all() and m.isnan().all() and l.isnan().all()
    b.status.zero_()
    check_step(b)


def test_captured_on_another_stream_beside_a_second_call():
    """Two steps on two streams at once, each with its own workspace; one of them captured and replayed on new queries."""
    a = Batch([0] * 20, [4000], [30] * 20, 16, 2, 128, 16, F16, 512, seed=13)
    b = Batch([0] * 9 + [1] * 9, [2000, 300], [30] * 18, 8, 8, 64, 32, BF16, 256, seed=14)
    out, lse = torch.empty(a.B, a.Hq, a.D, device=DEV), torch.empty(a.B, a.Hq, device=DEV)
    ws = torch.empty(pkg.hg_attn_shared_workspace_bytes(a.desc, a.prefix), dtype=torch.uint8, device=DEV)
    s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=s):
        pkg.hg_attn_decode_shared(a.q, a.k, a.v, a.seq_lens, a.tok_begin, a.tok_end, [], out, lse, ws, a.desc, a.prefix)
    torch.cuda.synchronize()
    for k in range(3):
        a.q.copy_(torch.randn_like(a.q.float()).to(F16))
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            g.replay()
        got = b.step()
        torch.cuda.synchronize()
        close(a, (out, lse), a.step64())
        close(b, got, b.step64())


def test_page_offsets_past_32_bits():
    """Pages that start beyond 2^31 elements."""
    D, P, n = 64, 16, 3
    stride = (1 << 31) + 8 * 1024
    whole = [torch.zeros(2 * stride + 2 * P * D, dtype=F16, device=DEV) for _ in range(2)]
    k, v = [x.as_strided((n, 1, P, D), (stride, P * D, D, 1)) for x in whole]
    for x in (k, v):
        x[1:].copy_(torch.randn(2, 1, P, D))
    b = Batch([0, 0], [32], [0, 0], 4, 1, D, P, F16, 128, seed=1)
    b.k, b.v = k, v
    b.table[:, :2] = ints([2, 1])
    b.desc.num_pages, b.desc.page_stride, b.desc.head_stride, b.desc.tok_stride = n, stride, P * D, D
    check_step(b)


def test_more_rows_per_sequence_than_an_item_has():
    check_step(Batch([0, 0, -1, 0], [300], [20, 0, 5, 131], Hq=300, Hkv=1, seed=12))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("own_chunk", [64, 192, 320])
def test_own_chunks_that_begin_inside_a_tile(own_chunk, D):
    b = Batch([0, 0, -1], [200], [330, 1, 700], seed=3, D=D)
    b.desc.chunk_tokens, b.desc.num_chunks = own_chunk, 700 // own_chunk + 2
    check_step(b)


def test_the_partials_do_not_use_the_own_chunk_fields():
    b = Batch([0, 0], [300], [5, 5], seed=9)
    want = b.partial()
    b.desc.chunk_tokens = b.desc.num_chunks = 0
    for x, y in zip(b.partial(), want):
        assert torch.equal(x, y)


def test_refused_by_the_binding():
    b = Batch([0, 0], [100], [5, 5], seed=2)
    o, m, l = b.partial()
    with pytest.raises(ValueError):
        pkg.hg_attn_prefix_partial(b.q[:1].contiguous(), b.k, b.v, o, m, l, b.desc, b.prefix)
    with pytest.raises(ValueError):
        pkg.hg_attn_prefix_partial(b.q, b.k, b.v, o, m[:1].contiguous(), l, b.desc, b.prefix)
    with pytest.raises(ValueError):
        pkg.hg_attn_prefix_partial(b.q.cpu(), b.k, b.v, o, m, l, b.desc, b.prefix)
    short = hg.prefix_desc(seq_group=ints([0]), group_row=ints([0]), group_begin=ints([0]), group_end=ints([9]), chunk_tokens=128, num_chunks=1)
    with pytest.raises(ValueError):
        pkg.hg_attn_prefix_partial(b.q, b.k, b.v, o, m, l, b.desc, short)
    with pytest.raises(ValueError):
        hg.prefix_desc(seq_group=ints([0]), group_row=ints([0]), group_begin=ints([0, 0]), group_end=ints([9]), chunk_tokens=128, num_chunks=1)


def test_fork_reserve_append_attend_compact():
    """The operators as they are used together: one prompt, branches by fork, new tokens by reserve + copy + append, the
    step over the shared prefix, the pool compacted under it - against a plain softmax over every branch's own tokens."""
    P, Hkv, Hq, D, B, n, S = 16, 2, 8, 64, 6, 60, 8
    gen = torch.Generator(device=DEV)
    gen.manual_seed(1)
    rnd = lambda *s: torch.randn(s, generator=gen, device=DEV).to(F16)   # noqa: E731
    k, v = torch.full((n, Hkv, P, D), float("nan"), dtype=F16, device=DEV), torch.full((n, Hkv, P, D), float("nan"), dtype=F16, device=DEV)
    table, ref, status = torch.full((B, S), -1, dtype=torch.int32, device=DEV), ints([0] * n), ints([0])
    lens, begin, end = ints([0] * B), ints([0] * B), ints([0] * B)
    cs, cd, cr, ready, nm, remap = ints([0] * B), ints([0] * B), ints([0] * B), ints([0] * B), ints([0]), ints([0] * n)
    ms, md = ints([0] * n), ints([0] * n)
    desc = hg.attn_desc(batch=B, num_q_heads=Hq, num_kv_heads=Hkv, head_dim=D, dtype=F16, page_size=P, num_pages=n, page_stride=k.stride(0),
                        head_stride=k.stride(1), tok_stride=k.stride(2), block_table=table, max_pages=S, chunk_tokens=64, num_chunks=3,
                        status=status)
    said = [[] for _ in range(B)]

    def append(new):
        """one token for the rows of `new`"""
        pkg.hg_kv_reserve(lens, ints([int(b in new) for b in range(B)]), ref, cs, cd, cr, ready, desc)
        pkg.hg_kv_copy_pages(cs, cd, cr, None, k, v, desc)
        kn, vn = rnd(B, Hkv, D), rnd(B, Hkv, D)
        before = lens.clone()
        pkg.hg_kv_append(kn, vn, k, v, lens, end, desc)            # rows without a page drop theirs
        status.zero_()
        keep = ints([int(b in new) for b in range(B)])
        lens.copy_(torch.where(keep > 0, lens, before))
        end.copy_(lens)
        for b in new:
            said[b].append((kn[b], vn[b]))

    for _ in range(37):
        append([0])
    shared = 37
    pkg.hg_kv_fork(ints([0] * 5 + [-1]), ref, lens, begin, end, desc)   # rows 1..4 branch off
    for b in range(1, 5):
        said[b] = list(said[0])
    for step in range(25):
        append([0, 1, 2, 3, 4])
        if step == 12:                                             # row 3 goes on from row 1, row 2 ends
            pkg.hg_kv_fork(ints([0, 1, -1, 1, 4, 5]), ref, lens, begin, end, desc)
            said[3], said[2] = list(said[1]), []
            for _ in range(2):
                append([3])
            break
    pkg.hg_kv_compact(ref, remap, ms, md, nm, desc)
    pkg.hg_kv_copy_pages(ms, md, None, nm, k, v, desc)
    used = int((ref > 0).sum())
    assert int(table.max()) == used - 1 and int(nm) > 0
    group = [0, 0, -1, 0, 0, -1]
    begin.copy_(ints([shared if g == 0 else 0 for g in group]))
    prefix = hg.prefix_desc(seq_group=ints(group), group_row=ints([4]), group_begin=ints([0]), group_end=ints([shared]), chunk_tokens=128,
                            num_chunks=1)
    q, out, lse = rnd(B, Hq, D), torch.empty(B, Hq, D, device=DEV), torch.empty(B, Hq, device=DEV)
    ws = torch.empty(pkg.hg_attn_shared_workspace_bytes(desc, prefix), dtype=torch.uint8, device=DEV)
    pkg.hg_attn_decode_shared(q, k, v, lens, begin, end, [], out, lse, ws, desc, prefix)
    assert int(status) == 0
    assert lens.tolist() == [len(x) for x in said] == [50, 50, 0, 52, 50, 0]
    for b in range(B):
        if not said[b]:
            assert torch.isinf(lse[b]).all() and not out[b].any()
            continue
        K, V = [torch.stack([x[i] for x in said[b]], 1).double().repeat_interleave(Hq // Hkv, 0) for i in (0, 1)]
        x = (q[b].double()[:, None] @ K.transpose(1, 2))[:, 0] * D ** -0.5
        assert (lse[b].double() - torch.logsumexp(x, 1)).abs().max() <= 1e-4
        assert (out[b].double() - (torch.softmax(x, 1)[:, None] @ V)[:, 0]).abs().max() <= 1e-4 * float(V.abs().max())


@pytest.mark.parametrize("own_chunk,slots", [(64, 6), (64, 26), (128, 4), (128, 14), (192, 5), (192, 10)])
@pytest.mark.parametrize("D,B,Hq", [(128, 96, 8), (64, 70, 4)])
def test_own_slices_of_several_chunks_in_a_large_batch(own_chunk, slots, D, B, Hq):
    """Many short own chunks, slices that begin anywhere in one; what does not fit the caller's chunk slots is left out, as
    hg_attn_partial does it, whatever grid the call works on."""
    r = np.random.RandomState(own_chunk + slots + D)
    group = r.randint(-1, 3, B).tolist()
    b = Batch(group, [77, 300, 515], r.randint(200, 1500, B).tolist(), Hq, 4, D, 16, F16, 256, seed=slots)
    b.desc.chunk_tokens, b.desc.num_chunks = own_chunk, slots
    assert B * 4 * slots >= 1024
    got = b.step()
    b.total = [min(t, (int(lo) // own_chunk + slots) * own_chunk) for t, lo in zip(b.total, b.tok_begin.tolist())]
    close(b, got, b.step64())
    assert int(b.status) == 0
