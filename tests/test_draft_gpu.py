"""Slot maps, rotary positions, accepted paths and a whole step of speculative decoding on the GPU.

Tolerances of the rotation.  A turned component is a c - b s with a, b of size at most M (the largest input): the sine and
cosine are of an angle that is off by at most pi * 2^-24 (the fp32 fraction of a turn) and have at most 2 ulp themselves, 2^-22;
together with two products and a sum in fp32 less than 2^-20 M; then it is rounded by at most u = eps / 2 of itself.
"""
import numpy as np
import pytest
import torch

import paper_2604_18529_b200 as pkg
from paper_2604_18529_b200 import binding as hg
from test_tree_gpu import BF16, DEV, F16, ints

pytestmark = pytest.mark.gpu


def pool_desc(table, P, num_pages, Hq=8, Hkv=2, D=64, dtype=F16, status=None, k=None):
    ps, hs, ts = (Hkv * P * D, P * D, D) if k is None else (k.stride(0), k.stride(1), k.stride(2))
    return hg.attn_desc(batch=1 if table is None else table.shape[0], num_q_heads=Hq, num_kv_heads=Hkv, head_dim=D, dtype=dtype, page_size=P,
                        num_pages=num_pages, page_stride=ps, head_stride=hs, tok_stride=ts, block_table=table,
                        max_pages=num_pages if table is None else table.shape[1], chunk_tokens=max(P, 128), num_chunks=1, status=status)


# ---- slots ----------------------------------------------------------------------------------------------------------------

def slots_plain(lens, n_new, parent, N, table, P, num_pages, words):
    """Row by row, on lists"""
    cut = 1 << 31 if parent is None and not words else min(1024, 32 * words if words else 1024)
    seq, pos, slot, mask, cu, status = [], [], [], [], [0], 0
    for b, n in enumerate(n_new):
        asked, n = max(n, 0), min(max(n, 0), cut)
        n = min(n, N - len(seq))
        if n < asked:
            status |= hg.HG_DEV_RANGE
        first, sees = len(seq), []
        for i in range(n):
            p = i - 1 if parent is None else parent[first + i]
            if p >= i:
                p, status = -1, status | hg.HG_DEV_RANGE
            sees.append(([] if p < 0 else sees[p]) + [i])
            t = max(lens[b], 0) + i
            e = -1
            if t // P >= len(table[b]):
                status |= hg.HG_DEV_RANGE
            else:
                e = table[b][t // P]
                if not 0 <= e < num_pages:
                    e, status = -1, status | hg.HG_DEV_BAD_PAGE
            seq.append(b)
            pos.append(max(lens[b], 0) + len(sees[i]) - 1)
            slot.append(-1 if e < 0 else e * P + t % P)
            row = [0] * words
            for j in sees[i]:
                if words:
                    row[j // 32] |= 1 << j % 32
            mask.append([w - (1 << 32) if w >> 31 else w for w in row])
        cu.append(len(seq))
    rest = N - len(seq)
    return cu, seq + [-1] * rest, pos + [0] * rest, slot + [-1] * rest, mask + [[0] * words] * rest, status


def slots_check(lens, n_new, N, P=16, parent=None, words=0, spare=2, holes=(), one_each=False, seed=0):
    r = np.random.RandomState(seed)
    n = [1] * len(lens) if one_each else n_new
    S = max([-(-(max(t, 0) + max(k, 0)) // P) for t, k in zip(lens, n)] + [1])
    num_pages = len(lens) * S + spare
    table = r.permutation(num_pages)[:len(lens) * S].reshape(len(lens), S).astype(np.int32)
    for b, s, e in holes:
        table[b, s] = e
    dev_table, status = torch.from_numpy(table).to(DEV), ints([0])
    want = slots_plain(lens, n, parent, N, table.tolist(), P, num_pages, words)
    B = len(lens)
    cu, seq, pos = [torch.full((m,), 99, dtype=torch.int32, device=DEV) for m in (B + 1, N, N)]
    slot = torch.full((N,), 99, dtype=torch.int64, device=DEV)
    mask = torch.full((N, words), 99, dtype=torch.int32, device=DEV) if words else None
    par = None if parent is None else ints((list(parent) + [-1] * N)[:N])
    hg.hg_kv_slots(ints(lens), None if one_each else ints(n_new), par, cu, seq, pos, slot, mask, pool_desc(dev_table, P, num_pages, status=status))
    torch.cuda.synchronize()
    got = [x.tolist() for x in (cu, seq, pos, slot)] + [mask.tolist() if words else [[]] * N, int(status)]
    for name, a, b in zip(("cu", "seq", "pos", "slot", "mask", "status"), got, want):
        assert a == list(b) if isinstance(a, list) else a == b, name
    return got


def random_parents(n_new, r):
    return [int(r.randint(-1, i)) if i else -1 for n in n_new for i in range(max(n, 0))]


@pytest.mark.parametrize("P", [16, 64, 256])
def test_slots_of_prompts(P):
    slots_check([0, 100, 7, 0, 31], [1000, 1, 0, 16, 700], 1717, P)
    slots_check([0, 100, 7, 0, 31], [1000, 1, 0, 16, 700], 1800, P)


def test_slots_of_single_tokens():
    slots_check([5, 0, 1000, 16, 15], None, 5, one_each=True)
    slots_check([5, 0, 1000, 16, 15], None, 9, one_each=True, words=1)
    slots_check([3], [1], 1)
    slots_check([0, 0, 0], [0, -4, 0], 3)


@pytest.mark.parametrize("sizes", [[1], [2, 31, 32, 33, 0, 64, 65, 1], [300, 5, 1024], [40] * 70])
def test_slots_of_trees_and_chains(sizes):
    r = np.random.RandomState(len(sizes))
    lens = [int(x) for x in r.randint(0, 500, len(sizes))]
    words = -(-max(sizes) // 32)
    slots_check(lens, sizes, sum(sizes) + 5, parent=random_parents(sizes, r), words=words)
    slots_check(lens, sizes, sum(sizes) + 5, words=words)
    slots_check(lens, sizes, sum(sizes), parent=random_parents(sizes, r))
    slots_check(lens, sizes, sum(sizes), parent=[i - 1 for n in sizes for i in range(n)], words=words)     # the longest way up


def test_slots_of_many_sequences():
    r = np.random.RandomState(1)
    n = [int(x) for x in r.randint(0, 7, 3000)]
    slots_check([int(x) for x in r.randint(0, 90, 3000)], n, sum(n) + 3)
    slots_check([int(x) for x in r.randint(0, 90, 1300)], n[:1300], sum(n[:1300]), words=1, parent=random_parents(n[:1300], r))


def test_slots_are_cut_where_they_do_not_fit():
    assert slots_check([10, 20, 30], [5, 6, 7], 9)[5] == hg.HG_DEV_RANGE                       # fewer rows
    assert slots_check([10, 20], [40, 6], 60, words=1)[5] == hg.HG_DEV_RANGE                   # more tokens than bits
    assert slots_check([10], [1030], 1100, parent=list(range(-1, 1029)))[5] == hg.HG_DEV_RANGE
    assert slots_check([10, 20], [5, 6], 20, holes=[(1, 1, -1)])[5] == hg.HG_DEV_BAD_PAGE
    assert slots_check([10, 20], [5, 6], 20, holes=[(0, 0, 10 ** 6)])[5] == hg.HG_DEV_BAD_PAGE
    assert slots_check([-3, 20], [5, 6], 20)[5] == 0
    assert slots_check([10, 20], [4, 3], 7, parent=[-1, 5, 0, 3, -7, 0, 2], words=1)[5] == hg.HG_DEV_RANGE


def test_slots_past_the_end_of_the_table():
    table, status = ints([[3, 1]]), ints([0])
    cu, seq, pos = ints([0, 0]), ints([0] * 8), ints([0] * 8)
    slot = ints([0] * 8, torch.int64)
    hg.hg_kv_slots(ints([28]), ints([8]), None, cu, seq, pos, slot, None, pool_desc(table, 16, 4, status=status))
    assert slot.tolist() == [28, 29, 30, 31, -1, -1, -1, -1] and int(status) == hg.HG_DEV_RANGE and cu.tolist() == [0, 8]
    hg.hg_kv_slots(ints([2 ** 31 - 4]), ints([8]), None, cu, seq, pos, slot, None, pool_desc(table, 16, 4, status=status))
    assert slot.tolist() == [-1] * 8


def ready_plain(lens, n_new, n_ready, parent, N, table, P, num_pages, words):
    """Row by row: packed by n_new, tokens without a place among them"""
    limit = 1 << 31 if parent is None and not words else min(1024, 32 * words if words else 1024)
    rows, cu, status = [], [0], 0
    for b, n in enumerate(n_new):
        first, L, sees = len(rows), max(lens[b], 0), []
        if max(n, 0) > limit:
            status |= hg.HG_DEV_RANGE
        for i in range(max(n, 0)):
            if len(rows) == N:
                status |= hg.HG_DEV_RANGE
                break
            if i >= min(n_ready[b], limit):
                rows.append((b, L, -1, [0] * words))
                continue
            p = i - 1 if parent is None else parent[first + i]
            sees.append(([] if p < 0 else sees[p]) + [i])
            e, t = -1, L + i
            if t // P >= len(table[b]):
                status |= hg.HG_DEV_RANGE
            else:
                e = table[b][t // P]
            word = [sum(1 << j % 32 for j in sees[i] if j // 32 == w) for w in range(words)]
            rows.append((b, L + len(sees[i]) - 1, -1 if e < 0 else e * P + t % P, [w - (1 << 32) if w >> 31 else w for w in word]))
        cu.append(len(rows))
    rows += [(-1, 0, -1, [0] * words)] * (N - len(rows))
    return [cu] + [list(x) for x in zip(*rows)] + [status]


@pytest.mark.parametrize("n_new,n_ready,words,N", [
    ([5, 9, 3, 0, 7], [5, 4, 3, 0, 7], 1, 30), ([5, 9, 3, 0, 7], [0, 9, -2, 5, 3], 1, 24), ([5, 9, 3, 0, 7], [5, 9, 2, 0, 100], 1, 20),
    ([40, 6, 33, 2], [40, 6, 33, 2], 1, 90), ([40, 6, 70, 2], [36, 6, 10, 0], 2, 118), ([1100, 8, 1030], [1100, 7, 1026], 32, 2200),
    ([600, 1, 0, 900], [17, 1, 0, 899], 0, 1502), ([3] * 2500, [3, 1, 0, 2, 3] * 500, 1, 7510), ([50] + [2] * 2400, [50] + [1, 2] * 1200, 1, 4850)])
@pytest.mark.parametrize("trees", [False, True])
def test_slots_of_tokens_that_got_no_page(n_new, n_ready, words, N, trees):
    """No row moves: with a mask and parents, without either (four rows a thread), in batches over and under 2048, and behind a
    sequence with more tokens than mask bits"""
    r = np.random.RandomState(len(n_new))
    P, B, lens = 16, len(n_new), [int(x) for x in r.randint(0, 90, len(n_new))]
    parent = random_parents(n_new, r) if trees else None
    S = max(-(-(t + n) // P) for t, n in zip(lens, n_new))
    num_pages = B * S + 1
    table = r.permutation(num_pages)[:B * S].reshape(B, S).astype(np.int32)
    cu, seq, pos = [torch.full((m,), 99, dtype=torch.int32, device=DEV) for m in (B + 1, N, N)]
    slot, status = torch.full((N,), 99, dtype=torch.int64, device=DEV), ints([0])
    mask = torch.full((N, words), 99, dtype=torch.int32, device=DEV) if words else None
    par = ints((parent + [-1] * N)[:max(N, len(parent))]) if trees else None
    hg.hg_kv_slots(ints(lens), ints(n_new), par, cu, seq, pos, slot, mask, pool_desc(torch.from_numpy(table).to(DEV), P, num_pages, status=status),
                   n_ready=ints(n_ready))
    torch.cuda.synchronize()
    want = ready_plain(lens, n_new, n_ready, parent, N, table.tolist(), P, num_pages, words)
    got = [x.tolist() for x in (cu, seq, pos, slot)] + [mask.tolist() if words else [[]] * N, int(status)]
    for name, a, b in zip(("cu", "seq", "pos", "slot", "mask", "status"), got, want):
        assert a == b, name


def test_ready_counts_of_all_tokens_change_nothing():
    lens, n = [5, 0, 31, 16], [7, 0, 20, 32]
    r = np.random.RandomState(0)
    parent, table = ints(random_parents(n, r) + [-1] * 3), ints(r.permutation(16).reshape(4, 4).tolist())
    results = []
    for ready in (None, ints(n), ints([99] * 4)):
        cu, seq, pos = ints([0] * 5), ints([0] * 62), ints([0] * 62)
        slot, mask = ints([0] * 62, torch.int64), torch.zeros((62, 1), dtype=torch.int32, device=DEV)
        pkg.prepare_kv_slots(ints(lens), ints(n), parent, cu, seq, pos, slot, mask, pool_desc(table, 16, 16), n_ready=ready)()
        torch.cuda.synchronize()
        results.append((cu, seq, pos, slot, mask))
    for other in results[1:]:
        for a, b in zip(results[0], other):
            assert torch.equal(a, b)


def test_slots_with_identity_paging_and_without_outputs():
    cu, slot = ints([0] * 3), ints([0] * 5, torch.int64)
    desc = hg.attn_desc(batch=2, num_q_heads=1, num_kv_heads=1, head_dim=64, dtype=F16, page_size=16, num_pages=8, page_stride=1024, head_stride=1024,
                        tok_stride=64, block_table=None, max_pages=4, chunk_tokens=128, num_chunks=1)
    hg.hg_kv_slots(ints([3, 15]), ints([2, 3]), None, cu, None, None, slot, None, desc)
    assert cu.tolist() == [0, 2, 5] and slot.tolist() == [3, 4, 64 + 15, 64 + 16, 64 + 17]
    hg.hg_kv_slots(ints([3, 15]), ints([2, 3]), None, cu, None, None, None, None, desc, num_rows=4)
    assert cu.tolist() == [0, 2, 4]
    with pytest.raises(ValueError):
        hg.hg_kv_slots(ints([3, 15]), ints([2, 3]), None, cu, None, None, None, None, desc)


def test_slots_beyond_31_bits():
    """2^24 pages of 256 tokens: a place past 2^31"""
    table = ints([[(1 << 24) - 1]])
    slot = ints([0] * 2, torch.int64)
    hg.hg_kv_slots(ints([7]), ints([2]), None, ints([0, 0]), None, None, slot, None, pool_desc(table, 256, 1 << 24))
    assert slot.tolist() == [((1 << 24) - 1) * 256 + 7, ((1 << 24) - 1) * 256 + 8]


# ---- rotary positions --------------------------------------------------------------------------------------------------------

def turned64(x, pos, freq, rot, layout, magnitude=1.0, sign=1.0):
    """Pairs as complex numbers in 64 bits"""
    x = x.double().clone()
    z = torch.polar(torch.full((x.shape[0], rot // 2), magnitude, dtype=torch.float64, device=x.device), sign * pos.double()[:, None] * freq[:rot // 2])
    i = torch.arange(rot // 2, device=x.device)
    a, b = (i, i + rot // 2) if layout == "half" else (2 * i, 2 * i + 1)
    y = torch.complex(x[..., a], x[..., b]) * z[:, None]
    x[..., a], x[..., b] = y.real, y.imag
    return x


def near(got, want, x, magnitude=1.0):
    u = torch.finfo(got.dtype).eps / 2
    return bool(((got.double() - want).abs() <= u * want.abs() + 2.0 ** -20 * magnitude * x.abs().max().double() + 2.0 ** -25).all())


def freqs(rot, theta=10000.0, **kw):
    f, m = pkg.hg_rope_frequencies(rot, theta, **kw)
    return f.to(DEV), m


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("D,rot", [(64, 64), (64, 16), (64, 48), (128, 128), (128, 64), (128, 96), (128, 112)])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_rope_and_append(layout, D, rot, dtype):
    g = torch.Generator(device=DEV)
    g.manual_seed(rot)
    for N, Hq, Hkv, P, nhd, fused in ((1, 8, 2, 16, False, False), (37, 7, 7, 32, True, True), (600, 12, 4, 64, False, True)):
        rows = torch.randn((N, Hq + 2 * Hkv, D), generator=g, device=DEV).to(dtype)
        q, k, v = rows.split([Hq, Hkv, Hkv], 1)
        if not fused:
            q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
        num_pages = -(-N // P) + 2
        kc, vc = [torch.zeros((num_pages, P, Hkv, D) if nhd else (num_pages, Hkv, P, D), dtype=dtype, device=DEV) for _ in range(2)]
        if nhd:
            kc, vc = kc.transpose(1, 2), vc.transpose(1, 2)
        r = np.random.RandomState(N)
        slot = torch.from_numpy(r.permutation(num_pages * P)[:N].astype(np.int64)).to(DEV)
        slot[N // 2:N // 2 + N // 10] = -1                                  # rows that have no place
        pos = torch.from_numpy(r.randint(0, 1 << 20, N).astype(np.int32)).to(DEV)
        freq, mag = freqs(rot, 500000.0, scale="index", factor=4.0, context=8192)
        status, out = ints([0]), torch.full((N + 1, Hq, D), -77.0, dtype=dtype, device=DEV)
        desc = pool_desc(None, P, num_pages, Hq, Hkv, D, dtype, status, kc)
        rope = hg.rope_desc(rot_dim=rot, freq=freq, layout=layout, magnitude=mag)
        hg.hg_kv_append_rope(q, k, v, pos, slot, out[:N], kc, vc, desc, rope)
        torch.cuda.synchronize()
        assert int(status) == 0 and (out[N] == -77).all()
        assert near(out[:N], turned64(q, pos, freq, rot, layout, mag), q, mag)
        assert torch.equal(out[:N, :, rot:], q[..., rot:])
        have = slot >= 0
        want = torch.zeros((num_pages, P, Hkv, D), dtype=torch.float64, device=DEV)
        want.view(-1, Hkv, D)[slot[have]] = turned64(k, pos, freq, rot, layout, mag)[have]
        assert near(kc.transpose(1, 2), want, k, mag)
        want = torch.zeros((num_pages, P, Hkv, D), dtype=dtype, device=DEV)
        want.view(-1, Hkv, D)[slot[have]] = v[have]
        assert torch.equal(vc.transpose(1, 2), want)
        if not fused:                                                      # in place, and without queries
            before, kc0 = out[:N].clone(), kc.clone()
            hg.hg_kv_append_rope(q, k, v, pos, slot, q, kc.zero_(), vc, desc, rope)
            assert torch.equal(q, before) and torch.equal(kc, kc0)
            hg.hg_kv_append_rope(None, k, v, pos, slot, None, kc.zero_(), vc, desc, rope)
            assert torch.equal(kc, kc0)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rope_alone_and_its_gradient(layout):
    """The gradient of sum(w * rope(x)) is the inverse rotation of w: against the formula, and against differences"""
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    N, H, D, rot = 50, 6, 64, 32
    freq, _ = freqs(rot)
    pos = torch.randint(0, 3000, (N,), generator=g, device=DEV, dtype=torch.int32)
    x, w = [torch.randn((N, H, D), generator=g, device=DEV).half() for _ in range(2)]
    y, grad, back = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    hg.hg_rope(x, y, pos, hg.rope_desc(rot_dim=rot, freq=freq, layout=layout, magnitude=1.25))
    hg.hg_rope(w, grad, pos, hg.rope_desc(rot_dim=rot, freq=freq, layout=layout, magnitude=1.25, inverse=True))
    torch.cuda.synchronize()
    assert near(y, turned64(x, pos, freq, rot, layout, 1.25), x, 1.25)
    assert near(grad, turned64(w, pos, freq, rot, layout, 1.25, -1.0), w, 1.25)
    leaf = x.double().requires_grad_()
    (turned64_grad(leaf, pos, freq, rot, layout, 1.25) * w.double()).sum().backward()
    assert near(grad, leaf.grad, w, 1.25)
    # differences: the map is linear, so a step of 1 in one component gives the derivative; each of the two outputs per
    # component is rounded by at most eps / 2 of itself
    u = torch.finfo(F16).eps / 2
    for c in (0, 1, 15, 16, 31, 32, 63):
        x2 = x.clone()
        x2[..., c] += 1
        step = (x2[..., c].double() - x[..., c].double())[..., None]
        y2 = torch.empty_like(x)
        hg.hg_rope(x2, y2, pos, hg.rope_desc(rot_dim=rot, freq=freq, layout=layout, magnitude=1.25))
        d = ((y2.double() - y.double()) * w.double()).sum(2) / step[..., 0]
        tol = (u * (y2.double().abs() + y.double().abs()) * w.double().abs()).sum(2) / step[..., 0].abs() + u * grad[..., c].double().abs() + 2e-5 * D
        assert ((d - grad[..., c].double()).abs() <= tol).all()
    hg.hg_rope(y, back, pos, hg.rope_desc(rot_dim=rot, freq=freq, layout=layout, magnitude=0.8, inverse=True))
    m = x.abs().max().double()
    assert ((back - x).double().abs() <= u * x.double().abs() + 2 * u * 1.25 * 1.5 * m * 0.8 + 2.0 ** -19 * m).all()


def turned64_grad(x, pos, freq, rot, layout, magnitude):
    angle = pos.double()[:, None] * freq
    c, s = magnitude * angle.cos()[:, None], magnitude * angle.sin()[:, None]
    i = torch.arange(rot // 2, device=x.device)
    a, b = (i, i + rot // 2) if layout == "half" else (2 * i, 2 * i + 1)
    y = torch.zeros_like(x)
    y = y.index_add(2, a, x[..., a] * c - x[..., b] * s).index_add(2, b, x[..., b] * c + x[..., a] * s)
    rest = torch.arange(rot, x.shape[2], device=x.device)
    return y.index_add(2, rest, x[..., rest])


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_parts_of_a_fused_projection_in_place_and_beside(layout):
    """Rows of equal strides that lie between one another are no overlap"""
    N, Hq, Hkv, D, P = 40, 6, 2, 64, 16
    rows = torch.randn((N, 2 * Hq + 2 * Hkv, D), device=DEV).half()
    q, k, v, other = rows.split([Hq, Hkv, Hkv, Hq], 1)
    freq, _ = freqs(D)
    pos, slot = torch.arange(N, device=DEV, dtype=torch.int32), torch.arange(N, device=DEV)
    want, keys = turned64(q, pos, freq, D, layout), turned64(k, pos, freq, D, layout)
    kc, vc = torch.zeros((2, 3, Hkv, P, D), device=DEV).half()
    desc, rope = pool_desc(None, P, 3, Hq, Hkv, D, F16, None, kc), hg.rope_desc(rot_dim=D, freq=freq, layout=layout)
    before = rows.clone()
    hg.hg_rope(q, other, pos, rope)
    torch.cuda.synchronize()
    assert near(other, want, q) and torch.equal(rows[:, :Hq + 2 * Hkv], before[:, :Hq + 2 * Hkv])
    hg.hg_kv_append_rope(q, k, v, pos, slot, q, kc, vc, desc, rope)
    torch.cuda.synchronize()
    assert torch.equal(q, other) and torch.equal(rows[:, Hq:Hq + 2 * Hkv], before[:, Hq:Hq + 2 * Hkv])
    assert near(kc.transpose(1, 2).reshape(-1, Hkv, D)[:N], keys, k) and torch.equal(vc.transpose(1, 2).reshape(-1, Hkv, D)[:N], v)


def test_far_and_negative_positions():
    freq, _ = freqs(128)
    pos = ints([0, -5, 2 ** 31 - 1, -2 ** 31, 10 ** 9, 1])
    x = torch.randn((6, 4, 128), device=DEV).to(BF16)
    y = torch.empty_like(x)
    for layout in ("half", "interleaved"):
        hg.hg_rope(x, y, pos, hg.rope_desc(rot_dim=128, freq=freq, layout=layout))
        # at 2^31 positions a frequency's own rounding (2^-53) is 2.4e-7 of a radian, here as in the 64-bit form: 2^-20 covers it
        assert near(y, turned64(x, pos, freq, 128, layout), x)
    assert torch.equal(y[0], x[0])


def test_places_outside_the_pool_are_refused():
    N, D, Hkv, P = 4, 64, 2, 16
    k, v, q = torch.randn((3, N, Hkv, D), device=DEV).half()
    kc, vc = torch.zeros((2, 3, Hkv, P, D), device=DEV).half()
    status, freq = ints([0]), freqs(D)[0]
    desc = pool_desc(None, P, 3, Hkv, Hkv, D, F16, status)
    hg.hg_kv_append_rope(q, k, v, ints([0] * N), ints([0, 48, -1, 1 << 40], torch.int64), q, kc, vc, desc, hg.rope_desc(rot_dim=D, freq=freq))
    torch.cuda.synchronize()
    assert int(status) == hg.HG_DEV_BAD_PAGE
    assert torch.equal(vc[0, :, 0], v[0]) and int((vc != 0).sum()) == int((v[0] != 0).sum())


# ---- accepted paths --------------------------------------------------------------------------------------------------------

def accept_setup(lens, nodes, Hkv=3, D=64, P=16, dtype=F16, nhd=False, seed=0):
    r = np.random.RandomState(seed)
    S = max(-(-(max(t, 0) + nodes) // P) for t in lens)
    num_pages = len(lens) * S + 2
    table = torch.from_numpy(r.permutation(num_pages)[:len(lens) * S].reshape(len(lens), S).astype(np.int32)).to(DEV)
    k, v = torch.randn((2, num_pages, P, Hkv, D) if nhd else (2, num_pages, Hkv, P, D), device=DEV).to(dtype)
    if nhd:
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    return table, k, v, ints([0]), num_pages


def accept_plain(pool, table, lens, paths, P):
    y = pool.clone()
    for b, path in enumerate(paths):
        for j, x in enumerate(path):
            a, c = max(lens[b], 0) + x, max(lens[b], 0) + j
            y[int(table[b, c // P]), :, c % P] = y[int(table[b, a // P]), :, a % P].clone()
    return y


@pytest.mark.parametrize("Hkv,D,P,nhd,dtype", [(3, 64, 16, False, F16), (40, 128, 64, False, BF16), (8, 128, 16, True, F16), (1, 64, 256, False, F16)])
def test_accept(Hkv, D, P, nhd, dtype):
    r = np.random.RandomState(Hkv)
    lens, nodes = [0, 15, 16, 100, 7, 31], 70
    paths = [[], [0], [3], list(range(20)), sorted(r.permutation(70)[:33].tolist()), [0, 1, 2, 40, 69]]
    table, k, v, status, n = accept_setup(lens, nodes, Hkv, D, P, dtype, nhd)
    most = max(map(len, paths)) + 2
    path = ints([p + [-9] * (most - len(p)) for p in paths])
    want = [accept_plain(x, table, lens, paths, P) for x in (k, v)]
    seq_lens, new = ints(lens), ints([0] * 6)
    desc = pool_desc(table, P, n, Hkv, Hkv, D, dtype, status, k)
    kc, vc = k.clone(), v.clone()                                            # (keeps the strides)
    hg.hg_kv_accept(path, ints(list(map(len, paths))), seq_lens, new, kc, vc, desc)
    torch.cuda.synchronize()
    assert torch.equal(kc, want[0]) and torch.equal(vc, want[1]) and int(status) == 0
    assert new.tolist() == [t + len(p) for t, p in zip(lens, paths)] and seq_lens.tolist() == lens
    kc, vc = k.clone(), v.clone()
    hg.hg_kv_accept(path, ints(list(map(len, paths))), seq_lens, None, kc, vc, desc)           # one layer, then the last
    assert torch.equal(kc, want[0]) and seq_lens.tolist() == lens
    kc, vc = k.clone(), v.clone()
    hg.hg_kv_accept(path, ints(list(map(len, paths))), seq_lens, seq_lens, kc, vc, desc)
    assert torch.equal(kc, want[0]) and torch.equal(vc, want[1]) and seq_lens.tolist() == new.tolist()


def test_accept_stops_at_what_is_wrong():
    lens, nodes, P = [10, 10, 10, 10, 10, 10, -4], 40, 16
    table, k, v, status, n = accept_setup(lens, nodes)
    table[2, 1] = -1                                                         # positions 16 .. 31
    asked = [[0, 2, 2, 3], [1, 5, 3, 7], [1, 3, 8, 30], [-1, 2, 3, 4], [4, 6, 70, 71], [5, 6, 7, 8], [1, 2, 3, 4]]
    kept = [[0, 2], [1, 5], [1, 3], [], [4, 6], [5, 6, 7], [1, 2, 3, 4]]
    counts = [4, 4, 4, 4, 4, 3, 9]
    new = ints([0] * 7)
    want = accept_plain(k, table, lens, kept, P)
    hg.hg_kv_accept(ints(asked), ints(counts), ints(lens), new, k, v, pool_desc(table, P, n, 3, 3, 64, F16, status))
    torch.cuda.synchronize()
    assert torch.equal(k, want) and new.tolist() == [max(t, 0) + len(p) for t, p in zip(lens, kept)]
    assert int(status) == hg.HG_DEV_RANGE | hg.HG_DEV_BAD_PAGE
    status.zero_()
    hg.hg_kv_accept(ints([[3, 1]] * 7), ints([1] * 6 + [-3]), ints(lens), new, k, v, pool_desc(table, P, n, 3, 3, 64, F16, status))
    assert int(status) == 0 and new.tolist() == [11] * 6 + [0]               # what lies behind the accepted part is not looked at


# ---- a step as a decode loop makes it ---------------------------------------------------------------------------------------

def test_steps_of_speculative_decoding():
    """reserve -> slots -> append with rotary positions -> tree attention -> accept, three steps of two layers in captured
    graphs, against a model that keeps every sequence's keys and values in lists and computes in 64 bits."""
    B, Hq, Hkv, D, P, layers, S, pages = 5, 8, 2, 64, 16, 2, 12, 64
    G, T, rot = Hq // Hkv, 9, 32
    r = np.random.RandomState(0)
    freq, mag = freqs(rot, 10000.0, scale="turns", factor=2.0, low=1.0, high=4.0, context=64)
    rope = hg.rope_desc(rot_dim=rot, freq=freq, magnitude=mag)
    status, table, ref = ints([0]), torch.full((B, S), -1, dtype=torch.int32, device=DEV), ints([0] * pages)
    pools = [torch.zeros((2, pages, Hkv, P, D), device=DEV).half() for _ in range(layers)]
    desc = pool_desc(table, P, pages, Hq, Hkv, D, F16, status)
    lens = ints([0] * B)
    N = B * T + 2
    n_new, parent = ints([0] * B), ints([-1] * N)
    cu, seq, pos, slot, mask = ints([0] * (B + 1)), ints([0] * N), ints([0] * N), ints([0] * N, torch.int64), torch.zeros((N, 1), dtype=torch.int32, device=DEV)
    copies = [ints([-1] * B) for _ in range(3)]
    ready, path, n_accept = ints([0] * B), ints([[0] * T] * B), ints([0] * B)
    rows = [torch.zeros((N, Hq + 2 * Hkv, D), device=DEV).half() for _ in range(layers)]
    q_out = [torch.zeros((N, Hq, D), device=DEV).half() for _ in range(layers)]
    outs, lses = [torch.zeros_like(x) for x in q_out], [torch.zeros((N, Hq), device=DEV) for _ in range(layers)]
    tree = hg.tree_desc(cu_nodes=cu, mask=mask, num_rows=N, max_nodes=T)
    ws = torch.empty(hg.hg_attn_tree_workspace_bytes(desc, tree), dtype=torch.uint8, device=DEV)

    def forward():
        hg.hg_kv_reserve(lens, n_new, ref, *copies, ready, desc)
        hg.hg_kv_slots(lens, ready, parent, cu, seq, pos, slot, mask, desc)
        for x in range(layers):
            q, k, v = rows[x].split([Hq, Hkv, Hkv], 1)
            hg.hg_kv_append_rope(q, k, v, pos, slot, q_out[x], pools[x][0], pools[x][1], desc, rope)
            hg.hg_attn_decode_tree(q_out[x], pools[x][0], pools[x][1], lens, None, [], outs[x], lses[x], ws, desc, tree)

    def accept():
        for x in range(layers):
            hg.hg_kv_accept(path, n_accept, lens, lens if x == layers - 1 else None, pools[x][0], pools[x][1], desc)

    graphs = []
    for f in (forward, accept):                                              # (nothing new, nothing accepted)
        f()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            f()
        graphs.append(g)
    cached = [[[] for _ in range(B)] for _ in range(layers)]                  # (position, key turned in 64 bits, value)
    for step in range(3):
        n = [int(r.randint(0, T + 1)) for _ in range(B)]
        n[0], n[1] = 1, T
        par = [p for m in n for p in ([-1] + [int(r.randint(-1, i)) for i in range(1, m)])[:m]]
        if step == 0:
            par = [i - 1 for m in n for i in range(m)]                       # the prompts: chains
        n_new.copy_(ints(n))
        parent.copy_(ints(par + [-1] * (N - len(par))))
        for x in rows:
            x.copy_(torch.randn(x.shape, device=DEV))
        graphs[0].replay()
        torch.cuda.synchronize()
        assert int(status) == 0 and cu.tolist() == np.concatenate([[0], np.cumsum(n)]).tolist()
        at, chosen = 0, []
        for b in range(B):
            sees = []
            for i in range(n[b]):
                p = par[at + i]
                sees.append((sees[p] if p >= 0 else []) + [i])
            best = max(sees, key=len) if sees else []
            chosen.append(best)
            for x in range(layers):
                q, k, v = rows[x][at:at + n[b]].split([Hq, Hkv, Hkv], 1)
                L = len(cached[x][b])
                where = torch.tensor([L + len(a) - 1 for a in sees], device=DEV)
                if not n[b]:
                    continue
                qr, kr = turned64(q, where, freq, rot, "half", mag), turned64(k, where, freq, rot, "half", mag)
                for i in range(n[b]):
                    ks = torch.stack([c[0] for c in cached[x][b]] + [kr[j] for j in sees[i]])        # [t][Hkv][D]
                    vs = torch.stack([c[1] for c in cached[x][b]] + [v[j].double() for j in sees[i]])
                    s = torch.einsum("hgd,thd->hgt", qr[i].reshape(Hkv, G, D), ks) * D ** -0.5
                    o = torch.einsum("hgt,thd->hgd", torch.softmax(s, 2), vs).reshape(Hq, D)
                    # turned queries and keys are rounded to fp16: a product of D = 64 pairs of size about 1, each off by 2 * 2^-11 of
                    # itself at most and with either sign, over sqrt(D): sqrt(64) * 2^-10 / 8 * 4 (four deviations) = 4e-3 of a logit, and
                    # larger components than 1 double that: 1e-2; weights and values follow, and the roundings of P and out are far below
                    assert float((lses[x][at + i].double() - torch.logsumexp(s, 2).reshape(Hq)).abs().max()) < 1e-2
                    assert float((outs[x][at + i].double() - o).abs().max()) < 2e-2 * float(vs.abs().max())
                for j in best:
                    cached[x][b].append((kr[j], v[j].double()))
            at += n[b]
        path.copy_(ints([c + [0] * (T - len(c)) for c in chosen]))
        n_accept.copy_(ints([len(c) for c in chosen]))
        graphs[1].replay()
        torch.cuda.synchronize()
        assert lens.tolist() == [len(c) for c in cached[0]] and int(status) == 0
    for x in range(layers):
        for b in range(B):
            for t, (kk, vv) in enumerate(cached[x][b]):
                page = int(table[b, t // P])
                assert torch.equal(pools[x][1][page, :, t % P].double(), vv)
                assert near(pools[x][0][page, :, t % P], kk, kk.abs().max() * 1.5)


@pytest.mark.parametrize("trees", [True, False])
def test_a_step_whose_pool_runs_out_of_pages(trees):
    """The second of three sequences gets one page of the three that it asked for, the third one of its own none, beside one that it
    shares.  Every token that got a place has the result of the same step in a large pool, bit for bit, its keys and values
    lie where they belong, and no other page changes."""
    Hq, Hkv, D, P, S = 8, 2, 64, 16, 8
    lens, n = [20, 16, 9], [5, 40, 10]
    r = np.random.RandomState(2)
    par = random_parents(n, r) if trees else [i - 1 for m in n for i in range(m)]
    N, cu_want = sum(n) + 2, [0, 5, 45, 55]
    rows = torch.randn((N, Hq + 2 * Hkv, D), device=DEV).half()
    history = torch.randn((2, 3, Hkv, 32, D), device=DEV).half()
    freq, _ = freqs(D)
    rope = hg.rope_desc(rot_dim=D, freq=freq)
    outs = []
    for pages in (20, 6):
        # pages 0 .. 4 hold the caches; sequence 2's only page is held by somebody else too
        table = torch.full((3, S), -1, dtype=torch.int32, device=DEV)
        table[0, :2], table[1, 0], table[2, 0] = ints([4, 1]), 3, 0
        ref = ints([2, 1, 1, 1, 1] + [0] * (pages - 5))
        pool = torch.full((2, pages, Hkv, P, D), 7.0, device=DEV).half()
        for b, L in enumerate(lens):
            for t in range(L):
                pool[:, int(table[b, t // P]), :, t % P] = history[:, b, :, t]
        before, status = pool.clone(), ints([0])
        desc = pool_desc(table, P, pages, Hq, Hkv, D, F16, status)
        seq_lens, n_new = ints(lens), ints(n)
        copies, ready = [ints([-1] * 3) for _ in range(3)], ints([0] * 3)
        cu, seq, pos = ints([0] * 4), ints([0] * N), ints([0] * N)
        slot, mask = ints([0] * N, torch.int64), torch.zeros((N, 2), dtype=torch.int32, device=DEV)
        parent = ints(par + [-1] * 2) if trees else None
        hg.hg_kv_reserve(seq_lens, n_new, ref, *copies, ready, desc)
        hg.hg_kv_copy_pages(copies[0], copies[1], copies[2], None, pool[0], pool[1], desc)
        torch.cuda.synchronize()
        counts, short = ready.tolist(), pages == 6
        assert counts == ([5, 16, 0] if short else n) and bool(int(status) & hg.HG_DEV_NO_PAGE) == short
        hg.hg_kv_slots(seq_lens, n_new, parent, cu, seq, pos, slot, mask if trees else None, desc, n_ready=ready)
        q, k, v = rows.split([Hq, Hkv, Hkv], 1)
        turned, out, lse = [torch.zeros((N, Hq, D), device=DEV).half() for _ in range(2)] + [torch.zeros((N, Hq), device=DEV)]
        tree = hg.tree_desc(cu_nodes=cu, mask=mask if trees else None, num_rows=N, max_nodes=40)
        ws = torch.empty(hg.hg_attn_tree_workspace_bytes(desc, tree), dtype=torch.uint8, device=DEV)
        hg.hg_kv_append_rope(q, k, v, pos, slot, turned, pool[0], pool[1], desc, rope)
        hg.hg_attn_decode_tree(turned, pool[0], pool[1], seq_lens, None, [], out, lse, ws, desc, tree)
        torch.cuda.synchronize()
        assert cu.tolist() == cu_want and int(status) & hg.HG_DEV_RANGE == 0
        placed = [cu_want[b] + i for b in range(3) for i in range(counts[b])]
        assert [x for x in range(N) if int(slot[x]) >= 0] == placed
        changed = torch.zeros(pages, P, dtype=torch.bool)
        for b in range(3):
            for i in range(counts[b]):
                page, row = int(table[b, (lens[b] + i) // P]), (lens[b] + i) % P
                changed[page, row] = True
                assert torch.equal(pool[1][page, :, row], v[cu_want[b] + i])
        if short:
            same = ~changed.to(DEV)
            assert torch.equal(pool.transpose(2, 3)[:, same], before.transpose(2, 3)[:, same])
        # a chain of accepted tokens where that is possible: nothing but what was placed
        path = ints([list(range(40))] * 3)
        hg.hg_kv_accept(path, torch.minimum(ready, ints([3, 30, 2])), seq_lens, seq_lens, pool[0], pool[1], desc)
        torch.cuda.synchronize()
        assert seq_lens.tolist() == [a + min(c, m) for a, c, m in zip(lens, counts, (3, 30, 2))]
        outs.append((placed, out, lse, turned))
    placed = outs[1][0]
    for a, b in zip(outs[0][1:], outs[1][1:]):
        assert torch.equal(a[placed], b[placed])
