"""The page operations on the GPU against the list oracle: tables, counts, lists and pool contents, bit for bit."""
import random

import pytest
import torch

import paper_2604_18529_b200 as pkg
from oracle import hg_pages as O
from paper_2604_18529_b200 import binding as hg

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def ints(a):
    return torch.tensor(a, dtype=torch.int32, device=DEV)


class Pool:
    """A pool, a block table and their mirror in the oracle's lists."""

    def __init__(self, B, S, n, P=16, Hkv=2, D=64, dtype=torch.float16, layout="HND", seed=0):
        self.B, self.S, self.n, self.P = B, S, n, P
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        shape = (n, Hkv, P, D) if layout == "HND" else (n, P, Hkv, D)
        if layout == "padded":                        # pages of a larger array, token rows with a gap behind them
            shape = (n + 1, P, Hkv + 1, D)
        made = [torch.randint(-2 ** 15, 2 ** 15, shape, generator=g, device=DEV, dtype=torch.int16).view(dtype) for _ in range(2)]
        self.whole = made
        if layout == "padded":
            made = [x[1:, :, 1:] for x in made]
        self.k, self.v = [x if layout == "HND" else x.transpose(1, 2) for x in made]         # [n][Hkv][P][D]
        self.table, self.ref = torch.full((B, S), -1, dtype=torch.int32, device=DEV), ints([0] * n)
        self.lens, self.begin, self.end = ints([0] * B), ints([0] * B), ints([0] * B)
        self.status = ints([0])
        self.copy = [ints([7] * B) for _ in range(3)]
        self.ready, self.n_moves, self.remap = ints([7] * B), ints([7]), ints([7] * n)
        self.moves = [ints([7] * n) for _ in range(2)]
        self.desc = hg.attn_desc(batch=B, num_q_heads=Hkv, num_kv_heads=Hkv, head_dim=D, dtype=dtype, page_size=P, num_pages=n,
                                 page_stride=self.k.stride(0), head_stride=self.k.stride(1), tok_stride=self.k.stride(2),
                                 block_table=self.table, max_pages=S, chunk_tokens=max(64, P), num_chunks=1, status=self.status)
        self.o_table, self.o_ref = [[-1] * S for _ in range(B)], [0] * n
        self.o_lens, self.o_begin, self.o_end = [0] * B, [0] * B, [0] * B

    def load(self, table, ref, lens=None):
        self.o_table, self.o_ref = [list(r) for r in table], list(ref)
        self.table.copy_(ints(table))
        self.ref.copy_(ints(ref))
        if lens is not None:
            self.o_lens = list(lens)
            self.lens.copy_(ints(lens))

    def take_status(self):
        s = int(self.status)
        self.status.zero_()
        return s

    def check(self, what=""):
        assert self.table.tolist() == self.o_table, what
        assert self.ref.tolist() == self.o_ref, what
        assert (self.lens.tolist(), self.begin.tolist(), self.end.tolist()) == (self.o_lens, self.o_begin, self.o_end), what

    def fork(self, src):
        pkg.hg_kv_fork(ints(src), self.ref, self.lens, self.begin, self.end, self.desc)
        want = O.fork(self.o_table, self.o_ref, src, self.o_lens, self.o_begin, self.o_end)
        assert self.take_status() == want
        self.check("fork")

    def reserve(self, new):
        pkg.hg_kv_reserve(self.lens, None if new is None else ints(new), self.ref, *self.copy, self.ready, self.desc)
        src, dst, rows, ready, want = O.reserve(self.o_table, self.o_ref, self.o_lens, [1] * self.B if new is None else new, self.P)
        assert self.take_status() == want
        assert [t.tolist() for t in self.copy] == [src, dst, rows]
        assert self.ready.tolist() == ready
        self.check("reserve")
        return ready

    def bits(self):
        return [x.contiguous().view(torch.int16).clone() for x in (self.k, self.v)]

    def copy_pages(self, src, dst, rows, n_pairs=None):
        want = self.bits()
        pkg.hg_kv_copy_pages(src, dst, rows, n_pairs, self.k, self.v, self.desc)
        for x in want:
            for i, (a, b) in enumerate(zip(src.tolist(), dst.tolist())):
                if n_pairs is not None and i >= int(n_pairs):
                    break
                m = self.P if rows is None else max(0, min(int(rows[i]), self.P))
                if 0 <= a < self.n and 0 <= b < self.n:
                    x[b, :, :m] = x[a, :, :m]
        for x, y in zip(want, self.bits()):
            assert torch.equal(x, y)

    def compact(self, most):
        src, dst = self.moves[0][:most], self.moves[1][:most]
        pkg.hg_kv_compact(self.ref, self.remap, src, dst, self.n_moves, self.desc)
        pairs, remap = O.compact(self.o_table, self.o_ref, most)
        pad = [-1] * (most - len(pairs))
        assert int(self.n_moves) == len(pairs)
        assert src.tolist() == [a for a, _ in pairs] + pad and dst.tolist() == [b for _, b in pairs] + pad
        assert self.remap.tolist() == remap
        self.check("compact")
        return src, dst


@pytest.mark.parametrize("layout,P,Hkv,D,dtype", [("HND", 16, 2, 64, torch.float16), ("NHD", 32, 3, 128, torch.bfloat16),
                                                  ("padded", 64, 1, 64, torch.bfloat16), ("HND", 256, 5, 128, torch.float16),
                                                  ("HND", 128, 1, 128, torch.float16)])
@pytest.mark.parametrize("B,S,n", [(1, 1, 1), (5, 3, 9), (17, 6, 60), (33, 9, 300)])
def test_histories_against_the_oracle(B, S, n, layout, P, Hkv, D, dtype):
    r = random.Random(B * 1000 + P)
    p = Pool(B, S, n, P, Hkv, D, dtype, layout, seed=B + P)
    outside = [x.clone() for x in p.whole]
    for _ in range(8):
        p.fork([r.randrange(-1, B + 1) if r.random() < 0.4 else b for b in range(B)])
        ready = p.reserve(None if r.random() < 0.2 else [r.choice([-3, 0, 1, 1, 2, P, r.randint(0, S * P + 5)]) for _ in range(B)])
        p.copy_pages(*p.copy)
        p.o_lens = [a + b for a, b in zip(p.o_lens, ready)]
        p.lens.copy_(ints(p.o_lens))
        if r.random() < 0.6:
            src, dst = p.compact(r.randint(1, n))
            p.copy_pages(src, dst, None, p.n_moves)
    if layout == "padded":                            # nothing outside the pool's view was touched
        for x, y in zip(p.whole, outside):
            assert torch.equal(x[0].view(torch.int16), y[0].view(torch.int16))
            assert torch.equal(x[:, :, 0].contiguous().view(torch.int16), y[:, :, 0].contiguous().view(torch.int16))


def test_large_pool_and_batch_take_the_cluster():
    """More pages than one CTA scans, more rows than one CTA's threads."""
    B, S, P, n = 1100, 12, 16, 20000
    r = random.Random(3)
    p = Pool(B, S, n, P, 1, 64)
    ids = list(range(n))
    r.shuffle(ids)
    table, lens, at = [[-1] * S for _ in range(B)], [0] * B, 0
    ref = [0] * n
    for b in range(B // 2):
        lens[b] = r.randint(0, (S - 2) * P)
        for s in range(-(-lens[b] // P)):
            table[b][s] = ids[at]
            ref[ids[at]] = 1
            at += 1
    p.load(table, ref, lens)
    p.fork([b if b < B // 2 else r.randrange(B // 2) for b in range(B)])
    p.reserve([r.choice([0, 1, 5, 30]) for _ in range(B)])
    p.copy_pages(*p.copy)
    p.fork([b if r.random() < 0.5 else -1 for b in range(B)])
    src, dst = p.compact(700)
    p.copy_pages(src, dst, None, p.n_moves)
    src, dst = p.compact(n)
    p.copy_pages(src, dst, None, p.n_moves)
    p.reserve([S * P] * B)


@pytest.mark.parametrize("S", [8, 9])
@pytest.mark.parametrize("n", [8192, 8193])
def test_compaction_renames_tables_of_all_sizes(S, n):
    """Pools and tables on both sides of what the compacting CTA renames by itself."""
    B, P = 1024, 16
    r = random.Random(S + n)
    p = Pool(B, S, n, P, 1, 64)
    pages = r.sample(range(n), 3000)
    table = [[r.choice(pages) if r.random() < 0.5 else r.choice([-1, n, n + 7]) for _ in range(S)] for _ in range(B)]
    ref = [0] * n
    for row in table:
        for e in row:
            if 0 <= e < n:
                ref[e] += 1
    p.load(table, ref, [0] * B)
    for most in (1, 500, n):
        src, dst = p.compact(most)
        p.copy_pages(src, dst, None, p.n_moves)


@pytest.mark.parametrize("n", [700, 16384, 16385])
@pytest.mark.parametrize("rows,new", [(300, 1), (1024, 1), (1025, 1), (300, 60), (0, 1)])
def test_few_slots_of_a_large_table(n, rows, new):
    """A table that takes the cluster, pools and numbers of slots on both sides of what one of its CTAs does alone."""
    B, S, P = 1100, 40, 16
    r = random.Random(n + rows)
    p = Pool(B, S, n, P, 1, 64)
    pages, table, lens, ref = r.sample(range(n), 400), [[-1] * S for _ in range(B)], [0] * B, [0] * n
    for b in range(B):
        lens[b] = r.randint(0, 3 * P)
        for s in range(-(-lens[b] // P)):
            table[b][s] = r.choice(pages)                  # shared by some eight rows each
            ref[table[b][s]] += 1
    p.load(table, ref, lens)
    want = r.sample(range(B), rows)
    for _ in range(2):
        ready = p.reserve([new if b in want else 0 for b in range(B)])
        p.copy_pages(*p.copy)
        p.o_lens = [a + b for a, b in zip(p.o_lens, ready)]
        p.lens.copy_(ints(p.o_lens))


@pytest.mark.parametrize("B,S", [(64, 3), (65, 40), (129, 300), (700, 33), (16384, 2), (65535, 3)])
def test_forks_of_large_batches(B, S):
    """Rows shared out over a cluster; random sources, every row possibly another's."""
    n = 500
    g = torch.Generator(device=DEV)
    g.manual_seed(B)
    rnd = lambda lo, hi, *s: torch.randint(lo, hi, s, generator=g, device=DEV, dtype=torch.int32)   # noqa: E731
    table, lens = rnd(-1, n, B, S), rnd(0, 99, B)
    ref = torch.bincount(table[table >= 0].long(), minlength=n).int()
    src = torch.where(torch.rand(B, generator=g, device=DEV) < 0.7, rnd(-1, B, B), torch.arange(B, dtype=torch.int32, device=DEV))
    want = torch.where((src < 0)[:, None], -1, table[src.clamp(min=0).long()])
    want_lens = torch.where(src < 0, 0, lens[src.clamp(min=0).long()])
    desc = hg.attn_desc(batch=B, num_q_heads=1, num_kv_heads=1, head_dim=64, dtype="f16", page_size=16, num_pages=n, page_stride=1024,
                        head_stride=1024, tok_stride=64, block_table=table, max_pages=S, chunk_tokens=64, num_chunks=1)
    pkg.hg_kv_fork(src, ref, lens, None, None, desc)
    assert torch.equal(table, want) and torch.equal(lens, want_lens)
    assert torch.equal(ref, torch.bincount(want[want >= 0].long(), minlength=n).int())


def test_one_row_takes_many_pages_and_the_pool_runs_dry():
    p = Pool(3, 4000, 9000, 16, 1, 64)
    assert p.reserve([0, 50000, 100]) == [0, 50000, 100]
    assert p.reserve([64000, 0, 0]) == [64000, 0, 0]
    p.fork([-1, 1, 2])
    assert p.reserve([64000, 0, 64000])[0] == 64000
    q = Pool(2, 6000, 9000, 16, 1, 64)
    assert q.reserve([96000, 96000]) == [96000, 48000]


def test_more_slots_than_one_call_looks_at():
    """The call hands out its 262144 slots' pages and says where it stopped."""
    B, S, n = 64, 5000, 300000
    table, ref = torch.full((B, S), -1, dtype=torch.int32, device=DEV), torch.zeros(n, dtype=torch.int32, device=DEV)
    status, lens = ints([0]), ints([0] * B)
    desc = hg.attn_desc(batch=B, num_q_heads=1, num_kv_heads=1, head_dim=64, dtype="f16", page_size=16, num_pages=n, page_stride=1024,
                        head_stride=1024, tok_stride=64, block_table=table, max_pages=S, chunk_tokens=64, num_chunks=1, status=status)
    cs, cd, ready = ints([0] * B), ints([0] * B), ints([0] * B)
    pkg.hg_kv_reserve(lens, ints([S * 16] * B), ref, cs, cd, None, ready, desc)
    whole, rest = divmod(262144, S)
    assert ready.tolist() == [S * 16] * whole + [rest * 16] + [0] * (B - whole - 1)
    assert torch.equal(table.reshape(-1)[:262144], torch.arange(262144, dtype=torch.int32, device=DEV))
    assert int((table.reshape(-1)[262144:] != -1).sum()) == 0 and int(ref.sum()) == 262144 and int(ref.max()) == 1
    lens.copy_(ready)
    pkg.hg_kv_reserve(lens, ints([S * 16] * B) - ready, ref, cs, cd, None, ready, desc)
    assert int(status) == hg.HG_DEV_NO_PAGE and int(ref.sum()) == n
    assert torch.equal(table.reshape(-1)[:n], torch.arange(n, dtype=torch.int32, device=DEV))


def test_entries_outside_the_pool_are_reported_and_left_alone():
    p = Pool(3, 2, 4)
    p.load([[0, 9], [0, 9], [4, -1]], [2, 0, 0, 0], [10, 20, 3])
    p.reserve([10, 1, 1])
    p.fork([1, 0, 0])
    p.compact(4)
    p.copy_pages(ints([0, 1, -1, 4, 2, 2]), ints([1, 1, 2, 3, 4, 3]), ints([20, 3, 16, 16, 16, -2]))
    assert p.take_status() == hg.HG_DEV_BAD_PAGE


def test_release_takes_what_eviction_lists():
    p = Pool(2, 8, 30)
    p.reserve([100, 100])
    p.lens.copy_(ints([100, 100]))
    p.o_lens = [100, 100]
    p.end.copy_(ints([100, 100]))
    k_out, v_out = (torch.empty(2, 64, 2, 64, dtype=torch.float16, device=DEV) for _ in range(2))
    freed, n_freed = ints([[0] * 6] * 2), ints([0, 0])
    pkg.hg_kv_evict(p.k, p.v, p.begin, p.end, ints([50, 16]), k_out, v_out, freed, n_freed, p.desc)
    assert n_freed.tolist() == [3, 1]
    pkg.hg_kv_release(freed, p.ref, p.desc)
    assert p.take_status() == 0
    for e in freed.reshape(-1).tolist():
        if e >= 0:
            p.o_ref[e] -= 1
    assert p.ref.tolist() == p.o_ref and sum(p.o_ref) == 10
    pkg.hg_kv_release(ints([29, 5, -4, 30]), p.ref, p.desc)                # a free page, one out of the pool
    p.o_ref[5] -= 1
    assert p.take_status() == hg.HG_DEV_BAD_PAGE and p.ref.tolist() == p.o_ref


def test_offsets_past_32_bits():
    """Pages whose offset in elements and in bytes does not fit 32 bits."""
    n, D, P = 3, 64, 16
    stride = (1 << 31) + 8 * 1024
    whole = torch.empty(2 * stride + P * D, dtype=torch.float16, device=DEV)
    k = whole.as_strided((n, 1, P, D), (stride, P * D, D, 1))
    k[:2].view(torch.int16).copy_(torch.randint(-2 ** 15, 2 ** 15, (2, 1, P, D), dtype=torch.int16))
    desc = hg.attn_desc(batch=1, num_q_heads=1, num_kv_heads=1, head_dim=D, dtype="f16", page_size=P, num_pages=n, page_stride=stride,
                        head_stride=P * D, tok_stride=D, block_table=ints([[0]]), max_pages=1, chunk_tokens=64, num_chunks=1)
    v = torch.zeros_like(whole).as_strided((n, 1, P, D), (stride, P * D, D, 1))
    pkg.hg_kv_copy_pages(ints([1]), ints([2]), None, None, k, v, desc)
    assert torch.equal(k[2].view(torch.int16), k[1].view(torch.int16)) and not torch.equal(k[2].view(torch.int16), k[0].view(torch.int16))


def test_captured_on_another_stream_and_replayed():
    """A branching step as a graph: every replay works on the state the one before left."""
    def fresh():
        p = Pool(6, 5, 40, seed=4)
        p.reserve([40, 17, 0, 0, 0, 0])
        p.o_lens = [40, 17, 0, 0, 0, 0]
        p.lens.copy_(ints(p.o_lens))
        return p

    p, src = fresh(), [0, 1, 0, 0, 1, 3]
    s, src_d = torch.cuda.Stream(), ints(src)
    g = torch.cuda.CUDAGraph()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=s):
        pkg.hg_kv_fork(src_d, p.ref, p.lens, p.begin, p.end, p.desc)
        pkg.hg_kv_reserve(p.lens, None, p.ref, *p.copy, p.ready, p.desc)
        pkg.hg_kv_copy_pages(*p.copy, None, p.k, p.v, p.desc)
    q = fresh()
    for _ in range(3):
        g.replay()
        q.fork(src)
        q.reserve(None)
        q.copy_pages(*q.copy)
        torch.cuda.synchronize()
        assert torch.equal(p.table, q.table) and torch.equal(p.ref, q.ref) and p.lens.tolist() == q.o_lens
        for x, y in zip(p.bits(), q.bits()):
            assert torch.equal(x, y)


def test_wrong_tensors_are_refused_by_the_binding():
    p = Pool(3, 2, 9)
    with pytest.raises(ValueError):
        pkg.hg_kv_fork(ints([0, 1]), p.ref, p.lens, None, None, p.desc)             # two rows for a batch of three
    with pytest.raises(ValueError):
        pkg.hg_kv_fork(ints([0, 1, 2]), p.ref[:5], p.lens, None, None, p.desc)      # fewer counts than pages
    with pytest.raises(ValueError):
        pkg.hg_kv_reserve(p.lens.long(), None, p.ref, *p.copy, None, p.desc)
    with pytest.raises(ValueError):
        pkg.hg_kv_copy_pages(p.copy[0], p.copy[1][:2], None, None, p.k, p.v, p.desc)
    with pytest.raises(hg.HgError):
        pkg.hg_kv_reserve(p.lens, None, torch.zeros(10, dtype=torch.int32, device=DEV)[1:], *p.copy, None, p.desc)  # misaligned


@pytest.mark.parametrize("same", ["end", "begin", "begin and end", "all"])
@pytest.mark.parametrize("B", [6, 300, 700])
def test_fork_moves_an_array_once_that_it_is_given_twice(B, same):
    """Callers whose tokens are all on the GPU keep one array for seq_lens and tok_end; rows swap, branch and end."""
    r = random.Random(B)
    S, n = 3, 4 * B
    table = [[r.choice([-1, r.randrange(n)]) for _ in range(S)] for _ in range(B)]
    ref = [0] * n
    for row in table:
        for e in row:
            if e >= 0:
                ref[e] += 1
    lens, begin, end = ([r.randint(1, 48) for _ in range(B)] for _ in range(3))
    src = [r.randrange(-1, B) for _ in range(B)]
    src[0], src[1] = 1, 0
    p = Pool(B, S, n, 16, 1, 64)
    p.load(table, ref, lens)
    p.begin.copy_(ints(begin))
    p.end.copy_(ints(end))
    args = {"end": (p.lens, p.begin, p.lens), "begin": (p.lens, p.lens, p.end), "begin and end": (p.lens, p.end, p.end),
            "all": (p.lens, p.lens, p.lens)}[same]
    p.o_begin, p.o_end = list(begin), list(end)
    moved = [{id(p.lens): p.o_lens, id(p.begin): p.o_begin, id(p.end): p.o_end}[i] for i in {id(t) for t in args}]
    pkg.hg_kv_fork(ints(src), p.ref, *args, p.desc)
    assert p.take_status() == O.fork(p.o_table, p.o_ref, src, *moved)
    p.check(same)


@pytest.mark.parametrize("Hq,Hkv,D,P", [(8, 2, 64, 16), (4, 4, 128, 16), (32, 2, 128, 64)])
def test_attention_directly_behind_table_operations(Hq, Hkv, D, P):
    """Attention launched as a programmatic dependent of the kernel that changes its table and ranges (few chunk slots, no
    counter to clear), the stream backed up so that it starts early: the bits of a run that waits after every call."""
    B, S, n, NC, rounds = 6, 8, 40, max(8 * P // 64, 1) + 1, 30

    def run(waits):
        r = random.Random(D + P)
        p = Pool(B, S, n, P, Hkv, D, seed=D)
        for i, x in enumerate((p.k, p.v)):
            g = torch.Generator(device=DEV)
            g.manual_seed(i)
            x.copy_(torch.randn(x.shape, generator=g, device=DEV))
        p.desc.num_q_heads, p.desc.num_chunks = Hq, NC
        p.desc.tune = 4 if waits else 0                       # HG_TUNE_NO_PDL for the side that is waited for
        q = torch.randn(B, Hq, D, generator=g, device=DEV).half()
        ws = torch.empty(pkg.hg_attn_workspace_bytes(p.desc, 0), dtype=torch.uint8, device=DEV)
        outs = [[torch.zeros(B, Hq, D, device=DEV), torch.zeros(B, Hq, device=DEV), torch.zeros(B, Hq, NC, D, device=DEV),
                 torch.zeros(B, Hq, NC, device=DEV), torch.zeros(B, Hq, NC, device=DEV)] for _ in range(4 * rounds)]
        srcs = [ints([r.randrange(-1, B) if r.random() < 0.7 else b for b in range(B)]) for _ in range(2 * rounds)]
        news = [ints([r.choice([0, 1, P, 3 * P + 5]) for _ in range(B)]) for _ in range(rounds)]
        most = [r.randint(1, n) for _ in range(rounds)]
        torch.cuda.synchronize()
        if not waits:
            torch.cuda._sleep(100_000_000)                    # some 50 ms: the calls below queue up behind it
        at = iter(outs)

        def call(f, *a):
            f(*a, p.desc)
            if waits:
                torch.cuda.synchronize()

        def attend(whole):
            out, lse, o, m, l = next(at)
            if whole:
                call(pkg.hg_attn_decode, q, p.k, p.v, p.lens, p.begin, p.end, [], out, lse, ws)
            else:
                call(pkg.hg_attn_partial, q, p.k, p.v, p.lens, p.begin, p.end, o, m, l)

        for i in range(rounds):
            call(pkg.hg_kv_fork, srcs[2 * i], p.ref, p.lens, p.begin, p.end)
            attend(i % 2)
            call(pkg.hg_kv_reserve, p.lens, news[i], p.ref, *p.copy, p.ready)
            call(pkg.hg_kv_copy_pages, *p.copy, None, p.k, p.v)
            attend((i + 1) % 2)
            p.lens.add_(p.ready)
            p.end.copy_(p.lens)
            call(pkg.hg_kv_compact, p.ref, p.remap, p.moves[0][:most[i]], p.moves[1][:most[i]], p.n_moves)
            call(pkg.hg_kv_copy_pages, p.moves[0][:most[i]], p.moves[1][:most[i]], None, p.n_moves, p.k, p.v)
            attend(i % 2)
            call(pkg.hg_kv_fork, srcs[2 * i + 1], p.ref, p.lens, p.begin, p.end)
            attend((i + 1) % 2)
        torch.cuda.synchronize()
        return [t for o in outs for t in o] + [p.table, p.ref, p.lens, p.status]

    want, got = run(True), run(False)
    assert sum(int(t.count_nonzero()) for t in want[:-4]) > 0
    for i, (x, y) in enumerate(zip(got, want)):
        assert torch.equal(x, y), i


def test_lists_of_31_bits():
    """The longest lists that the calls take: every entry is looked at or written, nothing behind them."""
    n, most = 64, 2 ** 31 - 1
    p = Pool(2, 3, n, 16, 1, 64)
    p.load([[5, -1, -1], [9, -1, -1]], [2 if i in (5, 9) else 0 for i in range(n)], [0, 0])
    ids = torch.full((most,), -1, dtype=torch.int32, device=DEV)
    ids[most - 1], ids[most - 300000] = 9, 5
    pkg.hg_kv_release(ids, p.ref, p.desc)
    assert p.take_status() == 0
    for e in (5, 9):
        p.o_ref[e] -= 1
    p.check("release")
    lists = [torch.full((most + 1,), 7, dtype=torch.int32, device=DEV) for _ in range(2)]
    del ids
    pkg.hg_kv_compact(p.ref, p.remap, lists[0][:most], lists[1][:most], p.n_moves, p.desc)
    pairs, remap = O.compact(p.o_table, p.o_ref, most)
    assert int(p.n_moves) == len(pairs) == 2 and p.remap.tolist() == remap
    p.check("compact")
    for x, want in zip(lists, zip(*pairs)):
        assert x[:2].tolist() == list(want) and int(x[most]) == 7
        assert int(x[2:most].max()) == int(x[2:most].min()) == -1
