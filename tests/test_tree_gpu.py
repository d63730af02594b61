"""Attention of a step's new tokens on the GPU against a plain softmax in 64 bits.

Tolerances.  q and k have components of order 1, so |q| |k| / sqrt(D) is about 14 * 15 / 11.3 = 18.6 at D = 128; a sum of D
products in fp32 has D roundings of at most 2^-24 of that, independent ones: sqrt(128) * 2^-24 * 18.6 * 4 (four standard
deviations) = 5e-5, doubled for an accumulator that truncates: a logit is off by at most 1e-4, and so is the log-sum-exp.
Weights, normalised, are off by twice that, half of them with the other sign: 1e-4 of the mean of |V| under the weights.
Then a weight is rounded to the 16-bit type, by at most u = eps / 2 of itself, or, with fp16, by 2^-25 of a weight of 1 (and
weights refer to a logit at most 2^8 below the largest): out is off by at most u of the mean of |V| under the weights, plus,
with fp16, 2^-25 of the sum of |V| over the tokens divided by the sum of weights, which is at least that of the largest, 1;
the sum by the tensor cores is cut off by 2.3e-9 of the same mean for every token; and out itself is rounded by u of itself.
The plain softmax gives those means with |V| in the place of V.
"""
import numpy as np
import pytest
import torch

import paper_2604_18529_b200 as pkg
from paper_2604_18529_b200 import binding as hg

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F16, BF16 = torch.float16, torch.bfloat16
LOGIT = 1e-4
INF = float("inf")


def ints(a, dtype=torch.int32):
    return torch.tensor(a, dtype=dtype, device=DEV)


def bits(rows, words):
    """Lists of visible tokens -> int32 [N][words]"""
    m = np.zeros((len(rows), words), dtype=np.uint32)
    for r, row in enumerate(rows):
        for j in row:
            m[r, j // 32] |= np.uint32(1) << np.uint32(j % 32)
    return torch.from_numpy(m.view(np.int32)).to(DEV)


def tree_rows(n, rng):
    """A random tree's ancestors (and itself) of every token"""
    rows = []
    for i in range(n):
        p = rng.randint(-1, i)
        rows.append((rows[p] if p >= 0 else []) + [i])
    return rows


class Step:
    """Sequences with cached tokens [begin, len) and new ones behind, pages anywhere in the pool, NaN wherever nobody looks."""

    def __init__(self, lens, nodes, Hq=8, Hkv=2, D=128, P=16, dtype=F16, begin=None, kind="tree", layout="HND", fused=False, pad=3, host=(),
                 seed=0, flags=0, scale=0.0, words=None, max_nodes=None, masks=None):
        B = len(lens)
        self.B, self.lens, self.nodes, self.Hq, self.Hkv, self.D, self.P, self.dtype = B, lens, nodes, Hq, Hkv, D, P, dtype
        self.begin = begin or [0] * B
        rng = np.random.RandomState(seed)
        self.cu = np.concatenate([[0], np.cumsum(nodes)]).tolist()
        self.N = self.cu[-1] + pad
        if masks is not None:
            self.sees = masks
        elif kind == "chain":
            self.sees = [[list(range(i + 1)) for i in range(n)] for n in nodes]
        elif kind == "tree":
            self.sees = [tree_rows(n, rng) for n in nodes]
        else:                                               # any bits, some rows without one
            self.sees = [[[j for j in range(n) if rng.rand() < 0.4] if rng.rand() < 0.7 else [] for _ in range(n)] for n in nodes]
        counts = [-(-(t + n) // P) for t, n in zip(lens, nodes)]
        S = max(counts + [1])
        n_pages = sum(counts) + 3
        table = np.full((B, S), -1, dtype=np.int32)
        ids = rng.permutation(n_pages).astype(np.int32)
        at = 0
        used = []
        for b, c in enumerate(counts):
            table[b, :c] = ids[at:at + c]
            table[b, :self.begin[b] // P] = -1               # what lies wholly in front is not mapped
            at += c
            for t in range(self.begin[b], lens[b] + nodes[b]):
                used.append((table[b, t // P], t % P))
        self.table = torch.from_numpy(table).to(DEV)
        gen = torch.Generator(device=DEV)
        gen.manual_seed(seed)
        shape = (n_pages, Hkv, P, D) if layout == "HND" else (n_pages, P, Hkv, D)
        k, v = [torch.randn(shape, generator=gen, device=DEV).to(dtype) for _ in range(2)]
        self.k, self.v = (k, v) if layout == "HND" else (k.transpose(1, 2), v.transpose(1, 2))
        nobody = torch.ones((n_pages, P), dtype=torch.bool)
        if used:
            nobody[tuple(torch.tensor(np.array(used)).T.long())] = False
        for x in (self.k, self.v):
            x.masked_fill_(nobody.to(DEV)[:, None, :, None], float("nan"))
        q = torch.randn((self.N, Hq + (2 * Hkv if fused else 0), D), generator=gen, device=DEV).to(dtype)
        q[self.cu[-1]:] = float("nan")
        self.q = q[:, :Hq]
        self.scale = scale or D ** -0.5
        self.host = []
        for nc in host:
            m = torch.randn((self.N, Hq, nc), generator=gen, device=DEV) * 3 + 1
            l = torch.rand((self.N, Hq, nc), generator=gen, device=DEV) * 20 + 1
            empty = torch.rand((self.N, Hq, nc), generator=gen, device=DEV) < 0.2
            m[empty], l[empty] = -INF, 0.0
            o = torch.randn((self.N, Hq, nc, D), generator=gen, device=DEV) * 5
            o[empty] = float("nan")                          # never read
            self.host.append((o, m, l))
        self.status = ints([0])
        self.desc = hg.attn_desc(batch=B, num_q_heads=Hq, num_kv_heads=Hkv, head_dim=D, dtype=dtype, page_size=P, num_pages=n_pages,
                                 page_stride=self.k.stride(0), head_stride=self.k.stride(1), tok_stride=self.k.stride(2),
                                 block_table=self.table, max_pages=S, chunk_tokens=max(128, P), num_chunks=1, scale=scale, status=self.status,
                                 flags=flags)
        most = max(nodes + [1])
        self.mask = None if kind == "chain" and masks is None else \
            bits([row for s in self.sees for row in s] + [[]] * pad, words or -(-most // 32))
        self.tree = hg.tree_desc(cu_nodes=ints(self.cu), mask=self.mask, num_rows=self.N, max_nodes=max_nodes or most)
        self.seq_lens, self.tok_begin = ints(lens), ints(self.begin) if begin else None
        self.ws = torch.full((hg.hg_attn_tree_workspace_bytes(self.desc, self.tree),), 0x7f, dtype=torch.uint8, device=DEV)
        self.out = torch.full((self.N, Hq, D), -77.0, dtype=dtype, device=DEV)
        self.lse = torch.full((self.N, Hq), -77.0, device=DEV)

    def call(self, **over):
        a = dict(out=self.out, lse=self.lse, ws=self.ws, stream=None)
        a.update(over)
        hg.hg_attn_decode_tree(self.q, self.k, self.v, self.seq_lens, self.tok_begin, self.host, a["out"], a["lse"], a["ws"], self.desc,
                               self.tree, a["stream"])

    def rows(self, pool, b, t):
        page = self.table[b].long()[t // self.P]
        return pool[page, :, t % self.P].double().transpose(0, 1)

    def exact(self, drop=()):
        """(out, lse, how far out may be off) of the rows in use; ``drop``: (sequence, position) pairs to leave out"""
        G, u = self.Hq // self.Hkv, torch.finfo(self.dtype).eps / 2
        outs, lses, offs = [], [], []
        for b in range(self.B):
            n, L = self.nodes[b], self.lens[b]
            if n == 0:
                continue
            t = torch.arange(self.begin[b], L + n, device=DEV)
            hidden = torch.zeros((n, t.numel()), dtype=torch.bool, device=DEV)
            hidden[:, t.numel() - n:] = True
            for i in range(n):
                for j in self.sees[b][i]:
                    if j < n:
                        hidden[i, t.numel() - n + j] = False
            for x, y in drop:
                if x == b:
                    hidden[:, y - self.begin[b]] = True
            k, v = self.rows(self.k, b, t), self.rows(self.v, b, t)             # [Hkv][t][D]
            q = self.q[self.cu[b]:self.cu[b + 1]].double().reshape(n, self.Hkv, G, self.D)
            x = torch.einsum("nhgd,htd->nhgt", q, k) * self.scale
            x = x.masked_fill(hidden[:, None, None], -INF)
            v = v.nan_to_num(0, 0, 0)                                          # (rows nobody sees, in the tests that plant such)
            m = x.amax(3, keepdim=True)
            p = (x - torch.where(m == -INF, 0.0, m)).exp()
            m, l = m[..., 0], p.sum(3)
            o, a = torch.einsum("nhgt,htd->nhgd", p, v), torch.einsum("nhgt,htd->nhgd", p, v.abs())
            small = v.abs().sum(1)[None, :, None] * 2.0 ** -25 * (self.dtype == F16)
            srcs = [(o, a, m, l)]
            for ho, hm, hl in self.host:
                s = slice(self.cu[b], self.cu[b + 1])
                ho = torch.where((hm[s] == -INF)[..., None], 0.0, ho[s]).double()
                for c in range(hm.shape[2]):
                    sh = (n, self.Hkv, G)
                    srcs.append((ho[:, :, c].reshape(*sh, self.D), None, hm[s, :, c].double().reshape(sh), hl[s, :, c].double().reshape(sh)))
            top = torch.stack([y[2] for y in srcs]).amax(0)
            w = [(y[2] - torch.where(top == -INF, 0.0, top)).exp() for y in srcs]
            L_ = sum(y[3] * z for y, z in zip(srcs, w))
            O = sum(y[0] * z[..., None] for y, z in zip(srcs, w))
            safe = torch.where(L_ == 0, 1.0, L_)[..., None]
            out = O / safe
            mean = a * w[0][..., None] / safe
            off = (u + LOGIT + 2.3e-9 * t.numel()) * mean + small * w[0][..., None] / safe + u * out.abs() + LOGIT * out.abs() + 2.0 ** -24
            outs.append(out.reshape(n, self.Hq, self.D))
            offs.append(off.reshape(n, self.Hq, self.D))
            lses.append((top + torch.where(L_ == 0, 1.0, L_).log()).reshape(n, self.Hq))
        e = torch.empty(0, self.Hq, self.D, dtype=torch.float64, device=DEV)
        return torch.cat(outs + [e]), torch.cat(lses + [e[..., 0]]), torch.cat(offs + [e])

    def check(self, drop=(), status=0):
        self.call()
        torch.cuda.synchronize()
        assert int(self.status) == status
        out, lse, off = self.exact(drop)
        n = self.cu[-1]
        got = self.out[:n].double()
        worst = ((got - out).abs() / off).max() if n else 0
        assert torch.isfinite(got).all() and float(worst) <= 1, float(worst)
        none = lse == -INF
        assert torch.equal(self.lse[:n] == -INF, none) and (got[none] == 0).all()
        assert n == 0 or float((self.lse[:n].double() - lse)[~none].abs().amax() if (~none).any() else 0) <= LOGIT
        assert (self.out[n:] == -77).all() and (self.lse[n:] == -77).all()       # rows behind the last


LENS, NODES = [300, 0, 17, 1, 128, 1000], [5, 7, 0, 1, 32, 3]


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kind", ["chain", "tree", "any"])
def test_types_components_and_masks(dtype, D, kind):
    Step(LENS, NODES, D=D, dtype=dtype, kind=kind).check()


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (4, 4), (7, 1), (10, 2), (12, 1), (64, 8), (24, 3), (96, 1), (128, 1)])
def test_heads(Hq, Hkv):
    Step([90, 200], [9, 33], Hq=Hq, Hkv=Hkv).check()


@pytest.mark.parametrize("P", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("layout", ["HND", "NHD"])
def test_pages_and_layouts(P, layout):
    Step([P - 1, P, P + 1, 3 * P + 5], [2, 40, 1, 19], P=P, layout=layout, kind="tree", D=64 if P == 32 else 128).check()


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 300])
@pytest.mark.parametrize("Hq,Hkv", [(16, 2), (2, 2)])
def test_numbers_of_new_tokens(n, Hq, Hkv):
    """Row tiles: of 16 tokens with 8 heads a KV head, of 128 with one; masks of several words"""
    Step([n + 100, 3], [n, 1], Hq=Hq, Hkv=Hkv, kind="tree" if n % 2 else "chain", dtype=BF16 if n > 64 else F16).check()


@pytest.mark.parametrize("length", [0, 1, 31, 32, 95, 96, 97, 127, 128, 129, 255, 256, 257, 384])
def test_cached_lengths_around_a_tile(length):
    Step([length] * 2, [32, 5], kind="any", seed=length).check()


@pytest.mark.parametrize("begin", [[0, 0], [5, 999], [128, 640], [300, 1000], [299, 513]])
def test_slices_that_begin_later(begin):
    s = Step([300, 1000], [6, 20], begin=begin, D=64)
    s.check()
    s.tok_begin = ints([b if b < n else b + 1000 for b, n in zip(begin, s.lens)])      # beyond the end: nothing of the cache
    s.check()


@pytest.mark.parametrize("host", [(1,), (3, 1), (1, 2, 1, 5, 1, 1, 1, 17)])
@pytest.mark.parametrize("D", [64, 128])
def test_host_partials(host, D):
    Step([400, 0, 77], [5, 3, 40], host=host, D=D, kind="any", dtype=BF16).check()


def test_rows_that_see_nothing():
    s = Step([0, 50], [4, 3], masks=[[[], [0, 1], [], [3]], [[], [], []]], begin=[0, 50])
    s.check()
    assert (s.lse[[0, 2, 4, 5, 6]] == -INF).all() and (s.out[[0, 2, 4, 5, 6]] == 0).all()
    h = Step([0, 50], [4, 3], masks=[[[], [0, 1], [], [3]], [[], [], []]], begin=[0, 50], host=(2,))
    h.check()


def test_wide_masks_and_spare_bits():
    """Bits of tokens that do not exist, and words that nobody needs"""
    s = Step([40, 20], [5, 9], masks=[[[i, 17, 63, 90] for i in range(5)], [[i, 9, 31, 32, 95] for i in range(9)]], words=3)
    s.check()
    t = Step([40, 20], [5, 9], masks=[[[i] for i in range(5)], [[i] for i in range(9)]], max_nodes=64, words=2)
    t.check()


@pytest.mark.parametrize("bad", [float("nan"), INF, -INF])
@pytest.mark.parametrize("dtype,D", [(F16, 128), (BF16, 64)])
@pytest.mark.parametrize("Hkv", [1, 4])                                       # 80 and 20 rows a KV head
def test_what_masked_tokens_hold_does_not_matter(bad, dtype, D, Hkv):
    """Token 3 of each sequence overflows; nobody but token 6 sees it"""
    sees = [[i] if i != 6 else [3, 6] for i in range(20)]
    s = Step([130, 9], [20, 7], masks=[sees, sees[:7]], dtype=dtype, D=D, Hq=4, Hkv=Hkv)
    s.call()
    want, want_lse = s.out.clone(), s.lse.clone()
    for b in range(2):
        t = s.lens[b] + 3
        page = int(s.table[b, t // s.P])
        s.k[page, :, t % s.P] = bad
        s.v[page, Hkv - 1, t % s.P, 5] = bad
    s.out.fill_(-77)
    s.call()
    torch.cuda.synchronize()
    others = [r for r in range(27) if r not in (3, 6, 20 + 3, 20 + 6)]       # (token 3 sees itself)
    assert torch.equal(s.out[others], want[others]) and torch.equal(s.lse[others], want_lse[others])
    s2 = Step([130, 9], [20, 7], masks=[sees, sees[:7]], dtype=dtype, D=D, Hq=4, Hkv=Hkv)
    for b in range(2):                                                      # only V: the logits of token 6 stay
        t = s2.lens[b] + 3
        s2.v[int(s2.table[b, t // s2.P]), Hkv - 1, t % s2.P, 5] = bad
    s2.call()
    torch.cuda.synchronize()
    seers = [3, 6, 23, 26]
    first = 4 - 4 // Hkv                                                    # of the heads that read the last KV head
    assert not torch.isfinite(s2.out[seers, first:, 5]).any() and torch.equal(s2.out[seers, :first], want[seers, :first])
    assert torch.equal(s2.out[others], want[others]) and torch.equal(s2.lse[:27], want_lse[:27])


def test_fused_queries_and_a_scale():
    Step([100, 30], [12, 3], fused=True, scale=0.25).check()


def one_logit(lens, nodes, logit, Hq, Hkv, D, dtype=F16, **kw):
    """A step whose logits are those of ``logit(position)`` (all heads alike, rounded to the type) and whose V are positive"""
    s = Step(lens, nodes, Hq=Hq, Hkv=Hkv, D=D, dtype=dtype, scale=1.0, **kw)
    s.q[...] = 0
    s.q[..., 0] = 4
    v = torch.rand(s.v.shape, device=DEV) * 500 + 500
    for b in range(s.B):
        t = torch.arange(lens[b] + nodes[b], device=DEV)
        page, row = s.table[b].long()[t // s.P], t % s.P
        key = torch.zeros((t.numel(), Hkv, D), device=DEV)
        key[..., 0] = (logit(t) / 4)[:, None]
        s.k[page, :, row] = key.to(dtype)
        s.v[page, :, row] = v[page, :, row].to(dtype)
    return s


SHAPES = [(8, 2, 3), (8, 2, 8), (8, 2, 20), (8, 2, 40)]                      # 12, 32, 80 and 160 rows a KV head


@pytest.mark.parametrize("depth", [12.0, 15.0, 17.0, 17.5])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv,n", SHAPES)
def test_small_weights_beside_large_ones(depth, D, Hq, Hkv, n):
    """Every 64th token takes nearly all the weight and has V = 0; out is what the others give, e^-depth of it each.

    A weight is off by u = 2^-11 of itself, or by 2^-32 of the largest where that is more (half a step of the smallest fp16
    numbers, 2^-25, in weights that are 2^7 times as large), so out, all V being positive, by u of itself and 2^-32 of the sum
    of V over the sum of weights, one for every 64 tokens at least; the rest is as in the tolerances above."""
    for length in (100, 1000, 9000):
        s = one_logit([length], [n], lambda t: torch.where(t % 64 == 0, 0.0, -depth - (t * 37 % 64) / 256), Hq, Hkv, D, kind="chain")
        t = torch.arange(length, device=DEV)
        page, row = s.table[0].long()[t // s.P], t % s.P
        s.v[page[::64], :, row[::64]] = 0
        s.call()
        torch.cuda.synchronize()
        out, lse, _ = s.exact()
        u, total = 2.0 ** -11, length + n
        off = (2 * u + LOGIT + 2.3e-9 * total) * out + 2.0 ** -32 * 1000 * 64 * total / (total - 63) + 2.0 ** -24
        worst = float(((s.out[:n].double() - out).abs() / off).max())
        assert worst <= 1, (length, worst)
        assert float((s.lse[:n].double() - lse).abs().max()) <= LOGIT


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("Hq,Hkv,n", SHAPES)
def test_one_token_above_a_long_tail(dtype, Hq, Hkv, n):
    """The first token, and 30 000 that are e^-14 of it together with it: a tenth of a percent of the weight"""
    for b in range(2):
        s = one_logit([30000], [n], lambda t: torch.where(t == 0, 0.0, -14.0 - (t % 64) / 64), Hq, Hkv, 64, dtype, kind="chain", P=64,
                      host=(2,) * b)
        s.check()


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("rise", [5.4, 5.7, 11.0])                           # nats a tile; a reference follows from 2^8 (5.5) on
@pytest.mark.parametrize("Hq,Hkv,n", SHAPES)
def test_logits_that_climb(dtype, rise, Hq, Hkv, n):
    s = one_logit([900], [n], lambda t: (t // 128) * rise - 30.0, Hq, Hkv, 128, dtype, kind="chain", host=(1,))
    s.check()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv,n", SHAPES)
def test_host_partials_with_fp16(D, Hq, Hkv, n):
    Step([400, 0, 2077], [n, 3, 1], Hq=Hq, Hkv=Hkv, D=D, host=(3, 1), kind="any").check()


def test_many_short_sequences():
    r = np.random.RandomState(3)
    Step(r.randint(0, 200, 700).tolist(), r.randint(0, 5, 700).tolist(), Hq=4, Hkv=2, D=64).check()


@pytest.mark.parametrize("Hq,Hkv,nodes", [(1500, 500, [70, 9, 0]), (600, 600, [300, 1, 40]), (2100, 2100, [2, 1, 3])])
def test_many_heads(Hq, Hkv, nodes):
    """Shares of the work that begin at any head, and at any unit of one"""
    Step([150, 3, 40], nodes, Hq=Hq, Hkv=Hkv, D=64, dtype=BF16).check()


def test_many_sequences_of_many_rows():
    r = np.random.RandomState(5)
    Step(r.randint(0, 900, 45).tolist(), r.randint(0, 61, 45).tolist(), Hq=24, Hkv=4, kind="any", host=(1,)).check()


def test_one_long_sequence():
    Step([70000], [24], Hq=16, Hkv=2, P=64, dtype=BF16).check()


def test_long_and_short_sequences():
    Step([20000, 3, 700, 9000, 0, 64], [3, 50, 1, 17, 2, 128], Hq=8, Hkv=1, P=32).check()


def test_pages_out_of_the_pool_are_left_out():
    s = Step([100, 60], [5, 20], kind="chain")
    s.table[0, 2] = s.desc.num_pages
    s.table[1, 4] = -1                                                      # positions 64 .. 79: tokens 4 .. 19
    drop = [(0, t) for t in range(32, 48)] + [(1, t) for t in range(64, 80)]
    s.call()
    torch.cuda.synchronize()
    assert int(s.status) == hg.HG_DEV_BAD_PAGE
    s.table[0, 2], s.table[1, 4] = 0, 0                                     # (any page: what it holds is dropped)
    out, lse, off = s.exact(drop)
    worst = (s.out[:25].double() - out).abs().nan_to_num(0) / off
    assert float((s.lse[:25].double() - lse).abs().max()) <= LOGIT and float(worst.max()) <= 1


def test_ranges_outside_are_cut():
    s = Step([64, 32], [8, 8], kind="chain", P=16)                          # rows of the table: 5 pages
    s.seq_lens = ints([76, -5])                                             # 76 + 8 > 80; a negative length is 0
    s.lens, s.nodes = [76, 0], [8, 8]
    s.call()
    torch.cuda.synchronize()
    assert int(s.status) == hg.HG_DEV_RANGE
    s.status.zero_()
    for cu in ([0, 8, 500], [-3, 8, 16], [0, 9, 9]):                        # rows beyond N, in front of 0, more than max_nodes
        s.out.fill_(-77)
        s.tree = hg.tree_desc(cu_nodes=ints(cu), num_rows=s.N, max_nodes=8)
        s.call()
        torch.cuda.synchronize()
        assert int(s.status) == hg.HG_DEV_RANGE
        s.status.zero_()


@pytest.mark.parametrize("Hq,Hkv", [(8, 2), (8, 1)])                          # 32 and 64 rows a KV head
@pytest.mark.parametrize("lens", [[76, -5], [80, 3], [100, 24]])
def test_results_of_what_is_cut(Hq, Hkv, lens):
    """Rows of the block table end at position 80: what lies behind is left out, whole rows that do not fit are left alone"""
    s = Step([72, 72], [8, 8], kind="chain", P=16, Hq=Hq, Hkv=Hkv)
    for x in (s.k, s.v):
        x.nan_to_num_(0.5, 0.5, 0.5)
    s.seq_lens, s.lens = ints(lens), [max(t, 0) for t in lens]
    narrow = s.table
    s.table = torch.cat([narrow, narrow], 1)                                # (any page behind the end: what it holds is dropped)
    drop = [(b, t) for b in range(2) for t in range(80, s.lens[b] + 8)]
    out, lse, off = s.exact(drop)
    s.table = narrow
    for cu, rows in ([0, 8, 16], range(16)), ([0, 8, 500], range(16)), ([-3, 8, 16], range(8, 16)), ([0, 9, 9], range(8)), ([3, 11, 11], range(3, 11)):
        s.out.fill_(-77)
        s.lse.fill_(-77)
        s.status.zero_()
        s.tree = hg.tree_desc(cu_nodes=ints(cu), num_rows=s.N, max_nodes=8)
        s.call()
        torch.cuda.synchronize()
        rows = list(rows)
        others = [r for r in range(s.N) if r not in rows]
        assert (s.out[others] == -77).all() and (s.lse[others] == -77).all()
        assert int(s.status) == hg.HG_DEV_RANGE                             # (sequence 0 passes the end, or cu is cut)
        if cu[0] == 3:                                                      # other queries: only that they are results
            assert torch.isfinite(s.out[rows]).all() and (s.lse[rows] != -77).all()
            continue
        assert float(((s.out[rows].double() - out[rows]).abs() / off[rows]).max()) <= 1
        assert float((s.lse[rows].double() - lse[rows]).abs().max()) <= LOGIT


def test_no_tokens_at_all():
    s = Step([10, 20], [0, 0], pad=4, max_nodes=5)
    s.check()


def test_results_do_not_change_from_call_to_call():
    s = Step([5000, 333, 12], [17, 40, 1], host=(2,), Hq=16, Hkv=2)
    s.call()
    torch.cuda.synchronize()
    out, lse = s.out.clone(), s.lse.clone()
    for i in range(5):
        s.ws.fill_(17 * i)
        s.out.fill_(-77)
        s.call()
        torch.cuda.synchronize()
        assert torch.equal(s.out, out) and torch.equal(s.lse, lse)


@pytest.mark.parametrize("lens,nodes", [([5000], [9]), ([2000, 700, 3], [40, 1, 17]), ([300] * 32, [4] * 32), ([260] * 33, [3] * 33)])
def test_calls_behind_one_another_in_one_workspace(lens, nodes):
    """Each call finds the flags and descriptions of another one's cut units, with up to 32 sequences and with more"""
    a, b = Step(lens, nodes, Hq=16), Step([1500, 40, 900], [5, 70, 1], Hq=4, Hkv=4, seed=1)
    a.check()
    b.check()
    size = max(a.ws.numel(), b.ws.numel())
    ws = torch.full((size,), 1, dtype=torch.uint8, device=DEV)
    results = [[(torch.full_like(s.out, -77), torch.full_like(s.lse, -77)) for s in (a, b)] for _ in range(40)]
    for pair in results:
        for s, (out, lse) in zip((a, b), pair):
            s.call(out=out, lse=lse, ws=ws)
    torch.cuda.synchronize()
    for pair in results:
        for s, (out, lse) in zip((a, b), pair):
            assert torch.equal(out, s.out) and torch.equal(lse, s.lse)


def test_two_streams_and_a_captured_call():
    a, b = Step([3000, 40], [9, 3], seed=1, Hq=16), Step([100, 2500, 7], [30, 2, 5], seed=2, dtype=BF16)
    a.call()
    b.call()
    torch.cuda.synchronize()
    want = [a.out.clone(), b.out.clone()]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    graphs = []
    for s, st in zip((a, b), streams):
        s.out.fill_(-77)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            s.call(stream=st)
        graphs.append(g)
    for _ in range(20):
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        a.call()
        torch.cuda.synchronize()
        assert torch.equal(a.out, want[0]) and torch.equal(b.out, want[1])
    a.seq_lens.copy_(ints([2900, 40]))                                      # lengths are read when the graph runs
    a.lens[0] = 2900
    b.out.fill_(-77)
    for g in graphs:
        g.replay()
    torch.cuda.synchronize()
    assert not torch.equal(a.out, want[0]) and torch.equal(b.out, want[1])


def test_without_lse():
    s = Step([200], [5])
    s.call()
    torch.cuda.synchronize()
    want = s.out.clone()
    s.out.fill_(-77)
    s.call(lse=None)
    torch.cuda.synchronize()
    assert torch.equal(s.out, want)


def test_offsets_beyond_32_bits():
    """A pool whose pages lie 2^28 elements apart: the last at 2.4e9 elements"""
    s = Step([120], [6], Hq=4, Hkv=2, D=64)
    far = torch.empty(9 * (1 << 28) + (1 << 16), dtype=F16, device=DEV)
    n = s.table.shape[1]
    pages = s.table[0].long()
    big = far[:9 * (1 << 28)].view(9, -1)[:, :2 * 16 * 64].view(9, 2, 16, 64)
    order = torch.randperm(9, device=DEV)[:n]
    order[-1] = 8
    order[:-1] = torch.randperm(8, device=DEV)[:n - 1]
    ks, vs = s.k[pages].clone(), s.v[pages].clone()
    s.k = big
    s.k[order] = ks
    far_v = torch.empty_like(far)
    s.v = far_v[:9 * (1 << 28)].view(9, -1)[:, :2 * 16 * 64].view(9, 2, 16, 64)
    s.v[order] = vs
    s.table[0] = order.int()
    s.desc.num_pages, s.desc.page_stride, s.desc.head_stride, s.desc.tok_stride = 9, s.k.stride(0), s.k.stride(1), s.k.stride(2)
    s.check()


def test_a_wait_that_runs_out_is_reported():
    s = Step([500, 90], [6, 40], flags=hg.HG_FLAG_TEST_STALL)
    s.call()
    torch.cuda.synchronize()
    assert int(s.status) & hg.HG_DEV_WAIT_TIMEOUT
    s.desc.flags = 0
    s.call()                                                                # skipped while the word is set
    torch.cuda.synchronize()
    s.status.zero_()
    s.check()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("nodes", [[4, 3], [8, 5]])                          # 16 and 32 rows a KV head
def test_a_wait_that_runs_out_with_few_rows(D, nodes):
    """The forms whose CTAs have sixteen warps: all of them take part in the unwinding, and the call returns normally"""
    s = Step([500, 90], nodes, D=D, flags=hg.HG_FLAG_TEST_STALL)
    s.call()
    torch.cuda.synchronize()
    assert int(s.status) & hg.HG_DEV_WAIT_TIMEOUT
    s.desc.flags = 0
    s.status.zero_()
    s.check()


def test_the_binding_refuses_wrong_tensors():
    s = Step([20], [3])
    ok = dict(q=s.q, out=s.out, lse=s.lse, ws=s.ws, host=[])

    def call(**over):
        a = dict(ok, **over)
        hg.hg_attn_decode_tree(a["q"], s.k, s.v, s.seq_lens, None, a["host"], a["out"], a["lse"], a["ws"], s.desc, s.tree)

    call()
    for over in (dict(q=s.q.float()), dict(q=s.q[:2]), dict(q=s.q.transpose(0, 1)), dict(q=s.q.cpu()), dict(out=s.out[:2]), dict(out=s.out.float()),
                 dict(lse=s.lse[:2]), dict(host=[(torch.zeros(2, 8, 1, 128, device=DEV), *[torch.zeros(2, 8, 1, device=DEV)] * 2)])):
        with pytest.raises(ValueError):
            call(**over)
    with pytest.raises(pkg.HgError):
        call(ws=s.ws[:0] if s.ws.numel() == 0 else s.ws[256:][:0])
    torch.cuda.synchronize()
