"""The operators on a step's new tokens without a GPU: struct layouts, refusals, frequencies of rotary positions."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import paper_2604_18529_b200 as pkg
from paper_2604_18529_b200 import binding as hg
from paper_2604_18529_b200 import build as hgbuild
from test_abi_cpu import FAKE, good_desc

INVALID, UNSUPPORTED = hg.HG_ERR_INVALID_ARG, hg.HG_ERR_UNSUPPORTED


@pytest.fixture(scope="module")
def lib():
    hgbuild.build()
    return hg.lib()


def offsets(struct):
    return {n: getattr(struct, n).offset for n, _ in struct._fields_}


def test_structs_match_the_c_layout():
    assert offsets(hg.HgTreeDesc) == dict(struct_size=0, max_nodes=4, num_rows=8, mask_words=12, cu_nodes=16, mask=24, q_stride=32)
    assert C.sizeof(hg.HgTreeDesc) == 40
    assert offsets(hg.HgRopeDesc) == dict(struct_size=0, num_rows=4, rot_dim=8, layout=12, freq=16, magnitude=24, flags=28, q_stride=32,
                                          q_out_stride=40, k_stride=48, v_stride=56)
    assert C.sizeof(hg.HgRopeDesc) == 64
    assert offsets(hg.HgRopeScaling) == dict(struct_size=0, kind=4, theta=8, factor=16, low=24, high=32, context=40)


def tree(**over):
    x = hg.HgTreeDesc()
    x.struct_size, x.max_nodes, x.num_rows, x.mask_words, x.cu_nodes, x.mask = C.sizeof(hg.HgTreeDesc), 40, 64, 2, FAKE, FAKE
    for n, v in over.items():
        setattr(x, n, v)
    return x


def tabled():
    d = good_desc()
    d.block_table = FAKE + (20 << 24)
    return d


def rope(**over):
    x = hg.HgRopeDesc()
    x.struct_size, x.num_rows, x.rot_dim, x.freq = C.sizeof(hg.HgRopeDesc), 5, 128, FAKE
    for n, v in over.items():
        setattr(x, n, v)
    return x


def decode(lib, d, x, src=None, n=0, ws=FAKE, size=1 << 40, **over):
    a = dict(q=FAKE, k=FAKE, v=FAKE, lens=FAKE, begin=FAKE, out=FAKE + (1 << 24))
    a.update(over)
    return lib.hg_attn_decode_tree(a["q"], a["k"], a["v"], a["lens"], a["begin"], src, n, a["out"], FAKE, ws, size, None,
                                   d and C.byref(d), x and C.byref(x))


@pytest.mark.parametrize("over,want", [
    (dict(max_nodes=0), INVALID), (dict(max_nodes=1025, mask=None), UNSUPPORTED), (dict(max_nodes=65), INVALID), (dict(num_rows=0), INVALID),
    (dict(mask_words=1), INVALID), (dict(cu_nodes=None), INVALID), (dict(q_stride=1028), INVALID), (dict(q_stride=1016), INVALID),
    (dict(q_stride=-1024), INVALID), (dict(struct_size=32), INVALID), (dict(num_rows=1 << 29), UNSUPPORTED)])
def test_bad_trees_are_refused(lib, over, want):
    d, x = good_desc(), tree(**over)
    assert decode(lib, d, x) == want
    assert lib.hg_attn_tree_workspace_bytes(C.byref(d), C.byref(x)) == 0


def test_tree_attention_refuses_what_it_cannot_run(lib):
    x = tree()
    for over, want in ((dict(batch=0), INVALID), (dict(head_dim=96), UNSUPPORTED), (dict(page_size=8), UNSUPPORTED), (dict(tok_stride=132), INVALID),
                       (dict(num_q_heads=516), UNSUPPORTED), (dict(num_q_heads=7), INVALID),
                       (dict(page_size=256, chunk_tokens=256, max_pages=1 << 24, num_pages=1 << 30), UNSUPPORTED)):
        assert decode(lib, good_desc(**over), x) == want, over
    d = good_desc()
    assert decode(lib, None, x) == INVALID and decode(lib, d, None) == INVALID
    for name in ("q", "k", "v", "lens", "out"):
        assert decode(lib, d, x, **{name: None}) == INVALID, name
    for name in ("q", "k", "v", "out"):
        assert decode(lib, d, x, **{name: FAKE + 8}) == INVALID, name
    need = lib.hg_attn_tree_workspace_bytes(C.byref(d), C.byref(x))
    assert need > 0
    assert decode(lib, d, x, size=need - 1) == hg.HG_ERR_WORKSPACE
    assert decode(lib, d, x, ws=None) == INVALID and decode(lib, d, x, ws=FAKE + 16) == INVALID
    # the result in the queries' place: rows of other CTAs' queries would be overwritten before they are read
    assert decode(lib, d, x, out=FAKE) == INVALID and decode(lib, d, x, q=FAKE + (1 << 24) + 16) == INVALID
    assert decode(lib, d, tree(q_stride=4096), out=FAKE + (63 * 4096 + d.num_q_heads * d.head_dim) * 2 - 16) == INVALID
    src = (hg.HgPartialSrc * 9)()
    for s in src:
        s.o, s.m, s.l, s.nc = FAKE, FAKE, FAKE, 1
    assert decode(lib, d, x, src, 9) == INVALID and decode(lib, d, x, src, -1) == INVALID and decode(lib, d, x, None, 1) == INVALID
    for name, bad in (("o", None), ("m", None), ("l", None), ("nc", 0), ("o", FAKE + 4)):
        was = getattr(src[1], name)
        setattr(src[1], name, bad)
        assert decode(lib, d, x, src, 2) == INVALID, name
        setattr(src[1], name, was)


class OnDevice:
    """What the binding looks at of a CUDA tensor, on a device of the test's choice"""

    def __init__(self, shape, dtype, device=0):
        self.shape, self.dtype, self.device, self.is_cuda = torch.Size(shape), dtype, torch.device("cuda", device), True

    numel = lambda self: math.prod(self.shape)
    dim = lambda self: len(self.shape)
    stride = lambda self, i=None: torch.empty(self.shape, device="meta").stride(i) if i is not None else torch.empty(self.shape, device="meta").stride()
    is_contiguous = lambda self: True
    data_ptr = lambda self: FAKE
    element_size = lambda self: self.dtype.itemsize


@pytest.mark.parametrize("which", ["q", "k", "v", "lens", "begin", "o", "m", "l", "out", "lse", "ws", "cu", "mask"])
def test_tree_attention_refuses_tensors_of_another_device(lib, monkeypatch, which):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    f16, f32, i32, N, d = torch.float16, torch.float32, torch.int32, 64, good_desc()
    shapes = dict(q=((N, 8, 128), f16), k=((64, 2, 16, 128), f16), v=((64, 2, 16, 128), f16), lens=((2,), i32), begin=((2,), i32),
                  o=((N, 8, 1, 128), f32), m=((N, 8, 1), f32), l=((N, 8, 1), f32), out=((N, 8, 128), f16), lse=((N, 8), f32),
                  ws=((1 << 26,), torch.uint8), cu=((3,), i32), mask=((N, 2), i32))

    def marshal(away):
        t = {n: OnDevice(*x, device=int(n == away)) for n, x in shapes.items()}
        x = hg.tree_desc(cu_nodes=t["cu"], mask=t["mask"], num_rows=N, max_nodes=40)
        return hg._decode_tree_args(t["q"], t["k"], t["v"], t["lens"], t["begin"], [(t["o"], t["m"], t["l"])], t["out"], t["lse"], t["ws"], d, x, 0)

    marshal(None)
    with pytest.raises(ValueError, match="cuda:1"):
        marshal(which)


def test_slots_refuse_bad_arguments(lib):
    far = [FAKE + (i << 24) for i in range(8)]
    names = ("lens", "n_new", "parent", "cu", "seq", "pos", "slot", "mask")

    def call(d=None, rows=100, words=2, **over):
        a = dict(zip(names, far))
        a.update(over)
        d = d or good_desc()
        return lib.hg_kv_slots(a["lens"], a["n_new"], a["parent"], rows, a["cu"], a["seq"], a["pos"], a["slot"], a["mask"], words, None, C.byref(d))

    assert call(lens=None) == INVALID and call(cu=None) == INVALID and call(rows=0) == INVALID and call(words=0) == INVALID
    assert call(words=33) == UNSUPPORTED and call(slot=far[6] + 4) == INVALID and call(d=good_desc(page_size=24)) == UNSUPPORTED
    assert lib.hg_kv_slots(far[0], None, None, 1, far[3], None, None, None, None, 0, None, None) == INVALID
    # outputs that overlap one another or an input: the last element of one is the first of the other
    assert call(seq=far[3] + 8) == INVALID and call(pos=far[4] + 396) == INVALID and call(slot=far[5] + 392) == INVALID
    assert call(mask=far[6] + 796) == INVALID and call(cu=far[0] + 4) == INVALID and call(seq=far[2]) == INVALID
    assert call(d=tabled(), pos=tabled().block_table) == INVALID


def test_slots_with_ready_counts_refuse_bad_arguments(lib):
    far = [FAKE + (i << 24) for i in range(9)]
    names = ("lens", "n_new", "parent", "cu", "seq", "pos", "slot", "mask", "ready")

    def call(d=None, rows=100, words=2, **over):
        a = dict(zip(names, far))
        a.update(over)
        d = d or good_desc()
        return lib.hg_kv_slots_ready(a["lens"], a["n_new"], a["ready"], a["parent"], rows, a["cu"], a["seq"], a["pos"], a["slot"], a["mask"],
                                     words, None, C.byref(d))

    assert call(lens=None) == INVALID and call(cu=None) == INVALID and call(rows=0) == INVALID and call(words=0) == INVALID
    assert call(words=33) == UNSUPPORTED and call(slot=far[6] + 4) == INVALID and call(d=good_desc(page_size=24)) == UNSUPPORTED
    # outputs in the counts' place
    for name in ("cu", "seq", "pos", "slot", "mask"):
        assert call(**{name: far[8]}) == INVALID, name
    assert call(cu=far[8] + 4) == INVALID and call(d=tabled(), pos=tabled().block_table) == INVALID


def test_rope_refuses_bad_arguments(lib):
    far = [FAKE + (i << 24) for i in range(4)]

    def plain(r=None, x=FAKE, y=far[1], pos=FAKE, heads=4, dim=128, dtype=0):
        return lib.hg_rope(x, y, pos, heads, dim, dtype, None, C.byref(r or rope()))

    def append(r=None, d=None, **over):
        a = dict(q=FAKE, k=far[1], v=far[2], pos=FAKE, slot=FAKE, out=far[3], kc=FAKE, vc=FAKE)
        a.update(over)
        d = d or good_desc()
        return lib.hg_kv_append_rope(a["q"], a["k"], a["v"], a["pos"], a["slot"], a["out"], a["kc"], a["vc"], None, C.byref(d), C.byref(r or rope()))

    for over, want in ((dict(num_rows=0), INVALID), (dict(rot_dim=0), INVALID), (dict(rot_dim=144), INVALID), (dict(rot_dim=24), UNSUPPORTED),
                       (dict(layout=2), INVALID), (dict(freq=None), INVALID), (dict(freq=FAKE + 4), INVALID), (dict(magnitude=math.inf), INVALID),
                       (dict(magnitude=math.nan), INVALID), (dict(flags=2), INVALID), (dict(q_stride=1020), INVALID), (dict(q_stride=504), INVALID),
                       (dict(q_out_stride=504), INVALID), (dict(struct_size=56), INVALID)):
        assert plain(rope(**over)) == want, over
        assert append(rope(**over)) == want, over
    assert append(rope(k_stride=248)) == INVALID and append(rope(v_stride=-8)) == INVALID
    for name in ("x", "y", "pos"):
        assert plain(**{name: None}) == INVALID
    assert plain(x=FAKE + 8) == INVALID and plain(y=FAKE + 8) == INVALID and plain(heads=0) == INVALID and plain(dtype=2) == INVALID
    assert plain(dim=96) == UNSUPPORTED and plain(dim=0) == INVALID
    assert plain(y=FAKE, r=rope(q_out_stride=1024)) == INVALID                       # in place, but with other strides
    # outputs that overlap an input: five rows of 4 heads of 128 components; the last 16 bytes of one, and rows 1536 elements apart
    assert plain(y=FAKE + 5 * 1024 - 16) == INVALID and plain(x=far[1] + 5 * 1024 - 16) == INVALID
    assert plain(rope(q_stride=1536, q_out_stride=1536), y=FAKE + 1008) == INVALID and plain(rope(q_stride=1536, q_out_stride=1536), y=FAKE + 2064) == INVALID
    assert plain(rope(q_stride=1536), y=FAKE + 1024) == INVALID
    for name in ("k", "v", "pos", "slot", "kc", "vc", "q", "out"):
        assert append(**{name: None}) == INVALID, name
    for name in ("k", "v", "kc", "vc", "q", "out"):
        assert append(**{name: FAKE + 8}) == INVALID, name
    assert append(slot=FAKE + 4) == INVALID and append(d=good_desc(head_dim=96)) == UNSUPPORTED
    assert append(out=far[1]) == INVALID and append(out=far[2]) == INVALID and append(out=FAKE + 16) == INVALID
    assert append(rope(q_out_stride=4096), out=FAKE) == INVALID
    assert append(rope(q_stride=1536, q_out_stride=1536, k_stride=1536), out=FAKE, k=FAKE + 1008) == INVALID
    assert lib.hg_rope(FAKE, FAKE, FAKE, 4, 128, 0, None, None) == INVALID


def test_accept_refuses_bad_arguments(lib):
    far = [FAKE + (i << 24) for i in range(4)]

    def call(most=4, d=None, path=far[0], n=far[1], lens=far[2], new=far[3], k=FAKE, v=FAKE):
        d = d or good_desc()
        return lib.hg_kv_accept(path, n, most, lens, new, k, v, None, C.byref(d))

    for name in ("path", "n", "lens", "k", "v"):
        assert call(**{name: None}) == INVALID
    assert call(0) == INVALID and call(1025) == UNSUPPORTED and call(k=FAKE + 8) == INVALID and call(v=FAKE + 8) == INVALID
    assert call(new=far[2] + 4) == INVALID and call(new=far[1]) == INVALID and call(new=far[0] + 28) == INVALID
    assert call(d=tabled(), new=tabled().block_table) == INVALID and call(d=good_desc(page_size=8)) == UNSUPPORTED


# ---- frequencies: against the formulas as the methods' authors state them ------------------------------------------------------

def test_plain_linear_and_base_frequencies():
    i = np.arange(64)
    f, m = pkg.hg_rope_frequencies(128, 10000.0)
    assert m == 1.0 and np.allclose(f.numpy(), 10000.0 ** (-i / 64), rtol=1e-14, atol=0)
    assert np.allclose(pkg.hg_rope_frequencies(128, 10000.0, "linear", 4.0)[0].numpy(), f.numpy() / 4, rtol=1e-14, atol=0)
    b = pkg.hg_rope_frequencies(128, 10000.0, "base", 8.0)[0].numpy()
    assert b[0] == 1.0 and math.isclose(b[-1], f[-1] / 8, rel_tol=1e-13)
    assert np.allclose(b, (10000.0 * 8 ** (128 / 126)) ** (-i / 64), rtol=1e-13, atol=0)
    assert pkg.hg_rope_frequencies(2, 10000.0, "base", 8.0)[0].tolist() == [1.0]


def test_frequencies_blended_by_turns():
    f, m = pkg.hg_rope_frequencies(128, 500000.0, "turns", 8.0, 1.0, 4.0, 8192)
    plain = 500000.0 ** (-np.arange(64) / 64)
    wave = 2 * np.pi / plain
    smooth = (8192 / wave - 1.0) / (4.0 - 1.0)
    want = np.where(wave < 8192 / 4.0, plain, np.where(wave > 8192 / 1.0, plain / 8, (1 - smooth) * plain / 8 + smooth * plain))
    assert m == 1.0 and np.allclose(f.numpy(), want, rtol=1e-13, atol=0)
    assert (f.numpy() == plain).any() and np.isclose(f.numpy(), plain / 8, rtol=1e-13).any()


def test_frequencies_blended_by_index():
    f, m = pkg.hg_rope_frequencies(128, 10000.0, "index", 16.0, 1.0, 32.0, 4096)
    plain = 10000.0 ** (-np.arange(64) / 64)
    lo = math.floor(128 * math.log(4096 / (32 * 2 * math.pi)) / (2 * math.log(10000.0)))
    hi = math.ceil(128 * math.log(4096 / (1 * 2 * math.pi)) / (2 * math.log(10000.0)))
    ramp = np.clip((np.arange(64) - lo) / (hi - lo), 0, 1)
    assert np.allclose(f.numpy(), plain / 16 * ramp + plain * (1 - ramp), rtol=1e-13, atol=0)
    assert math.isclose(m, 0.1 * math.log(16.0) + 1, rel_tol=1e-7)
    one, m = pkg.hg_rope_frequencies(64, 10000.0, "index", 1.0, 1.0, 32.0, 4096)
    assert np.allclose(one.numpy(), 10000.0 ** (-np.arange(32) / 32), rtol=1e-14, atol=0) and m == 1.0


@pytest.mark.parametrize("args", [(0,), (7,), (64, 1.0), (64, math.inf), (64, 10.0, "linear", 0.5), (64, 10.0, "linear", math.nan),
                                  (64, 10.0, "turns", 2.0, 0.0, 4.0, 100.0), (64, 10.0, "turns", 2.0, 4.0, 4.0, 100.0),
                                  (64, 10.0, "index", 2.0, 1.0, 4.0, 0.0), (64, 10.0, "index", 2.0, 1.0, math.inf, 100.0)])
def test_bad_scalings_are_refused(args):
    with pytest.raises(pkg.HgError):
        pkg.hg_rope_frequencies(*args)
