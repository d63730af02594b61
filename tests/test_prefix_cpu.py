"""The shared-prefix entry points without a GPU: struct layout and refusals."""
import ctypes as C

import pytest

import paper_2604_18529_b200 as pkg
from paper_2604_18529_b200 import binding as hg
from paper_2604_18529_b200 import build as hgbuild
from test_abi_cpu import FAKE, good_desc


@pytest.fixture(scope="module")
def lib():
    hgbuild.build()
    return hg.lib()


def groups(**over):
    x = hg.HgPrefixDesc()
    x.struct_size, x.num_groups, x.chunk_tokens, x.num_chunks = C.sizeof(hg.HgPrefixDesc), 3, 256, 4
    x.seq_group = x.group_row = x.group_begin = x.group_end = FAKE
    for n, v in over.items():
        setattr(x, n, v)
    return x


def test_struct_matches_the_c_layout():
    f = {n: getattr(hg.HgPrefixDesc, n).offset for n, _ in hg.HgPrefixDesc._fields_}
    assert f == dict(struct_size=0, num_groups=4, seq_group=8, group_row=16, group_begin=24, group_end=32, chunk_tokens=40, num_chunks=44)
    assert C.sizeof(hg.HgPrefixDesc) == 48


def partial(lib, d, x, **over):
    a = dict(q=FAKE, k=FAKE, v=FAKE, o=FAKE, m=FAKE, l=FAKE)
    a.update(over)
    return lib.hg_attn_prefix_partial(a["q"], a["k"], a["v"], a["o"], a["m"], a["l"], None, d, x)


@pytest.mark.parametrize("over,want", [
    (dict(num_groups=0), hg.HG_ERR_INVALID_ARG), (dict(num_groups=513), hg.HG_ERR_UNSUPPORTED),
    (dict(chunk_tokens=0), hg.HG_ERR_INVALID_ARG), (dict(chunk_tokens=64), hg.HG_ERR_UNSUPPORTED),
    (dict(chunk_tokens=200), hg.HG_ERR_UNSUPPORTED), (dict(num_chunks=0), hg.HG_ERR_INVALID_ARG),
    (dict(seq_group=None), hg.HG_ERR_INVALID_ARG), (dict(group_row=None), hg.HG_ERR_INVALID_ARG),
    (dict(group_begin=None), hg.HG_ERR_INVALID_ARG), (dict(group_end=None), hg.HG_ERR_INVALID_ARG), (dict(struct_size=40), hg.HG_ERR_INVALID_ARG)])
def test_bad_groups_are_refused(lib, over, want):
    d, x = good_desc(), groups(**over)
    assert partial(lib, C.byref(d), C.byref(x)) == want
    assert lib.hg_attn_shared_workspace_bytes(C.byref(d), C.byref(x)) == 0
    assert lib.hg_attn_decode_shared(*[FAKE] * 6, None, 0, FAKE, FAKE, FAKE, 1 << 40, None, C.byref(d), C.byref(x)) == want


def test_bad_descriptions_and_pointers_are_refused(lib):
    x = groups()
    for over, want in ((dict(batch=0), hg.HG_ERR_INVALID_ARG), (dict(head_dim=96), hg.HG_ERR_UNSUPPORTED),
                       (dict(page_size=8), hg.HG_ERR_UNSUPPORTED), (dict(tok_stride=132), hg.HG_ERR_INVALID_ARG),
                       (dict(page_size=256, chunk_tokens=256, max_pages=1 << 24, num_pages=1 << 30), hg.HG_ERR_UNSUPPORTED)):
        d = good_desc(**over)
        assert partial(lib, C.byref(d), C.byref(x)) == want, over
    d = good_desc(page_size=256, chunk_tokens=256)
    assert partial(lib, C.byref(d), C.byref(groups(chunk_tokens=128))) == hg.HG_ERR_UNSUPPORTED
    d = good_desc()
    for name in "qkvoml":
        assert partial(lib, C.byref(d), C.byref(x), **{name: None}) == hg.HG_ERR_INVALID_ARG
    for name in "qkvo":
        assert partial(lib, C.byref(d), C.byref(x), **{name: FAKE + 8}) == hg.HG_ERR_INVALID_ARG
    assert partial(lib, C.byref(d), C.byref(x), o=FAKE + 16) == hg.HG_ERR_INVALID_ARG          # rows are stored 32 bytes at a time
    assert partial(lib, None, C.byref(x)) == hg.HG_ERR_INVALID_ARG and partial(lib, C.byref(d), None) == hg.HG_ERR_INVALID_ARG


def test_the_joined_step_refuses_what_it_cannot_run(lib):
    d, x = good_desc(), groups()
    need = lib.hg_attn_shared_workspace_bytes(C.byref(d), C.byref(x))
    rows = 2 * 8
    assert need >= rows * (4 + 2) * 130 * 4 and need % 256 == 0
    src = (hg.HgPartialSrc * 8)()
    for s in src:
        s.o, s.m, s.l, s.nc = FAKE, FAKE, FAKE, 1

    def call(args=None, n=0, ws=FAKE, size=need, sources=src):
        a = [FAKE] * 6 if args is None else args
        return lib.hg_attn_decode_shared(*a, sources, n, FAKE, None, ws, size, None, C.byref(d), C.byref(x))

    assert call(size=need - 1) == hg.HG_ERR_WORKSPACE
    assert call(ws=None) == hg.HG_ERR_INVALID_ARG and call(ws=FAKE + 16) == hg.HG_ERR_INVALID_ARG
    assert call(n=7) == hg.HG_ERR_INVALID_ARG and call(n=-1) == hg.HG_ERR_INVALID_ARG and call(n=1, sources=None) == hg.HG_ERR_INVALID_ARG
    for i in range(6):
        assert call([None if j == i else FAKE for j in range(6)]) == hg.HG_ERR_INVALID_ARG
    src[1].nc = 0
    assert call(n=2) == hg.HG_ERR_INVALID_ARG
    src[1].nc, src[0].o = 1, FAKE + 4
    assert call(n=2) == hg.HG_ERR_INVALID_ARG


def test_suggested_chunks_are_legal():
    for page in (16, 32, 64, 128, 256):
        for tokens in (0, 1, 1000, 131072, 10 ** 9):
            for groups_, members in ((1, 1), (1, 128), (12, 90), (512, 512), (3, 0)):
                for hq, hkv in ((8, 8), (32, 8), (64, 8), (56, 56), (24, 1)):
                    c = pkg.hg_attn_prefix_suggest_chunk(tokens, groups_, members, hq, hkv, page)
                    assert c % 128 == 0 and c % page == 0 and c >= 128
    for bad in ((-1, 1, 1, 8, 8, 16), (10, 0, 1, 8, 8, 16), (10, 1, -1, 8, 8, 16), (10, 1, 1, 8, 3, 16), (10, 1, 1, 8, 8, 24)):
        with pytest.raises(pkg.HgError):
            pkg.hg_attn_prefix_suggest_chunk(*bad)


def test_unwinding_waits_for_the_tiles_on_their_way(tmp_path):
    """The ring arithmetic of the kernel's unwinding, compiled for the host, against random runs of its loaders."""
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    exe = str(tmp_path / "ring")
    subprocess.check_call(["g++", "-std=c++17", "-Wall", "-Werror", "-O1", os.path.join(root, "tests", "c_abi", "ring_unwind.cpp"), "-o", exe,
                           "-I", os.path.join(root, "paper_2604_18529_b200", "csrc")])
    run = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert run.returncode == 0 and "ring OK" in run.stdout, run.stderr
