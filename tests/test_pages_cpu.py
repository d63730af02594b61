"""The page operations without a GPU: the oracle against hand-worked cases and invariants, and the library's refusals."""
import ctypes as C
import random

import pytest

from oracle import hg_pages as O
from paper_2604_18529_b200 import binding as hg
from paper_2604_18529_b200 import build as hgbuild
from test_abi_cpu import FAKE, good_desc


# ---- oracle ----------------------------------------------------------------------------------------------------------

def test_oracle_fork_swaps_frees_and_shares():
    table, ref = [[0, 1], [2, -1], [3, 4]], [1, 1, 1, 1, 1, 0]
    lens, end = [5, 3, 8], [5, 2, 8]
    assert O.fork(table, ref, [1, 0, 0], lens, end) == 0
    assert table == [[2, -1], [0, 1], [0, 1]] and ref == [2, 2, 1, 0, 0, 0]
    assert lens == [3, 5, 5] and end == [2, 5, 5]
    assert O.fork(table, ref, [0, -1, 9], lens) == O.RANGE
    assert table == [[2, -1], [-1, -1], [0, 1]] and ref == [1, 1, 1, 0, 0, 0] and lens == [3, 0, 5]


def test_oracle_reserve_last_writer_keeps_the_page():
    table, ref = [[0, 1], [0, 1], [0, 1]], [3, 3, 0, 0, 0]
    src, dst, rows, ready, status = O.reserve(table, ref, [20, 20, 20], [1, 1, 1], 16)
    assert table == [[0, 2], [0, 3], [0, 1]] and ref == [3, 1, 1, 1, 0] and status == 0
    assert (src, dst, rows, ready) == ([1, 1, -1], [2, 3, -1], [4, 4, 0], [1, 1, 1])


def test_oracle_reserve_somebody_else_still_reads():
    table, ref = [[0], [0], [0]], [3, 0, 0]
    src, dst, _, ready, _ = O.reserve(table, ref, [3, 3, 3], [1, 0, 1], 16)
    assert table == [[1], [0], [2]] and ref == [1, 1, 1] and src == [0, -1, 0] and dst == [1, -1, 2] and ready == [1, 0, 1]


def test_oracle_reserve_out_of_pages_and_end_of_row():
    table, ref = [[0, -1], [0, -1]], [2, 0]
    src, dst, rows, ready, status = O.reserve(table, ref, [16, 16], [20, 1], 16)
    assert table == [[0, 1], [0, -1]] and ready == [16, 0] and status == O.RANGE | O.NO_PAGE and src == [-1, -1]
    table, ref = [[0], [0]], [2, 1]                  # nobody gets a copy: nobody may write
    _, _, _, ready, status = O.reserve(table, ref, [3, 3], [1, 1], 16)
    assert table == [[0], [0]] and ref == [2, 1] and ready == [0, 0] and status == O.NO_PAGE


def test_oracle_compact_and_release():
    table, ref = [[5, 2], [5, -1], [9, 9]], [0, 0, 1, 0, 0, 2]
    assert O.compact(table, ref, 1) == ([(5, 0)], [0, 1, 2, 3, 4, 0])
    assert table == [[0, 2], [0, -1], [9, 9]] and ref == [2, 0, 1, 0, 0, 0]
    assert O.compact(table, ref, 9)[0] == [(2, 1)] and ref == [2, 1, 0, 0, 0, 0]
    assert O.release(ref, [0, -1, 0, 1]) == 0 and ref == [0] * 6
    assert O.release(ref, [1, 6]) == O.BAD_PAGE and ref == [0] * 6


def test_oracle_invariants_over_random_histories():
    """Counts equal the table's entries, no page is written by two rows, tokens survive forks, copies and moves."""
    r = random.Random(5)
    for _ in range(60):
        B, S, P, n = r.randint(1, 6), r.randint(1, 5), 4, r.randint(3, 25)
        table, ref, lens = [[-1] * S for _ in range(B)], [0] * n, [0] * B
        said = [[] for _ in range(B)]                 # what each row should hold
        pool = [[None] * P for _ in range(n)]
        for step in range(12):
            src = [r.randrange(-1, B) if r.random() < 0.3 else b for b in range(B)]
            O.fork(table, ref, src, lens)
            said = [list(said[s]) if s >= 0 else [] for s in src]
            new = [r.randint(0, 7) for _ in range(B)]
            cs, cd, rows, ready, _ = O.reserve(table, ref, lens, new, P)
            O.copy_pages(pool, cs, cd, rows, n, P)
            for b in range(B):
                for _ in range(ready[b]):
                    e = table[b][lens[b] // P]
                    assert ref[e] == 1
                    pool[e][lens[b] % P] = (step, b, lens[b])
                    said[b].append((step, b, lens[b]))
                    lens[b] += 1
            if r.random() < 0.5:
                moves, _ = O.compact(table, ref, r.randint(1, n))
                assert not {a for a, _ in moves} & {b for _, b in moves}
                O.copy_pages(pool, [a for a, _ in moves], [b for _, b in moves], None, n, P)
            for p in range(n):
                assert ref[p] == sum(row.count(p) for row in table)
            for b in range(B):
                assert [pool[table[b][t // P]][t % P] for t in range(lens[b])] == said[b]


# ---- refusals: nothing is launched, no pointer is read --------------------------------------------------------------------

@pytest.fixture(scope="module")
def lib():
    hgbuild.build()
    return hg.lib()


def table_desc(**over):
    d = good_desc(**over)
    d.block_table = FAKE
    return d


CALLS = {
    "hg_kv_fork": lambda L, d, a: L.hg_kv_fork(a(0), a(1), a(2), a(8), a(9), None, d),
    "hg_kv_reserve": lambda L, d, a: L.hg_kv_reserve(a(0), a(8), a(1), a(2), a(3), a(9), a(10), None, d),
    "hg_kv_release": lambda L, d, a: L.hg_kv_release(a(0), 5, a(1), None, d),
    "hg_kv_compact": lambda L, d, a: L.hg_kv_compact(a(0), a(1), a(2), a(3), 5, a(4), None, d),
    "hg_kv_copy_pages": lambda L, d, a: L.hg_kv_copy_pages(a(0), a(1), a(8), 5, a(9), a(2), a(3), None, d),
}
REQUIRED = {"hg_kv_fork": 3, "hg_kv_reserve": 4, "hg_kv_release": 2, "hg_kv_compact": 5, "hg_kv_copy_pages": 4}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_page_calls_refuse_missing_pointers_and_bad_descriptions(lib, name):
    call = CALLS[name]
    good = lambda i: FAKE   # noqa: E731
    for missing in range(REQUIRED[name]):
        d = table_desc()
        assert call(lib, C.byref(d), lambda i: None if i == missing else FAKE) == hg.HG_ERR_INVALID_ARG, missing
    assert call(lib, None, good) == hg.HG_ERR_INVALID_ARG
    for over, want in ((dict(batch=0), hg.HG_ERR_INVALID_ARG), (dict(page_size=24), hg.HG_ERR_UNSUPPORTED),
                       (dict(num_pages=0), hg.HG_ERR_INVALID_ARG), (dict(head_dim=96), hg.HG_ERR_UNSUPPORTED),
                       (dict(tok_stride=132), hg.HG_ERR_INVALID_ARG), (dict(dtype="f16", max_pages=0), hg.HG_ERR_INVALID_ARG)):
        d = table_desc(**over)
        assert call(lib, C.byref(d), good) == want, over


@pytest.mark.parametrize("name", ["hg_kv_fork", "hg_kv_reserve", "hg_kv_compact"])
def test_table_operations_refuse_identity_paging_and_huge_tables(lib, name):
    d = good_desc()
    assert CALLS[name](lib, C.byref(d), lambda i: FAKE) == hg.HG_ERR_INVALID_ARG
    d = table_desc(batch=65535, max_pages=40000, num_pages=2 ** 31 - 1)
    assert CALLS[name](lib, C.byref(d), lambda i: FAKE + 64 * i) == hg.HG_ERR_UNSUPPORTED


def test_batch_limits_alignment_and_counts(lib):
    good = lambda i: FAKE   # noqa: E731
    d = table_desc(batch=16385, max_pages=2)
    assert CALLS["hg_kv_reserve"](lib, C.byref(d), lambda i: FAKE + 64 * i) == hg.HG_ERR_UNSUPPORTED
    d = table_desc()
    assert CALLS["hg_kv_reserve"](lib, C.byref(d), lambda i: FAKE + 4 * (i == 1)) == hg.HG_ERR_INVALID_ARG
    distinct = lambda i: FAKE + 64 * i   # noqa: E731
    for same in (0, 8):                                             # n_ready is written while seq_lens and n_new are read
        assert CALLS["hg_kv_reserve"](lib, C.byref(d), lambda i: distinct(same if i == 10 else i)) == hg.HG_ERR_INVALID_ARG
    assert CALLS["hg_kv_compact"](lib, C.byref(d), lambda i: FAKE + 4 * (i == 0)) == hg.HG_ERR_INVALID_ARG
    assert CALLS["hg_kv_copy_pages"](lib, C.byref(d), lambda i: FAKE + 8 * (i == 2)) == hg.HG_ERR_INVALID_ARG
    assert lib.hg_kv_compact(FAKE, FAKE, FAKE, FAKE, 0, FAKE, None, C.byref(d)) == hg.HG_ERR_INVALID_ARG
    assert lib.hg_kv_release(FAKE, -1, FAKE, None, C.byref(d)) == hg.HG_ERR_INVALID_ARG
    assert lib.hg_kv_copy_pages(FAKE, FAKE, None, -1, None, FAKE, FAKE, None, C.byref(d)) == hg.HG_ERR_INVALID_ARG
    assert lib.hg_kv_release(FAKE, 0, FAKE, None, C.byref(d)) == hg.HG_OK           # an empty list launches nothing
    assert lib.hg_kv_copy_pages(FAKE, FAKE, None, 0, None, FAKE, FAKE, None, C.byref(d)) == hg.HG_OK


def test_fork_refuses_arrays_that_overlap(lib):
    """Whole arrays may be the same; a part of one, and the rows' sources among what is written, may not."""
    d = table_desc(batch=64)
    at = lambda **over: [over.get(n, FAKE + 4096 * i) for i, n in enumerate(("src", "ref", "lens", "begin", "end"))]   # noqa: E731
    lens = FAKE + 4096 * 2
    for over in (dict(begin=lens + 4), dict(end=lens - 4), dict(end=lens + 252), dict(begin=FAKE + 4096 * 4 + 128), dict(src=lens),
                 dict(src=lens + 128), dict(src=FAKE + 4096 * 3), dict(src=FAKE + 4096 * 4 - 252)):
        assert lib.hg_kv_fork(*at(**over), None, C.byref(d)) == hg.HG_ERR_INVALID_ARG, over


def test_reserve_refuses_to_write_what_it_reads(lib):
    d = table_desc(batch=64)
    for i in (2, 3, 9, 10):                                         # copy_src, copy_dst, copy_rows, n_ready
        for j in (0, 8):                                            # seq_lens, n_new
            for off in (0, 4, -4, 252, -252):
                at = lambda x: FAKE + 4096 * (j if x == i else x) + (off if x == i else 0)   # noqa: E731
                assert CALLS["hg_kv_reserve"](lib, C.byref(d), at) == hg.HG_ERR_INVALID_ARG, (i, j, off)


def test_binding_refuses_lists_whose_length_passes_31_bits():
    import torch
    d, few, many = good_desc(), torch.empty(4, dtype=torch.int32, device="meta"), torch.empty(2 ** 32 + 4, dtype=torch.int32, device="meta")
    assert hg._count(few, "x") == 4
    for call in (lambda: hg.hg_kv_release(many, few, d, stream=0), lambda: hg.hg_kv_compact(few, few, many, many, few, d, stream=0),
                 lambda: hg.hg_kv_copy_pages(many, many, None, None, few, few, d, stream=0)):
        with pytest.raises(ValueError, match="entries"):
            call()


@pytest.mark.parametrize("name", ["hg_kv_reserve", "hg_kv_compact"])
def test_scans_refuse_pools_whose_last_group_passes_31_bits(lib, name):
    for n in (2 ** 31 - 255, 2 ** 31 - 1):
        d = table_desc(num_pages=n)
        assert CALLS[name](lib, C.byref(d), lambda i: FAKE + (1 << 40) * i) == hg.HG_ERR_UNSUPPORTED, n


def test_binding_refuses_host_tensors():
    import torch
    t = torch.zeros(64, dtype=torch.int32)
    d = good_desc()
    for call in (lambda: hg.hg_kv_fork(t, t, t, None, None, d, stream=0),
                 lambda: hg.hg_kv_reserve(t, None, t, t, t, None, None, d, stream=0),
                 lambda: hg.hg_kv_release(t, t, d, stream=0), lambda: hg.hg_kv_compact(t, t, t, t, t, d, stream=0),
                 lambda: hg.hg_kv_copy_pages(t, t, None, None, t, t, d, stream=0)):
        with pytest.raises(ValueError):
            call()
