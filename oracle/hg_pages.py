"""CPU oracle of the page operations (hg_kv_fork, hg_kv_reserve, hg_kv_release, hg_kv_compact, hg_kv_copy_pages).

Plain lists, one step after the other, nothing shared with the CUDA library.  A pool's state is the block table (rows of
page ids, -1 where nothing is mapped) and the pages' reference counts.
"""

BAD_PAGE, RANGE, NO_PAGE = 2, 4, 8


def fork(table, ref, src_row, *vectors):
    """Rows take the pages of the rows they name, as these were before the call; returns the status bits."""
    status, B, n = 0, len(table), len(ref)
    old = [list(r) for r in table]
    old_vec = [list(v) for v in vectors]
    for b, s in enumerate(src_row):
        if s >= B:
            status |= RANGE
            continue
        if s == b:
            continue
        table[b] = [-1] * len(old[b]) if s < 0 else list(old[s])
        for v, o in zip(vectors, old_vec):
            v[b] = 0 if s < 0 else o[s]
        for now, was in zip(table[b], old[b]):
            if 0 <= now < n:
                ref[now] += 1
            if 0 <= was < n:
                ref[was] -= 1
    return status


def reserve(table, ref, seq_lens, n_new, page_size):
    """Serves the sequences in order, their slots in order; returns (copy_src, copy_dst, copy_rows, n_ready, status)."""
    B, S, n, status = len(table), len(table[0]), len(ref), 0
    src, dst, rows, ready = [-1] * B, [-1] * B, [0] * B, [0] * B
    for b in range(B):
        length, want = max(seq_lens[b], 0), n_new[b]
        if want <= 0:
            continue
        if length + want > S * page_size:
            status |= RANGE
            want = max(S * page_size - length, 0)
        ok, pos = True, length
        while pos < length + want:
            slot = pos // page_size
            e, here = table[b][slot], True
            if e >= n:
                status |= BAD_PAGE
                here = False
            elif e < 0 or ref[e] > 1:
                page = next((p for p in range(n) if ref[p] == 0), None)
                if page is None:
                    status |= NO_PAGE
                    here = False
                else:
                    ref[page] = 1
                    table[b][slot] = page
                    if e >= 0:
                        ref[e] -= 1
                        if pos % page_size:
                            src[b], dst[b], rows[b] = e, page, pos % page_size
            if not here and ok:
                ok = False
                ready[b] = pos - length
            pos = (slot + 1) * page_size
        if ok:
            ready[b] = want
    return src, dst, rows, ready, status


def release(ref, ids):
    status = 0
    for p in ids:
        if p < 0:
            continue
        if p >= len(ref) or ref[p] <= 0:
            status |= BAD_PAGE
        else:
            ref[p] -= 1
    return status


def compact(table, ref, max_moves):
    """Highest pages into the lowest holes; returns (pairs, remap)."""
    moves, remap = [], list(range(len(ref)))
    while len(moves) < max_moves:
        low = next((p for p in range(len(ref)) if ref[p] <= 0), len(ref))
        high = next((p for p in range(len(ref) - 1, -1, -1) if ref[p] > 0), -1)
        if low >= high:
            break
        moves.append((high, low))
        remap[high], ref[low], ref[high] = low, ref[high], 0
    for row in table:
        row[:] = [remap[e] if 0 <= e < len(ref) else e for e in row]
    return moves, remap


def copy_pages(pool, src, dst, rows, n_pages, page_axis_rows):
    """pool: a mapping page -> list of token rows (mutable); copies the first rows[i] rows of src[i] to dst[i]."""
    status = 0
    for i, (s, d) in enumerate(zip(src, dst)):
        if s < 0 or d < 0:
            continue
        if s >= n_pages or d >= n_pages:
            status |= BAD_PAGE
            continue
        m = page_axis_rows if rows is None else max(0, min(rows[i], page_axis_rows))
        for t in range(m):
            pool[d][t] = pool[s][t]
    return status
