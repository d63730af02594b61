"""Decode attention over a shared prefix, and the page operations that make prefixes shared: cases, plain forms, exact values.

Three passes are measured:

* ``shared``   one decode step of a batch whose sequences fall into groups with a common prefix: attention over the
               group's pages and over the sequence's own, joined into the softmax over both;
* ``branch``   one step of a branching decode (beams, parallel samples): the rows of the block table are re-assigned to
               their parents' pages, pages for the next tokens are reserved (copy on write) and the shared last pages copied;
* ``compact``  a turn-over of requests: half of the rows are freed, the pool is compacted (pages moved, tables renamed) and
               pages for the new prompts are reserved.
"""
import random

import numpy as np
import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


def _shared(name, dtype, B, Hq, Hkv, D, page, groups, prefix, own_tokens, ragged, lens_seed):
    return {"name": name, "op": "shared", "dtype": dtype, "B": B, "Hq": Hq, "Hkv": Hkv, "D": D, "page": page, "groups": groups,
            "prefix": prefix, "own_tokens": own_tokens, "ragged": ragged, "lens_seed": lens_seed}


def _branch(name, dtype, parents, children, Hkv, D, page, tokens, n_new, lens_seed):
    return {"name": name, "op": "branch", "dtype": dtype, "parents": parents, "children": children, "Hkv": Hkv, "D": D,
            "page": page, "tokens": tokens, "n_new": n_new, "lens_seed": lens_seed}


def _compact(name, dtype, B, Hkv, D, page, tokens, lens_seed):
    return {"name": name, "op": "compact", "dtype": dtype, "B": B, "Hkv": Hkv, "D": D, "page": page, "tokens": tokens,
            "lens_seed": lens_seed}


def listed():
    return [
        # four chat turns over one short system prompt: latency
        _shared("shared_small", "f16", 4, 32, 8, 128, 16, 1, 512, 32, False, 1),
        # 32 questions about one long document, Llama-70B-shaped layer, small pages
        _shared("shared_document", "f16", 32, 64, 8, 128, 16, 1, 131072, 300, False, 2),
        # one head per KV head (OPT-30B-shaped): few rows per head, bound by the cache's bytes
        _shared("shared_one_head", "bf16", 16, 56, 56, 128, 64, 1, 16384, 500, False, 3),
        # several applications' prompts of different lengths, some requests without any
        _shared("shared_ragged", "f16", 96, 32, 8, 128, 16, 12, 16384, 700, True, 4),
        # a small model with 64 components a head and many samples per prompt
        _shared("shared_d64", "bf16", 64, 8, 8, 64, 32, 2, 2048, 100, True, 5),
        # a large batch over a long prompt: bound by arithmetic
        _shared("shared_large", "bf16", 128, 64, 8, 128, 64, 1, 65536, 256, False, 6),
        # beam search of width 4 over one request: latency
        _branch("branch_beam", "f16", 1, 3, 8, 128, 16, 2000, 1, 7),
        # best-of-8 sampling of 32 requests
        _branch("branch_samples", "bf16", 32, 7, 8, 128, 16, 8000, 1, 8),
        # many branches with several new tokens each (a draft's), one head per KV head, larger pages
        _branch("branch_drafts", "f16", 64, 15, 40, 128, 64, 4000, 5, 9),
        # a small pool: latency
        _compact("compact_small", "f16", 8, 8, 64, 16, 1000, 10),
        # a pool of small pages
        _compact("compact_pages16", "f16", 64, 8, 128, 16, 8000, 11),
        # a pool of some gigabytes with larger pages
        _compact("compact_large", "bf16", 64, 40, 128, 64, 5000, 12),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    op = rng.choice(["shared", "shared", "branch", "compact"])
    dtype = rng.choice(["f16", "bf16"])
    page = rng.choice([16, 32, 64, 128])
    seed = rng.randrange(1 << 20)
    if op == "shared":
        hq, hkv, d = rng.choice([(8, 8, 64), (40, 40, 128), (56, 56, 128), (64, 8, 128), (32, 8, 128), (28, 4, 128), (20, 20, 64)])
        b = _log_int(rng, 1, 128)
        groups = _log_int(rng, 1, max(1, b // 2))
        own_tokens = _log_int(rng, 1, 600)
        # no costlier than the largest listed cases: the cells of the logits, the elements of the cache
        prefix = min(_log_int(rng, 1, 131072), 65536 * 128 * 64 // (b * hq * (2 if groups > 1 else 1)), (1 << 27) // (hkv * d * groups))
        own_tokens = min(own_tokens, (1 << 27) // (b * hkv * d))
        return _shared("shared", dtype, b, hq, hkv, d, page, groups, max(1, prefix), own_tokens, rng.random() < 0.6, seed)
    hkv, d = rng.choice([(8, 64), (8, 128), (40, 128), (20, 64), (4, 128), (1, 128)])
    if op == "branch":
        parents, children = _log_int(rng, 1, 64), rng.randint(1, 15)
        tokens = _log_int(rng, 17, 8000)
        tokens = max(17, min(tokens, 64 * 4000 * 40 * 128 // (parents * hkv * d)))
        return _branch("branch", dtype, parents, children, hkv, d, page, tokens, _log_int(rng, 1, 40), seed)
    b = _log_int(rng, 2, 64)
    tokens = max(17, min(_log_int(rng, 17, 16000), 64 * 5000 * 40 * 128 // (b * hkv * d)))
    return _compact("compact", dtype, b, hkv, d, page, tokens, seed)


# ---- lengths: from the case alone, so that its work is known ---------------------------------------------------------

def _shared_plan(c):
    """(group of every sequence or -1, group lengths, own lengths)"""
    r = random.Random(c["lens_seed"])
    B, NG = c["B"], c["groups"]
    if not c["ragged"]:
        return [b % NG for b in range(B)], [c["prefix"]] * NG, [c["own_tokens"]] * B
    group = list(range(NG)) + [r.randrange(NG) if r.random() < 0.9 else -1 for _ in range(B - NG)]
    r.shuffle(group)
    lens = [c["prefix"]] + [r.randint(1, c["prefix"]) for _ in range(NG - 1)]
    return group, lens, [r.randint(1, c["own_tokens"]) for _ in range(B)]


def _row_lens(c, n):
    r = random.Random(c["lens_seed"])
    return [r.randint(max(1, c["tokens"] // 2), c["tokens"]) for _ in range(n)]


def _pages(n, page):
    return -(-n // page)


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(shape, dtype, g):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dtype) if np.prod(shape) < 1 << 28 else \
        torch.randn(shape, generator=g, device="cuda", dtype=dtype)


def _ints(a):
    return torch.as_tensor(np.asarray(a, dtype=np.int32)).cuda()


def prepare(case, seed):
    return {"shared": _prepare_shared, "branch": _prepare_branch, "compact": _prepare_compact}[case["op"]](case, seed)


def _prepare_shared(c, seed):
    """A batch in mid-decode: pools, block table (members list their group's whole pages, then pages of their own), queries."""
    group, glen, own_len = _shared_plan(c)
    P, B, NG = c["page"], c["B"], c["groups"]
    start = [glen[g] if g >= 0 else 0 for g in group]
    total = [s + n for s, n in zip(start, own_len)]
    max_pages = max([_pages(t, P) for t in total] + [_pages(n, P) for n in glen])
    n_shared = [n // P for n in glen]
    n_pages = sum(n_shared) + sum(_pages(t, P) - (n_shared[g] if g >= 0 else 0) for t, g in zip(total, group))
    ids = np.random.RandomState(seed % (1 << 32)).permutation(n_pages).astype(np.int32)
    table = np.full((B, max_pages), -1, dtype=np.int32)
    first, at = {}, 0
    for b, g in enumerate(group):
        own_from = 0
        if g >= 0:
            if g not in first:
                first[g] = (b, at)
                at += n_shared[g]
            own_from = n_shared[g]
            table[b, :own_from] = ids[first[g][1]:first[g][1] + own_from]
        n = _pages(total[b], P) - own_from
        table[b, own_from:own_from + n] = ids[at:at + n]
        at += n
    gen, dt = _generator(seed), DTYPES[c["dtype"]]
    shape = (n_pages, c["Hkv"], P, c["D"])
    return {"case": c, "q": _normal((B, c["Hq"], c["D"]), dt, gen), "k": _normal(shape, dt, gen), "v": _normal(shape, dt, gen),
            "table": _ints(table), "seq_lens": _ints(total), "tok_begin": _ints(start), "tok_end": _ints(total),
            "seq_group": _ints(group), "group_row": _ints([first[g][0] if g in first else 0 for g in range(NG)]),
            "group_begin": _ints([0] * NG), "group_end": _ints([glen[g] if g in first else 0 for g in range(NG)]),
            "n_max": max([1] + [group.count(g) for g in range(NG)]), "prefix_max": max(glen), "own_max": max(own_len),
            "shared_tokens": sum(glen), "n_members": sum(g >= 0 for g in group)}


def _pools(c, n_pages, seed):
    """One page more than the pool has: where the plain form puts what a list does not ask for."""
    gen, dt = _generator(seed), DTYPES[c["dtype"]]
    shape = (n_pages + 1, c["Hkv"], c["page"], c["D"])
    k, v = _normal(shape, dt, gen), _normal(shape, dt, gen)
    return {"k_all": k, "v_all": v, "k": k[:n_pages], "v": v[:n_pages]}


def _prepare_branch(c, seed):
    """Parents in mid-decode, their pages anywhere in the pool, and empty rows for the branches."""
    P, n, kids = c["page"], c["parents"], c["children"]
    lens, B = _row_lens(c, n), n * (1 + kids)
    max_pages = _pages(c["tokens"] + c["n_new"], P) + 1
    used = sum(_pages(t, P) for t in lens)
    n_pages = used + B * (_pages(c["n_new"], P) + 2)
    r = np.random.RandomState(seed % (1 << 32))
    ids, at = r.permutation(n_pages).astype(np.int32), 0
    table, ref, src = np.full((B, max_pages), -1, dtype=np.int32), np.zeros(n_pages, dtype=np.int32), np.arange(B)
    for p, t in enumerate(lens):
        m = _pages(t, P)
        table[p, :m] = ids[at:at + m]
        ref[ids[at:at + m]] = 1
        at += m
    src[n:] = r.randint(0, n, n * kids)
    return {"case": c, "table": _ints(table), "ref": _ints(ref), "src_row": _ints(src), "seq_lens": _ints(lens + [0] * (n * kids)),
            "tok_begin": _ints([0] * B), "tok_end": _ints(lens + [0] * (n * kids)), "n_new": _ints([c["n_new"]] * B),
            "copy_src": _ints([-1] * B), "copy_dst": _ints([-1] * B), "copy_rows": _ints([0] * B), "n_ready": _ints([0] * B),
            **_pools(c, n_pages, seed)}


def _prepare_compact(c, seed):
    """A full batch whose pages lie anywhere in the pool, and the prompts that will take the freed rows (in turn)."""
    P, B = c["page"], c["B"]
    lens = _row_lens(c, B)
    max_pages = _pages(max(lens), P)
    used = sum(_pages(t, P) for t in lens)
    n_pages = used + used // 8 + 1
    r = np.random.RandomState(seed % (1 << 32))
    ids, at = r.permutation(n_pages).astype(np.int32), 0
    table, ref = np.full((B, max_pages), -1, dtype=np.int32), np.zeros(n_pages, dtype=np.int32)
    for b, t in enumerate(lens):
        m = _pages(t, P)
        table[b, :m] = ids[at:at + m]
        ref[ids[at:at + m]] = 1
        at += m
    rows, half = np.arange(B), np.random.RandomState(seed % (1 << 32) ^ 1).permutation(B) < B // 2
    return {"case": c, "turn": 0, "table": _ints(table), "ref": _ints(ref), "seq_lens": _ints(lens), "tok_begin": _ints([0] * B),
            "tok_end": _ints(lens), "src_rows": [_ints(np.where(h, -1, rows)) for h in (half, ~half)],
            "n_news": [_ints(np.where(h, lens, 0)) for h in (half, ~half)],
            "remap": _ints(np.arange(n_pages)), "move_src": _ints([-1] * n_pages), "move_dst": _ints([-1] * n_pages),
            "n_moves": _ints([0]), "copy_src": _ints([-1] * B), "copy_dst": _ints([-1] * B), "copy_rows": _ints([0] * B),
            "n_ready": _ints([0] * B), **_pools(c, n_pages, seed)}


# ---- one pass ------------------------------------------------------------------------------------------------------------

def run(state):
    op = state["case"]["op"]
    if own:
        return {"shared": _shared_own, "branch": _branch_own, "compact": _compact_own}[op](state)
    return {"shared": _shared_plain, "branch": _branch_plain, "compact": _compact_plain}[op](state)


def _desc(hg, s, hq, chunk, num_chunks):
    c, k = s["case"], s["k"]
    return hg.attn_desc(batch=s["table"].shape[0], num_q_heads=hq, num_kv_heads=c["Hkv"], head_dim=c["D"], dtype=DTYPES[c["dtype"]],
                        page_size=c["page"], num_pages=k.shape[0], page_stride=k.stride(0), head_stride=k.stride(1), tok_stride=k.stride(2),
                        block_table=s["table"], max_pages=s["table"].shape[1], chunk_tokens=chunk, num_chunks=num_chunks)


def _shared_own(s):
    if "step" not in s:      # the buffers and the marshalled call that a decode loop keeps
        import paper_2604_18529_b200 as hg
        c = s["case"]
        B, hq = c["B"], c["Hq"]
        chunk = hg.hg_attn_suggest_chunk(B * s["own_max"], hq, c["Hkv"], c["page"])
        desc = _desc(hg, s, hq, chunk, s["own_max"] // chunk + 2)
        pchunk = hg.hg_attn_prefix_suggest_chunk(s["shared_tokens"], c["groups"], s["n_members"], hq, c["Hkv"], c["page"])
        prefix = hg.prefix_desc(seq_group=s["seq_group"], group_row=s["group_row"], group_begin=s["group_begin"],
                                group_end=s["group_end"], chunk_tokens=pchunk, num_chunks=_pages(s["prefix_max"], pchunk))
        s["out"] = torch.empty((B, hq, c["D"]), dtype=torch.float32, device="cuda")
        s["lse"] = torch.empty((B, hq), dtype=torch.float32, device="cuda")
        ws = torch.empty(hg.hg_attn_shared_workspace_bytes(desc, prefix), dtype=torch.uint8, device="cuda")
        s["step"] = hg.prepare_decode_shared(s["q"], s["k"], s["v"], s["seq_lens"], s["tok_begin"], s["tok_end"], [], s["out"], s["lse"],
                                             ws, desc, prefix)
    s["step"]()
    return {"out": s["out"], "lse": s["lse"]}


def _branch_own(s):
    if "steps" not in s:
        import paper_2604_18529_b200 as hg
        desc = _desc(hg, s, s["case"]["Hkv"], 128, 1)
        s["steps"] = [hg.prepare_kv_fork(s["src_row"], s["ref"], s["seq_lens"], s["tok_begin"], s["tok_end"], desc),
                      hg.prepare_kv_reserve(s["seq_lens"], s["n_new"], s["ref"], s["copy_src"], s["copy_dst"], s["copy_rows"],
                                            s["n_ready"], desc),
                      hg.prepare_kv_copy_pages(s["copy_src"], s["copy_dst"], s["copy_rows"], None, s["k"], s["v"], desc)]
    for step in s["steps"]:
        step()
    return _branch_outputs(s)


def _compact_own(s):
    if "steps" not in s:
        import paper_2604_18529_b200 as hg
        desc = _desc(hg, s, s["case"]["Hkv"], 128, 1)
        s["steps"] = [[hg.prepare_kv_fork(s["src_rows"][t], s["ref"], s["seq_lens"], s["tok_begin"], s["tok_end"], desc),
                       hg.prepare_kv_compact(s["ref"], s["remap"], s["move_src"], s["move_dst"], s["n_moves"], desc),
                       hg.prepare_kv_copy_pages(s["move_src"], s["move_dst"], None, s["n_moves"], s["k"], s["v"], desc),
                       hg.prepare_kv_reserve(s["seq_lens"], s["n_news"][t], s["ref"], s["copy_src"], s["copy_dst"], s["copy_rows"],
                                             s["n_ready"], desc)] for t in (0, 1)]
    for step in s["steps"][s["turn"]]:
        step()
    s["turn"] ^= 1
    return _compact_outputs(s)


def _branch_outputs(s):
    return {n: s[n] for n in ("table", "ref", "seq_lens", "tok_begin", "tok_end", "copy_src", "copy_dst", "copy_rows", "n_ready", "k", "v")}


def _compact_outputs(s):
    return {n: s[n] for n in ("table", "ref", "seq_lens", "remap", "move_src", "move_dst", "n_moves", "n_ready", "k", "v")}


# ---- plain forms ---------------------------------------------------------------------------------------------------------

def _slice_rows(pool, table, n):
    """The first n token rows that each row of the table lists, in 32 bits: [rows][Hkv][n][D]"""
    P = pool.shape[2]
    x = pool[table[:, :_pages(n, P)].clamp(min=0).long()].float()
    R, np_, H, _, D = x.shape
    return x.permute(0, 2, 1, 3, 4).reshape(R, H, np_ * P, D)[:, :, :n]


def _own_rows(pool, table, begin, n):
    """n token rows from position begin[b] of every row, in 32 bits: [B][Hkv][n][D]"""
    P = pool.shape[2]
    t = (begin.long()[:, None] + torch.arange(n, device=begin.device)).clamp(max=table.shape[1] * P - 1)
    page = table.long().gather(1, t // P).clamp(min=0)
    return pool[page, :, t % P].float().transpose(1, 2)


def _shared_plain(s):
    c, q, dev = s["case"], s["q"].float(), s["q"].device
    B, H, G, D, NG, N = c["B"], c["Hkv"], c["Hq"] // c["Hkv"], c["D"], c["groups"], s["n_max"]
    inf, scale = float("inf"), D ** -0.5
    group = s["seq_group"].long()
    member = group >= 0
    same = (group[:, None] == group[None, :]).tril(-1)
    at = torch.where(member, group * N + same.sum(1), NG * N)                      # a sequence's place among the groups' members
    place = torch.zeros(NG * N + 1, dtype=torch.long, device=dev).scatter(0, at, torch.arange(B, device=dev))
    qg = q[place[:-1]].reshape(NG, N, H, G, D).transpose(1, 2).reshape(NG, H, N * G, D) * scale
    Lp, Lo = s["prefix_max"], s["own_max"]
    sg = qg @ _slice_rows(s["k"], s["table"][s["group_row"].long()], Lp).transpose(2, 3)
    t = torch.arange(Lp, device=dev)
    sg = sg.masked_fill(((t < s["group_begin"][:, None]) | (t >= s["group_end"][:, None]))[:, None, None], -inf)
    so = (q.reshape(B, H, G, D) * scale) @ _own_rows(s["k"], s["table"], s["tok_begin"], Lo).transpose(2, 3)
    so = so.masked_fill((torch.arange(Lo, device=dev) >= (s["tok_end"] - s["tok_begin"])[:, None])[:, None, None], -inf)

    def of_members(x):                                                             # [NG][H][N*G][...] -> [B][H][G][...]
        x = x.reshape(NG, H, N, G, -1).transpose(1, 2).reshape(NG * N, H, G, -1)
        return torch.where(member[:, None, None, None], x[at.clamp(max=NG * N - 1)], 0.0)

    def of_groups(x):                                                              # [B][H][G] -> [NG][H][N*G]
        return x[place[:-1]].reshape(NG, N, H, G).transpose(1, 2).reshape(NG, H, N * G)

    mg = torch.where(member[:, None, None], of_members(sg.amax(3, keepdim=True))[..., 0], -inf)
    m = torch.maximum(mg, so.amax(3))
    pg, po = (sg - of_groups(m)[..., None]).exp(), (so - m[..., None]).exp()
    weight = po.sum(3) + of_members(pg.sum(3, keepdim=True))[..., 0]
    value = po @ _own_rows(s["v"], s["table"], s["tok_begin"], Lo)
    value = value + of_members(pg @ _slice_rows(s["v"], s["table"][s["group_row"].long()], Lp))
    return {"out": (value / weight[..., None]).reshape(B, H * G, D), "lse": (m + weight.log()).reshape(B, H * G)}


def _count(n, entries, mask, dev):
    """How often each of n pages is among the masked entries."""
    return torch.zeros(n + 1, dtype=torch.int32, device=dev).index_add(0, torch.where(mask, entries, n).long().reshape(-1),
                                                                     torch.ones(entries.numel(), dtype=torch.int32, device=dev))[:n]


def _fork_plain(s, src):
    table, n, dev = s["table"], s["ref"].shape[0], s["table"].device
    rows = torch.arange(table.shape[0], device=dev)
    free, taken = (src < 0)[:, None], table[src.clamp(min=0).long()]
    new = torch.where(free, -1, taken)
    moved = (src != rows)[:, None].expand_as(table)
    ref = s["ref"] + _count(n, new, moved & (new >= 0), dev) - _count(n, table, moved & (table >= 0), dev)
    for name in ("seq_lens", "tok_begin", "tok_end"):
        s[name].copy_(torch.where(free[:, 0], 0, s[name][src.clamp(min=0).long()]))
    s["ref"].copy_(ref)
    table.copy_(new)


def _reserve_plain(s, n_new):
    table, ref, P, dev = s["table"], s["ref"], s["case"]["page"], s["table"].device
    (B, S), n = table.shape, ref.shape[0]
    lens, slot, order = s["seq_lens"][:, None], torch.arange(S, device=dev), torch.arange(B * S, device=dev).reshape(B, S)
    wanted = (slot >= lens // P) & (slot <= (lens + n_new[:, None] - 1) // P) & (n_new[:, None] > 0)
    mapped = wanted & (table >= 0)
    page = torch.where(mapped, table, n).long()
    writers = _count(n, table, mapped, dev)
    last = torch.full((n + 1,), -1, device=dev).scatter_reduce(0, page.reshape(-1), order.reshape(-1), "amax")
    refs, writers = torch.cat([ref, ref.new_zeros(1)])[page], torch.cat([writers, writers.new_zeros(1)])[page]
    shared = mapped & ((writers < refs) | (order != last[page]))
    need = (wanted & (table < 0)) | shared
    rank = need.reshape(-1).cumsum(0).reshape(B, S) - 1
    free = torch.cat([(ref != 0).to(torch.int8).argsort(stable=True).int(), table.new_full((B * S,), -1)])
    got = need & (rank < (ref == 0).sum())
    fresh = torch.where(got, free[rank.clamp(min=0)], -1)
    data = (slot == lens // P) & (lens % P != 0) & shared & got                      # the page holds tokens that the branch keeps
    s["copy_src"].copy_(torch.where(data, table, -1).amax(1))
    s["copy_dst"].copy_(torch.where(data, fresh, -1).amax(1))
    s["copy_rows"].copy_(torch.where(data.any(1), lens[:, 0] % P, 0))
    ref = ref + _count(n, fresh, got, dev) - _count(n, table, shared & got, dev)
    new = torch.where(got, fresh, table)
    held = torch.cat([ref, ref.new_zeros(1)])[torch.where(wanted & (new >= 0), new, n).long()]
    ready = wanted & (new >= 0) & (held == 1)
    stop = torch.where(wanted & ~ready, slot, S).amin(1, keepdim=True) * P
    s["n_ready"].copy_((torch.minimum(stop, lens + n_new[:, None].clamp(min=0)) - lens).clamp(min=0)[:, 0])
    s["ref"].copy_(ref)
    table.copy_(new)


def _compact_tables_plain(s):
    ref, table, dev = s["ref"], s["table"], s["table"].device
    n = ref.shape[0]
    ids, used = torch.arange(n, device=dev), ref > 0
    count = used.sum()
    hole, stray = ~used & (ids < count), used & (ids >= count)
    moves = hole.sum()
    dst = (~hole).to(torch.int8).argsort(stable=True)                                # holes, lowest first
    src = n - 1 - (~stray).flip(0).to(torch.int8).argsort(stable=True)               # pages beyond, highest first
    listed_ = ids < moves
    src, dst = torch.where(listed_, src, -1), torch.where(listed_, dst, -1)
    at = torch.where(listed_, src, n)
    remap = torch.arange(n + 1, device=dev).scatter(0, at, torch.where(listed_, dst, n))[:n]
    s["remap"].copy_(remap)
    s["move_src"].copy_(src)
    s["move_dst"].copy_(dst)
    s["n_moves"].copy_(moves)
    s["ref"].copy_(ref.new_zeros(n).scatter(0, remap, ref, reduce="add"))
    table.copy_(torch.where(table >= 0, remap[table.clamp(min=0).long()], table))


def _copy_plain(s, src, dst, rows):
    n, P = s["ref"].shape[0], s["case"]["page"]
    src, dst = torch.where(src < 0, n, src).long(), torch.where(src < 0, n, dst).long()
    for pool in (s["k_all"], s["v_all"]):
        data = pool[src]
        if rows is not None:
            data = torch.where((torch.arange(P, device=pool.device) < rows[:, None])[:, None, :, None], data, pool[dst])
        pool.index_copy_(0, dst, data)


def _branch_plain(s):
    _fork_plain(s, s["src_row"])
    _reserve_plain(s, s["n_new"])
    _copy_plain(s, s["copy_src"], s["copy_dst"], s["copy_rows"])
    return _branch_outputs(s)


def _compact_plain(s):
    _fork_plain(s, s["src_rows"][s["turn"]])
    _compact_tables_plain(s)
    _copy_plain(s, s["move_src"], s["move_dst"], None)
    _reserve_plain(s, s["n_news"][s["turn"]])
    s["turn"] ^= 1
    return _compact_outputs(s)


# ---- work ------------------------------------------------------------------------------------------------------------

def work(case):
    c = case
    if c["op"] == "shared":
        group, glen, own_len = _shared_plan(c)
        cells = sum(glen[g] for g in group if g >= 0) + sum(own_len)
        tokens = sum(glen[g] for g in set(group) if g >= 0) + sum(own_len)
        rows = c["B"] * c["Hq"]
        return {"bytes": tokens * (c["Hkv"] * c["D"] * 4 + 4 / c["page"]) + rows * (c["D"] * 6 + 4), "flops": 4 * cells * c["Hq"] * c["D"]}
    page_bytes = c["page"] * c["Hkv"] * c["D"] * 2 * 2
    if c["op"] == "branch":
        n = c["parents"] * c["children"]
        lens = _row_lens(c, c["parents"])
        entries = sum(_pages(t, c["page"]) for t in lens) * (1 + c["children"])
        copied = n * c["page"] / 2 * c["Hkv"] * c["D"] * 2 * 2       # half a page on average, K and V
        return {"bytes": 2 * copied + entries * 4 * 2 + (n + c["parents"]) * 40, "flops": entries}
    lens = _row_lens(c, c["B"])
    used = sum(_pages(t, c["page"]) for t in lens)
    return {"bytes": 2 * (used // 2) * page_bytes + used * 4 * 6, "flops": used * 4}


# ---- exact values ----------------------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "shared":
        return _shared_exact(s)
    names = ("table", "ref", "seq_lens", "tok_begin", "tok_end", "copy_src", "copy_dst", "copy_rows", "n_ready") if case["op"] == "branch" \
        else ("table", "ref", "seq_lens", "remap", "move_src", "move_dst", "n_moves", "n_ready")
    origin = _branch_exact(s) if case["op"] == "branch" else _compact_exact(s)
    return dict({n: None for n in names}, k=origin(s["k"]), v=origin(s["v"]))


def _shared_exact(s):
    """Sequence by sequence: its tokens in a row, one softmax in 64 bits."""
    c = s["case"]
    P, G = c["page"], c["Hq"] // c["Hkv"]
    group = s["seq_group"].tolist()
    rep, gend = s["group_row"].tolist(), s["group_end"].tolist()
    begin, end = s["tok_begin"].tolist(), s["tok_end"].tolist()
    table = s["table"].long()
    outs, lses = [], []
    for b in range(c["B"]):
        t = torch.arange(begin[b], end[b], device="cuda")
        page, row = table[b, t // P], t % P
        if group[b] >= 0:
            t = torch.arange(gend[group[b]], device="cuda")
            page, row = torch.cat([table[rep[group[b]], t // P], page]), torch.cat([t % P, row])
        out, lse = [], []
        for h in range(c["Hkv"]):
            k, v = s["k"][page, h, row].double(), s["v"][page, h, row].double()
            x = torch.einsum("jd,td->jt", s["q"][b, h * G:(h + 1) * G].double(), k) / c["D"] ** 0.5
            lse.append(torch.logsumexp(x, 1))
            out.append(torch.softmax(x, 1) @ v)
        outs.append(torch.cat(out))
        lses.append(torch.cat(lse))
    return {"out": torch.stack(outs), "lse": torch.stack(lses)}


def _branch_exact(s):
    """The operations one after the other, on lists; returns what builds a pool's values."""
    P, n_new = s["case"]["page"], s["case"]["n_new"]
    ref, lens, src = s["ref"].tolist(), s["seq_lens"].tolist(), s["src_row"].tolist()
    old = s["table"].tolist()
    table, lens = [list(old[p]) for p in src], [lens[p] for p in src]
    for b, p in enumerate(src):
        for e in table[b]:
            if p != b and e >= 0:
                ref[e] += 1
        for e in old[b]:
            if p != b and e >= 0:
                ref[e] -= 1
    copies = []
    free = iter([p for p, r in enumerate(ref) if r == 0])
    for b, row in enumerate(table):
        for slot in range(lens[b] // P, (lens[b] + n_new - 1) // P + 1):
            e = row[slot]
            if e >= 0 and ref[e] == 1:
                continue
            row[slot] = next(free)
            if e >= 0:
                ref[e] -= 1
                if slot == lens[b] // P and lens[b] % P:
                    copies.append((e, row[slot], lens[b] % P))

    def values(pool):
        x = pool.double()
        for a, b, n in copies:
            x[b, :, :n] = pool[a, :, :n].double()
        return x

    return values


def _compact_exact(s):
    ref, table = s["ref"].tolist(), s["table"].tolist()
    for b, p in enumerate(s["src_rows"][0].tolist()):
        for e in table[b] if p < 0 else []:
            if e >= 0:
                ref[e] -= 1
    low, high, moves = 0, len(ref) - 1, []
    while True:
        while low < len(ref) and ref[low]:
            low += 1
        while high >= 0 and not ref[high]:
            high -= 1
        if low >= high:
            break
        moves.append((high, low))
        ref[low], ref[high] = ref[high], 0

    def values(pool):
        x = pool.double()
        if moves:
            a, b = torch.tensor(moves, device=pool.device).unbind(1)
            x[b] = pool[a].double()
        return x

    return values
