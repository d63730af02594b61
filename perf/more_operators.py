"""One step of speculative decoding on the paged pool: cases, plain forms, exact values.

Four passes are measured, in the order in which a step makes them:

* ``slots``    what the kernels of the step need to know of its new tokens (drafted trees, prompts, single tokens), from the
               requests' lengths: rows, positions, places in the pool, masks of ancestors;
* ``rope``     rotary positions of the queries and keys, the keys and values going to their places in the pool;
* ``tree``     attention of the drafted tokens over the cache and over their ancestors;
* ``accept``   the rows of the accepted path move together behind the cache.
"""
import random

import numpy as np
import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


def _tree(name, dtype, B, Hq, Hkv, D, page, tokens, nodes, ragged, chain, host, lens_seed):
    return {"name": name, "op": "tree", "dtype": dtype, "B": B, "Hq": Hq, "Hkv": Hkv, "D": D, "page": page, "tokens": tokens,
            "nodes": nodes, "ragged": ragged, "chain": chain, "host": host, "lens_seed": lens_seed}


def _rope(name, dtype, rows, Hq, Hkv, D, page, rot, layout, far, fused):
    return {"name": name, "op": "rope", "dtype": dtype, "rows": rows, "Hq": Hq, "Hkv": Hkv, "D": D, "page": page, "rot": rot,
            "layout": layout, "far": far, "fused": fused}


def _slots(name, B, page, tokens, n_new, trees, lens_seed):
    return {"name": name, "op": "slots", "B": B, "page": page, "tokens": tokens, "n_new": n_new, "trees": trees, "lens_seed": lens_seed}


def _accept(name, dtype, B, Hkv, D, page, tokens, nodes, path, lens_seed):
    return {"name": name, "op": "accept", "dtype": dtype, "B": B, "Hkv": Hkv, "D": D, "page": page, "tokens": tokens, "nodes": nodes,
            "path": path, "lens_seed": lens_seed}


def listed():
    return [
        # two chats with a small draft each: latency
        _tree("tree_small", "f16", 2, 32, 8, 128, 16, 1000, 16, True, False, False, 1),
        # one long document, a wide draft: few sequences share all SMs, bound by arithmetic
        _tree("tree_document", "bf16", 1, 64, 8, 128, 64, 131072, 64, False, False, False, 2),
        # a busy server: requests and drafts of all lengths
        _tree("tree_ragged", "f16", 48, 32, 8, 128, 16, 16384, 32, True, False, False, 3),
        # one head per KV head, short drafts that are chains, the older half of the cache on the host
        _tree("tree_hybrid", "bf16", 16, 56, 56, 128, 64, 16384, 5, True, True, True, 4),
        # single tokens and their successors (drafts of two) in a large batch of short requests, 64 components a head
        _tree("tree_pairs_d64", "bf16", 128, 32, 8, 64, 32, 1500, 2, True, True, False, 5),
        # single tokens of a small batch: latency
        _rope("rope_step", "f16", 16, 32, 8, 128, 16, 128, "half", False, False),
        # drafts of a batch, far positions, rows of a fused projection
        _rope("rope_drafts", "bf16", 1024, 64, 8, 128, 64, 128, "half", True, True),
        # a long prompt, half of the head rotated, neighbouring pairs
        _rope("rope_prompt", "f16", 16384, 40, 40, 128, 64, 64, "interleaved", False, False),
        # drafted trees of a batch: latency
        _slots("slots_trees", 64, 16, 8000, 48, True, 6),
        # prompts of a few hundred requests
        _slots("slots_prompts", 300, 16, 2000, 4000, False, 7),
        # a small batch: latency
        _accept("accept_small", "f16", 8, 8, 128, 16, 2000, 16, 5, 8),
        # a large batch with one head per KV head and long accepted paths
        _accept("accept_large", "bf16", 128, 40, 128, 64, 2000, 64, 16, 9),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    op = rng.choice(["tree", "tree", "tree", "rope", "rope", "slots", "accept"])
    dtype = rng.choice(["f16", "bf16"])
    page = rng.choice([16, 32, 64, 128])
    seed = rng.randrange(1 << 20)
    hq, hkv, d = rng.choice([(8, 8, 64), (40, 40, 128), (56, 56, 128), (64, 8, 128), (32, 8, 128), (28, 4, 128), (20, 20, 64), (32, 8, 64)])
    if op == "tree":
        b, nodes = _log_int(rng, 1, 128), _log_int(rng, 1, 256)
        # no costlier than the largest listed cases: the cells of the logits, the elements of the cache
        tokens = min(_log_int(rng, 1, 131072), 131072 * 64 * 64 // (b * hq * nodes), (1 << 28) // (hkv * d * b))
        return _tree("tree", dtype, b, hq, hkv, d, page, max(1, tokens), nodes, rng.random() < 0.7, rng.random() < 0.4, rng.random() < 0.25, seed)
    if op == "rope":
        rows = min(_log_int(rng, 1, 16384), 16384 * 120 * 128 // ((hq + 2 * hkv) * d))
        return _rope("rope", dtype, rows, hq, hkv, d, page, rng.choice([d, d // 2, d // 4, 3 * d // 4]), rng.choice(["half", "interleaved"]),
                     rng.random() < 0.4, rng.random() < 0.5)
    if op == "slots":
        trees = rng.random() < 0.5
        b = _log_int(rng, 1, 512)
        n_new = _log_int(rng, 1, 256 if trees else 8000)
        return _slots("slots", b, page, _log_int(rng, 1, 16000), min(n_new, max(1, (1 << 16 if trees else 600000) // b)), trees, seed)
    b = _log_int(rng, 1, 128)
    nodes = _log_int(rng, 1, 256)
    tokens = max(1, min(_log_int(rng, 1, 8000), 128 * 2000 * 40 * 128 // (b * hkv * d)))
    return _accept("accept", dtype, b, hkv, d, page, tokens, nodes, rng.randint(1, min(nodes, 24)), seed)


# ---- lengths: from the case alone, so that its work is known ---------------------------------------------------------

def _tree_plan(c):
    """(cached tokens, first token on the GPU, drafted tokens) of every sequence"""
    r = random.Random(c["lens_seed"])
    if not c["ragged"]:
        lens, nodes = [c["tokens"]] * c["B"], [c["nodes"]] * c["B"]
    else:
        lens, nodes = [r.randint(1, c["tokens"]) for _ in range(c["B"])], [r.randint(1, c["nodes"]) for _ in range(c["B"])]
        lens[0], nodes[-1] = c["tokens"], c["nodes"]
    return lens, [n // 2 if c["host"] else 0 for n in lens], nodes


def _row_plan(c):
    """(cached tokens, new tokens) of every sequence"""
    r = random.Random(c["lens_seed"])
    return [r.randint(0, c["tokens"]) for _ in range(c["B"])], [r.randint(1, c["n_new"]) for _ in range(c["B"])]


def _pages(n, page):
    return -(-n // page)


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(shape, dtype, g):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dtype) if np.prod(shape) < 1 << 28 else \
        torch.randn(shape, generator=g, device="cuda", dtype=dtype)


def _ints(a, dtype=np.int32):
    return torch.as_tensor(np.asarray(a, dtype=dtype)).cuda()


def _table(lens, page, r, spare=0):
    """Pages for rows of these lengths, anywhere in the pool: (table [B][most], pages in the pool)"""
    counts = [_pages(n, page) for n in lens]
    n_pages = sum(counts) + spare
    ids, at = r.permutation(n_pages).astype(np.int32), 0
    table = np.full((len(lens), max(counts) + 1), -1, dtype=np.int32)
    for b, m in enumerate(counts):
        table[b, :m] = ids[at:at + m]
        at += m
    return table, n_pages


def _parents(counts, r):
    """Random trees, packed: a node's parent is any node before it, or -1, the end of the cache"""
    i = np.concatenate([np.arange(n) for n in counts])
    return (r.random_sample(i.size) * (i + 1)).astype(np.int32) - 1


def prepare(case, seed):
    return {"tree": _prepare_tree, "rope": _prepare_rope, "slots": _prepare_slots, "accept": _prepare_accept}[case["op"]](case, seed)


def _prepare_tree(c, seed):
    """A batch in the middle of decoding: keys and values of the drafts are in the pool already, behind the cache."""
    lens, begin, nodes = _tree_plan(c)
    r = np.random.RandomState(seed % (1 << 32))
    table, n_pages = _table([t + n for t, n in zip(lens, nodes)], c["page"], r)
    gen, dt = _generator(seed), DTYPES[c["dtype"]]
    N, cu = sum(nodes), np.concatenate([[0], np.cumsum(nodes)])
    s = {"case": c, "q": _normal((N, c["Hq"], c["D"]), dt, gen), "k": _normal((n_pages, c["Hkv"], c["page"], c["D"]), dt, gen),
         "v": _normal((n_pages, c["Hkv"], c["page"], c["D"]), dt, gen), "table": _ints(table), "seq_lens": _ints(lens),
         "tok_begin": _ints(begin), "cu": _ints(cu), "mask": None, "T": max(nodes), "host": []}
    if not c["chain"]:
        parent = _ints(_parents(nodes, r))
        s["mask"] = _ancestors(parent, s["cu"], max(nodes), _pages(max(nodes), 32))[0]
    if c["host"]:
        # what the host found in its part: as softmax partials of logits like the device's
        x = torch.randn((N, c["Hq"], 1), generator=gen, device="cuda")
        far = torch.as_tensor(np.repeat(np.maximum(begin, 1), nodes)).cuda().float()[:, None, None]
        o = torch.randn((N, c["Hq"], 1, c["D"]), generator=gen, device="cuda") * far.sqrt()[..., None]
        s["host"] = [(o, x * 0.3 + 2.5, far * 0.15 + x.square())]
    return s


def _frequencies(rot, far):
    """Radians per position; for far positions the slow ones are divided by 16, those between are blended."""
    f = 500000.0 ** (-np.arange(0, rot, 2, dtype=np.float64) / rot)
    turns = 8192 * f / (2 * np.pi)
    part = np.clip((turns - 1) / 3, 0, 1) if far else 1.0
    return f * part + f / 16 * (1 - part)


def _prepare_rope(c, seed):
    """The projections' outputs of new tokens, their positions, and their places in the pool."""
    N, P = c["rows"], c["page"]
    r = np.random.RandomState(seed % (1 << 32))
    gen, dt = _generator(seed), DTYPES[c["dtype"]]
    heads, D = [c["Hq"], c["Hkv"], c["Hkv"]], c["D"]
    if c["fused"]:
        rows = _normal((N, sum(heads), D), dt, gen)
        q, k, v = rows.split(heads, 1)
    else:
        q, k, v = [_normal((N, h, D), dt, gen) for h in heads]
    n_pages = _pages(N, P) + 3
    shape = (n_pages, c["Hkv"], P, D)
    pos = r.randint(0, 1 << 20 if c["far"] else 8192, N)
    return {"case": c, "q": q, "k_new": k, "v_new": v, "q_out": torch.zeros((N, c["Hq"], D), dtype=dt, device="cuda"),
            "k": _normal(shape, dt, gen), "v": _normal(shape, dt, gen), "pos": _ints(pos),
            "slot": _ints(r.permutation(n_pages * P)[:N], np.int64), "freq": torch.as_tensor(_frequencies(c["rot"], c["far"])).cuda(),
            "magnitude": 1.2772588722 if c["far"] else 1.0}


def _prepare_slots(c, seed):
    lens, n_new = _row_plan(c)
    r = np.random.RandomState(seed % (1 << 32))
    table, n_pages = _table([t + n for t, n in zip(lens, n_new)], c["page"], r)
    N, B, W = sum(n_new) + 7, c["B"], _pages(max(n_new), 32)      # a few rows more than there are tokens
    s = {"case": c, "table": _ints(table), "n_pages": n_pages, "seq_lens": _ints(lens), "n_new": _ints(n_new), "T": max(n_new),
         "parent": None, "cu": _ints([0] * (B + 1)), "seq": _ints([0] * N), "pos": _ints([0] * N), "slot": _ints([0] * N, np.int64), "mask": None}
    if c["trees"]:
        s["parent"] = _ints(np.concatenate([_parents(n_new, r), np.full(7, -1)]))
        s["mask"] = _ints(np.zeros((N, W)))
    return s


def _prepare_accept(c, seed):
    """The drafts' keys and values in the pool, and what the verification accepted of them."""
    q = random.Random(c["lens_seed"])
    lens = [q.randint(1, c["tokens"]) for _ in range(c["B"])]
    r = np.random.RandomState(seed % (1 << 32))
    table, n_pages = _table([t + c["nodes"] for t in lens], c["page"], r)
    path = np.stack([np.sort(r.permutation(c["nodes"])[:c["path"]]) for _ in range(c["B"])])
    gen, dt = _generator(seed), DTYPES[c["dtype"]]
    shape = (n_pages + 1, c["Hkv"], c["page"], c["D"])      # a page more than the pool has: where the plain form puts what does not move
    k, v = _normal(shape, dt, gen), _normal(shape, dt, gen)
    return {"case": c, "table": _ints(table), "seq_lens": _ints(lens), "path": _ints(path), "n_accept": _ints(r.randint(0, c["path"] + 1, c["B"])),
            "new_lens": _ints(lens), "k_all": k, "v_all": v, "k": k[:n_pages], "v": v[:n_pages]}


# ---- one pass ------------------------------------------------------------------------------------------------------------

def run(state):
    op = state["case"]["op"]
    if own:
        if "step" not in state:      # the buffers and the marshalled call that a decode loop keeps
            {"tree": _tree_own, "rope": _rope_own, "slots": _slots_own, "accept": _accept_own}[op](state)
        state["step"]()
    else:
        state.update({"tree": _tree_plain, "rope": _rope_plain, "slots": _slots_plain, "accept": _accept_plain}[op](state))
    names = {"tree": ("out", "lse"), "rope": ("q_out", "k", "v"), "slots": ("cu", "seq", "pos", "slot", "mask"), "accept": ("new_lens", "k", "v")}
    return {n: state[n] for n in names[op] if state[n] is not None}


def _desc(hg, s, **over):
    c, k, table = s["case"], s.get("k"), s.get("table")
    H, P, D = c.get("Hkv", 1), c["page"], c.get("D", 64)
    a = dict(batch=1 if table is None else table.shape[0], num_q_heads=c.get("Hq", H), num_kv_heads=H, head_dim=D, dtype=DTYPES[c.get("dtype", "f16")],
             page_size=P, num_pages=s["n_pages"] if k is None else k.shape[0], page_stride=H * P * D, head_stride=P * D, tok_stride=D,
             block_table=table, max_pages=1 if table is None else table.shape[1], chunk_tokens=128, num_chunks=1)
    return hg.attn_desc(**dict(a, **over))


def _tree_own(s):
    import paper_2604_18529_b200 as hg
    c, N = s["case"], s["q"].shape[0]
    desc = _desc(hg, s)
    tree = hg.tree_desc(cu_nodes=s["cu"], mask=s["mask"], num_rows=N, max_nodes=s["T"])
    s["out"] = torch.empty((N, c["Hq"], c["D"]), dtype=DTYPES[c["dtype"]], device="cuda")
    s["lse"] = torch.empty((N, c["Hq"]), dtype=torch.float32, device="cuda")
    ws = torch.empty(hg.hg_attn_tree_workspace_bytes(desc, tree), dtype=torch.uint8, device="cuda")
    s["step"] = hg.prepare_decode_tree(s["q"], s["k"], s["v"], s["seq_lens"], s["tok_begin"], s["host"], s["out"], s["lse"], ws, desc, tree)


def _rope_own(s):
    import paper_2604_18529_b200 as hg
    c = s["case"]
    rope = hg.rope_desc(rot_dim=c["rot"], layout=c["layout"], freq=s["freq"], magnitude=s["magnitude"])
    s["step"] = hg.prepare_kv_append_rope(s["q"], s["k_new"], s["v_new"], s["pos"], s["slot"], s["q_out"], s["k"], s["v"],
                                          _desc(hg, s, max_pages=s["k"].shape[0]), rope)


def _slots_own(s):
    import paper_2604_18529_b200 as hg
    s["step"] = hg.prepare_kv_slots(s["seq_lens"], s["n_new"], s["parent"], s["cu"], s["seq"], s["pos"], s["slot"], s["mask"], _desc(hg, s))


def _accept_own(s):
    import paper_2604_18529_b200 as hg
    s["step"] = hg.prepare_kv_accept(s["path"], s["n_accept"], s["seq_lens"], s["new_lens"], s["k"], s["v"], _desc(hg, s))


# ---- plain forms ---------------------------------------------------------------------------------------------------------

def _rows(pool, table, begin, n):
    """n token rows from position begin[b] of every row, in 32 bits: [B][Hkv][n][D]"""
    P = pool.shape[2]
    t = (begin.long()[:, None] + torch.arange(n, device=begin.device)).clamp(max=table.shape[1] * P - 1)
    page = table.long().gather(1, t // P).clamp(min=0)
    return pool[page, :, t % P].float().transpose(1, 2)


def _owner(cu, n):
    """The sequence of every row (the number of sequences behind the last), and its place in it"""
    row = torch.arange(n, device=cu.device)
    seq = torch.searchsorted(cu[1:].contiguous(), row, right=True)
    return seq, row - cu.long()[seq.clamp(max=cu.numel() - 2)]


def _ancestors(parent, cu, T, words):
    """Ancestors of every packed node (itself among them) as bits of 32-bit words, and how many there are besides itself"""
    B, N, dev = cu.numel() - 1, parent.numel(), parent.device
    seq, i = _owner(cu, N)
    last = seq >= B
    seq, i = torch.where(last, B, seq), torch.where(last, 0, i)
    step = torch.zeros((B + 1, T, T + 1), device=dev)
    step[seq, i, torch.where(parent < 0, T, parent).long()] = 1
    reach = step[:, :, :T] + torch.eye(T, device=dev)
    for _ in range(max(1, (T - 1).bit_length())):
        reach = (reach @ reach).clamp(max=1)
    bits = torch.zeros((B + 1, T, words * 32), dtype=torch.long, device=dev)
    bits[:, :, :T] = reach.long()
    mask = (bits.reshape(B + 1, T, words, 32) << torch.arange(32, device=dev)).sum(3)
    mask = torch.where(last[:, None], 0, mask[seq, i])
    return torch.where(mask >= 1 << 31, mask - (1 << 32), mask).int(), torch.where(last, 0, bits.sum(2)[seq, i] - 1)


def _tree_plain(s):
    c, dev = s["case"], s["q"].device
    B, H, G, D, T, N = c["B"], c["Hkv"], c["Hq"] // c["Hkv"], c["D"], s["T"], s["q"].shape[0]
    lens, begin, count = s["seq_lens"].long(), s["tok_begin"].long(), s["cu"].long().diff()
    seq, at = _owner(s["cu"], N)
    node = torch.arange(T, device=dev)
    exists = node < count[:, None]
    row = (s["cu"].long()[:-1, None] + node).clamp(max=N - 1)
    q = s["q"].float()[row].reshape(B, T, H, G, D).transpose(1, 2).reshape(B, H, T * G, D)
    n = c["tokens"] - (c["tokens"] // 2 if c["host"] else 0) + T           # the most tokens that a sequence has on the GPU
    x = (q * D ** -0.5) @ _rows(s["k"], s["table"], begin, n).transpose(2, 3)
    draft = begin[:, None] + torch.arange(n, device=dev) - lens[:, None]   # [B][n]: which node a token is, negative in the cache
    if s["mask"] is None:
        sees = node[:, None] >= node
    else:
        words = s["mask"].long()[row]
        sees = ((words[..., None] >> torch.arange(32, device=dev)) & 1).flatten(2)[:, :, :T].bool()
    sees = (sees & exists[:, None]).expand(B, T, T)
    sees = sees.gather(2, draft.clamp(0, T - 1)[:, None].expand(B, T, n)) & (draft < T)[:, None] | (draft < 0)[:, None]
    x = x.reshape(B, H, T, G, n).masked_fill(~sees[:, None, :, None], -float("inf"))

    def packed(y):                                                         # [B][H][T][G][...] -> [N][Hq][...]
        return y.transpose(1, 2)[seq, at].reshape(N, H * G, *y.shape[4:])

    m = x.amax(4)
    p = (x - m[..., None]).exp()
    o = p.reshape(B, H, T * G, n) @ _rows(s["v"], s["table"], begin, n)
    m, l, o = packed(m), packed(p.sum(4)), packed(o.reshape(B, H, T, G, D))
    if s["host"]:
        ho, hm, hl = [y[:, :, 0] for y in s["host"][0]]
        top = torch.maximum(m, hm)
        a, b = (m - top).exp(), (hm - top).exp()
        m, l, o = top, l * a + hl * b, o * a[..., None] + ho * b[..., None]
    return {"out": (o / l[..., None]).to(s["q"].dtype), "lse": m + l.log()}


def _rotated(x, s, wide):
    """Rows [N][heads][D] with their first `rot` components rotated, in the type `wide`"""
    c = s["case"]
    N, heads, D = x.shape
    angle = s["pos"].double()[:, None] * s["freq"]
    cos, sin = [(f(angle) * s["magnitude"]).to(wide)[:, None] for f in (torch.cos, torch.sin)]
    x = x.to(wide)
    r = x[..., :c["rot"]].reshape(N, heads, -1, 2).transpose(2, 3) if c["layout"] == "interleaved" else x[..., :c["rot"]].reshape(N, heads, 2, -1)
    a, b = r.unbind(2)
    r = torch.stack([a * cos - b * sin, b * cos + a * sin], 3 if c["layout"] == "interleaved" else 2)
    return torch.cat([r.reshape(N, heads, c["rot"]), x[..., c["rot"]:]], 2)


def _rope_plain(s):
    P, slot, dt = s["case"]["page"], s["slot"], s["q"].dtype
    s["q_out"].copy_(_rotated(s["q"], s, torch.float32).to(dt))
    s["k"][slot // P, :, slot % P] = _rotated(s["k_new"], s, torch.float32).to(dt)
    s["v"][slot // P, :, slot % P] = s["v_new"]
    return {}


def _slots_plain(s):
    P, N, table = s["case"]["page"], s["seq"].numel(), s["table"]
    B = table.shape[0]
    s["cu"].copy_(torch.cat([s["n_new"].new_zeros(1), s["n_new"].cumsum(0)]))
    seq, at = _owner(s["cu"], N)
    last = seq >= B
    seq = seq.clamp(max=B - 1)
    place = s["seq_lens"].long()[seq] + at
    depth = at
    if s["mask"] is not None:
        mask, depth = _ancestors(s["parent"], s["cu"], s["T"], s["mask"].shape[1])
        s["mask"].copy_(mask)
    page = table[seq, (place // P).clamp(max=table.shape[1] - 1)].long()
    s["seq"].copy_(torch.where(last, -1, seq))
    s["pos"].copy_(torch.where(last, 0, s["seq_lens"].long()[seq] + depth))
    s["slot"].copy_(torch.where(last | (page < 0), -1, page * P + place % P))
    return {}


def _accept_plain(s):
    P, table, n = s["case"]["page"], s["table"].long(), s["k"].shape[0]
    step = torch.arange(s["path"].shape[1], device=table.device)
    moves = step < s["n_accept"][:, None]
    source, target = s["seq_lens"].long()[:, None] + s["path"], s["seq_lens"].long()[:, None] + step
    from_page = torch.where(moves, table.gather(1, source // P), n)
    to_page = torch.where(moves, table.gather(1, target // P), n)
    for pool in (s["k_all"], s["v_all"]):
        pool[to_page, :, target % P] = pool[from_page, :, source % P]
    s["new_lens"].copy_(s["seq_lens"] + s["n_accept"])
    return {}


# ---- work ------------------------------------------------------------------------------------------------------------

def work(case):
    c = case
    if c["op"] == "tree":
        lens, begin, nodes = _tree_plan(c)
        tokens = sum(t - b + n for t, b, n in zip(lens, begin, nodes))
        cells = sum(n * (t - b + 1) for t, b, n in zip(lens, begin, nodes))
        rows = sum(nodes) * c["Hq"]
        return {"bytes": tokens * (c["Hkv"] * c["D"] * 4 + 4 / c["page"]) + rows * (c["D"] * (4 + 4 * c["host"]) + 4 + 8 * c["host"]),
                "flops": 4 * cells * c["Hq"] * c["D"]}
    if c["op"] == "rope":
        row = (c["Hq"] + 2 * c["Hkv"]) * c["D"] * 4 + 12
        return {"bytes": c["rows"] * row + c["rot"] * 4, "flops": c["rows"] * (c["Hq"] + c["Hkv"]) * c["rot"] * 3}
    if c["op"] == "slots":
        lens, n_new = _row_plan(c)
        words = _pages(max(n_new), 32) if c["trees"] else 0
        return {"bytes": sum(n_new) * (16 + 4 * c["trees"] + 4 * words) + sum(_pages(n, c["page"]) for n in n_new) * 4 + c["B"] * 12, "flops": sum(n_new)}
    # half of the paths on average, whatever the seed
    return {"bytes": c["B"] * (c["path"] / 2 * c["Hkv"] * c["D"] * 2 * 2 * 2 + c["path"] * 4 + 16), "flops": c["B"] * c["path"]}


# ---- exact values ----------------------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "tree":
        return _tree_exact(s)
    if case["op"] == "rope":
        return _rope_exact(s)
    if case["op"] == "accept":
        return _accept_exact(s)
    return None                                                            # whole numbers


def _tree_exact(s):
    """Sequence by sequence: the visible tokens in a row, one softmax in 64 bits."""
    c = s["case"]
    P, G, inf = c["page"], c["Hq"] // c["Hkv"], float("inf")
    cu, lens, begin, table = s["cu"].tolist(), s["seq_lens"].tolist(), s["tok_begin"].tolist(), s["table"].long()
    outs, lses = [], []
    for b in range(c["B"]):
        n = cu[b + 1] - cu[b]
        t = torch.arange(begin[b], lens[b] + n, device="cuda")
        page, row = table[b, t // P], t % P
        hidden = torch.zeros((n, t.numel()), dtype=torch.bool, device="cuda")
        for i in range(n):
            if s["mask"] is None:
                hidden[i, t.numel() - n + i + 1:] = True
            else:
                words = [w & 0xffffffff for w in s["mask"][cu[b] + i].tolist()]
                hidden[i, t.numel() - n:] = torch.tensor([not words[j // 32] >> (j % 32) & 1 for j in range(n)], device="cuda")
        out, lse = [], []
        for h in range(c["Hkv"]):
            k, v = s["k"][page, h, row].double(), s["v"][page, h, row].double()
            x = torch.einsum("ngd,td->ngt", s["q"][cu[b]:cu[b + 1], h * G:(h + 1) * G].double(), k) / c["D"] ** 0.5
            x = x.masked_fill(hidden[:, None], -inf)
            z = torch.logsumexp(x, 2)
            o = torch.softmax(x, 2) @ v
            if s["host"]:
                ho, hm, hl = [y[cu[b]:cu[b + 1], h * G:(h + 1) * G, 0].double() for y in s["host"][0]]
                hz = hm + hl.log()
                both = torch.logaddexp(z, hz)
                o = o * (z - both).exp()[..., None] + (ho / hl[..., None]) * (hz - both).exp()[..., None]
                z = both
            out.append(o)
            lse.append(z)
        outs.append(torch.cat(out, 1))
        lses.append(torch.cat(lse, 1))
    return {"out": torch.cat(outs), "lse": torch.cat(lses)}


def _rope_exact(s):
    """Pairs as complex numbers, turned by their angles in 64 bits."""
    c = s["case"]
    P, rot, slot = c["page"], c["rot"], s["slot"]
    turn = torch.polar(torch.full((c["rows"], rot // 2), s["magnitude"], dtype=torch.float64, device="cuda"),
                       s["pos"].double()[:, None] * s["freq"])[:, None]
    first = torch.arange(rot // 2, device="cuda") * (2 if c["layout"] == "interleaved" else 1)
    second = first + (1 if c["layout"] == "interleaved" else rot // 2)

    def turned(x):
        x = x.double()
        z = torch.complex(x[..., first], x[..., second]) * turn
        x[..., first], x[..., second] = z.real, z.imag
        return x

    k, v = s["k"].double(), s["v"].double()
    k[slot // P, :, slot % P] = turned(s["k_new"])
    v[slot // P, :, slot % P] = s["v_new"].double()
    return {"q_out": turned(s["q"]), "k": k, "v": v}


def _accept_exact(s):
    """Row by row, in the order of the path."""
    P = s["case"]["page"]
    table, lens, path, count = s["table"].tolist(), s["seq_lens"].tolist(), s["path"].tolist(), s["n_accept"].tolist()
    moves = [(table[b][(t + x) // P], (t + x) % P, table[b][(t + j) // P], (t + j) % P)
             for b, t in enumerate(lens) for j, x in enumerate(path[b][:count[b]]) if j != x]
    pools = []
    for pool in (s["k"], s["v"]):
        y = pool.double()
        for a, i, b, j in moves:
            y[b, :, j] = y[a, :, i].clone()
        pools.append(y)
    return {"new_lens": None, "k": pools[0], "v": pools[1]}
