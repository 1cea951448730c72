"""Serving drafted tokens over a paged compressed cache, as cases that can be measured.

Three operators that a server calls one after the other in every step of speculative decoding:

  tables   commvq_page_tables: block tables grown and slots laid out from the requests' lengths
  store    commvq_store_pages: new code records (and positions) written to their slots in the pages
  tree     commvq_tree_attn: attention of a tree of drafted tokens per sequence over the pages and over the drafted
           tokens' own keys and values; positions of one to four axes; one node per sequence is ordinary decoding

A case is a dict of plain values:

  what     "tables", "store" or "tree"
  tables   batch requests, cached tokens each (between cached_least and cached_most), new tokens each (between new_least and
           new_most), block tokens a page; spread: the seed of the lengths
  store    tokens, kv_heads, m_key, m_val, block, axes; skipped: one token in so many has no slot (0: none)
  tree     q_heads, kv_heads, batch, shortest, longest (cached tokens), nodes_least, nodes_most (drafted tokens), m_key, m_val,
           block, axes, storage "bf16" or "f32", shape "tree" (random parents) or "chain"; spread: the seed of lengths and trees

`own` False: the plain form, elementary torch operations in 32 bits.  `own` True: the library's calls.
"""
import math
import random

import torch

own = False

HEAD_DIM, PAIRS, WORDS = 128, 64, 256
ROPE_BASE, MAX_POSITION = 500000.0, 131200
# pairs of a head that turn with the first, second and third axis (time, height, width), as models for images and video
# cut them; a fourth axis, where there is one, takes the last eight of the third
SECTIONS = {1: (64,), 2: (32, 32), 3: (16, 24, 24), 4: (16, 24, 16, 8)}


def _tables(name=None, **kw):
    case = {"what": "tables", "batch": 1, "cached_least": 0, "cached_most": 0, "new_least": 1, "new_most": 1, "block": 16, "spread": 0}
    case.update(kw)
    return case if name is None else dict(case, name=name)


def _store(name=None, **kw):
    case = {"what": "store", "tokens": 1, "kv_heads": 8, "m_key": 16, "m_val": 16, "block": 16, "axes": 1, "skipped": 0, "spread": 0}
    case.update(kw)
    return case if name is None else dict(case, name=name)


def _tree(name=None, **kw):
    case = {"what": "tree", "q_heads": 32, "kv_heads": 8, "batch": 1, "shortest": 1, "longest": 1, "nodes_least": 1, "nodes_most": 1,
            "m_key": 16, "m_val": 16, "block": 16, "axes": 1, "storage": "bf16", "shape": "tree", "spread": 0}
    case.update(kw)
    return case if name is None else dict(case, name=name)


def listed():
    return [
        # one step of a small server: 24 chats, a drafted tree's worth of room each
        _tables("tables_24_chats", batch=24, cached_least=0, cached_most=4000, new_least=0, new_most=9, spread=1),
        # admission of a large batch of prompts next to running chats
        _tables("tables_1000_prompts", batch=1000, cached_least=0, cached_most=600, new_least=1, new_most=520, block=32, spread=2),
        # the accepted tokens of one step of eight sequences
        _store("store_accepted", tokens=27, m_key=32, m_val=32, skipped=9, spread=3),
        # a long prompt, encoded in one go, of the 8B-shaped layer with positions of three axes
        _store("store_prompt_90k", tokens=90001, m_key=16, m_val=32, block=64, axes=3, spread=4),
        # the beginning of a chat: few cached tokens, a small tree; all latency
        _tree("tree_chat_700", shortest=701, longest=701, nodes_least=8, nodes_most=8, m_key=32, m_val=32, spread=5),
        # a single fp32 head over a short context
        _tree("tree_one_head_f32", q_heads=1, kv_heads=1, shortest=4096, longest=4096, nodes_least=5, nodes_most=5, m_key=32, m_val=32,
              storage="f32", spread=6),
        # a chat batch of ragged lengths, some of them just begun
        _tree("tree_batch_16", batch=16, shortest=0, longest=6000, nodes_least=1, nodes_most=16, m_key=32, m_val=32, spread=7),
        # a long document, 2 bits a scalar, a full tree of 64 nodes
        _tree("tree_8b_32k_64", shortest=32768, longest=32768, nodes_least=64, nodes_most=64, m_key=32, m_val=32, block=64, spread=8),
        # ordinary decoding over pages: one node per sequence, 1 bit a scalar, 128K tokens
        _tree("single_8b_128k", shortest=131072, longest=131072, block=64, shape="chain", spread=9),
        # an ordinary tree over the headline context
        _tree("tree_8b_128k_26", shortest=131072, longest=131072, nodes_least=26, nodes_most=26, block=64, spread=10),
        # a video: positions of three axes, stored with the cache, and a short chain of drafted tokens
        _tree("axes_8b_3x20k", batch=3, shortest=9000, longest=20011, nodes_least=4, nodes_most=6, axes=3, shape="chain", spread=11),
        # the 70B-shaped layer, four long sequences, 2-bit keys and 1-bit values
        _tree("tree_70b_4x128k", q_heads=64, batch=4, shortest=131072, longest=131072, nodes_least=16, nodes_most=16, m_key=32, m_val=16,
              block=128, spread=12),
    ]


def _between(rng, lo, hi):
    """A whole number on [lo, hi], even over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the ranges that the listed ones stand for."""
    spread, block = rng.randrange(1 << 20), rng.choice((16, 16, 32, 64, 128, 256))
    kind = rng.choice(("tables", "store", "chat", "f32", "batch", "long", "long", "single", "axes"))
    if kind == "tables":
        batch = _between(rng, 1, 2000)
        new = _between(rng, 1, max(1, 500000 // batch))
        return _tables(batch=batch, cached_most=_between(rng, 1, 8000), new_least=rng.choice((0, 1)), new_most=new, block=block, spread=spread)
    if kind == "store":
        return _store(tokens=_between(rng, 1, 90000), kv_heads=rng.choice((1, 2, 8, 8)), m_key=rng.choice((16, 32)), m_val=rng.choice((16, 32)), block=block,
                      axes=rng.choice((1, 1, 2, 3, 4)), skipped=rng.choice((0, 0, 3, 50)), spread=spread)
    layer = {"m_key": rng.choice((16, 32)), "m_val": rng.choice((16, 32)), "block": block, "spread": spread,
             "shape": rng.choice(("tree", "tree", "chain"))}
    heads = {"q_heads": 8 * rng.choice((1, 2, 4, 4, 8))}
    nodes = _between(rng, 1, 64)
    some = {"nodes_least": max(1, nodes // 2), "nodes_most": nodes}
    if kind == "chat":
        n = _between(rng, 1, 2500)
        return _tree(shortest=n, longest=n, **some, **layer, **heads)
    if kind == "f32":
        n = _between(rng, 100, 6000)
        kv = rng.choice((1, 2))
        return _tree(q_heads=kv * rng.choice((1, 4)), kv_heads=kv, shortest=n, longest=n, storage="f32", **some, **layer)
    if kind == "batch":
        batch = _between(rng, 2, 40)
        n = _between(rng, 200, 120000 // batch)
        return _tree(batch=batch, shortest=rng.choice((0, n // 4)), longest=n, **some, **layer, **heads)
    if kind == "long":
        n = _between(rng, 4000, 131072)
        return _tree(shortest=n, longest=n, **some, **layer, **heads)
    if kind == "single":
        batch = _between(rng, 1, 8)
        n = _between(rng, 300, 131072 // batch)
        return _tree(batch=batch, shortest=max(1, n // 2), longest=n, **layer, **heads)
    batch = _between(rng, 1, 6)
    n = _between(rng, 500, 100000 // batch)
    return _tree(batch=batch, shortest=max(1, n // 3), longest=n, axes=rng.choice((2, 3, 4)), **some, **layer, **heads)


# ------------------------------------------------------------------ inputs
def _normal(gen, shape, std=1.0, bf16=True):
    x = torch.randn(shape, generator=gen, device="cuda").mul_(std)
    return x.to(torch.bfloat16) if bf16 else x


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _running(values):
    out = [0]
    for v in values:
        out.append(out[-1] + v)
    return out


def _table_lengths(case):
    r = random.Random(case["spread"])
    cached = [r.randint(case["cached_least"], case["cached_most"]) for _ in range(case["batch"])]
    new = [r.randint(case["new_least"], case["new_most"]) for _ in range(case["batch"])]
    new[r.randrange(len(new))] = case["new_most"]
    return cached, new


def _tree_lengths(case):
    r = random.Random(case["spread"])
    lens = [r.randint(case["shortest"], case["longest"]) for _ in range(case["batch"])]
    nodes = [r.randint(case["nodes_least"], case["nodes_most"]) for _ in range(case["batch"])]
    lens[r.randrange(len(lens))] = case["longest"]
    nodes[r.randrange(len(nodes))] = case["nodes_most"]
    return lens, nodes


def _pages_of(tokens, block):
    return -(-tokens // block)


def _inputs_tables(case, gen):
    block = case["block"]
    cached, new = _table_lengths(case)
    held = [_pages_of(c, block) for c in cached]
    need = [_pages_of(c + n, block) - h for c, n, h in zip(cached, new, held)]
    widest = max(1, max(h + n for h, n in zip(held, need)))
    pool = sum(held) + sum(need) + 3
    order = torch.randperm(pool, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((case["batch"], widest), -1, dtype=torch.int32, device="cuda")
    have = torch.arange(widest, device="cuda")[None, :] < _int32(held)[:, None]
    table[have] = order[:sum(held)]
    return {"cached": _int32(cached), "new": _int32(new), "free": order[sum(held):].contiguous(), "table": table, "pool": pool, "total": sum(new)}


def _inputs_store(case, gen):
    n, block, hkv = case["tokens"], case["block"], case["kv_heads"]
    pool = _pages_of(n, block) + 2
    slots = torch.randperm(pool * block, generator=gen, device="cuda")[:n].to(torch.int32)
    if n > block:  # whole pages follow each other in a prompt, pages in any order
        pages = torch.randperm(pool, generator=gen, device="cuda").to(torch.int32)
        at = torch.arange(n, device="cuda") + random.Random(case["spread"]).randrange(block)
        slots = pages[at // block] * block + (at % block).to(torch.int32)
    if case["skipped"]:
        slots[::case["skipped"]] = -1
    codes = lambda *shape: torch.randint(0, WORDS, shape, generator=gen, device="cuda", dtype=torch.uint8)
    return {"slots": slots, "key_codes": codes(n, hkv, case["m_key"]), "val_codes": codes(n, hkv, case["m_val"]),
            "pos": torch.randint(0, MAX_POSITION, (n, case["axes"]), generator=gen, device="cuda", dtype=torch.int32),
            "key_pages": codes(pool, hkv, block, case["m_key"]), "val_pages": codes(pool, hkv, block, case["m_val"]),
            "page_pos": torch.zeros((pool * block, case["axes"]), dtype=torch.int32, device="cuda"), "pool": pool}


def _inputs_tree(case, gen):
    block, hkv, hq, axes, bf16 = case["block"], case["kv_heads"], case["q_heads"], case["axes"], case["storage"] == "bf16"
    lens, nodes = _tree_lengths(case)
    r = random.Random(case["spread"] + 1)
    held = [_pages_of(n, block) for n in lens]
    pool = sum(held) + 3
    order = torch.randperm(pool, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((case["batch"], max(1, max(held))), -1, dtype=torch.int32, device="cuda")
    table[torch.arange(table.shape[1], device="cuda")[None, :] < _int32(held)[:, None]] = order[:sum(held)]
    masks, pos = [], []
    key_pos = None
    if axes > 1:  # frames of 12 x 16 patches, then text: every axis goes on together
        key_pos = torch.zeros((pool * block, axes), dtype=torch.int32, device="cuda")
    for b, (n, k) in enumerate(zip(lens, nodes)):
        if axes > 1:
            i = torch.arange(n, device="cuda")
            frame, y, x = i // 192, i // 16 % 12, i % 16
            rows = torch.stack((frame, frame + y, frame + x, frame)[:axes], 1).to(torch.int32)
            slot = table[b].long()[i // block] * block + i % block
            key_pos[slot] = rows
            start = n // 192 + 16
        else:
            start = n
        mine, depth = [], []
        for i in range(k):
            parent = i - 1 if case["shape"] == "chain" else (r.randrange(max(0, i - 8), i) if i else -1)
            mine.append((mine[parent] if parent >= 0 else 0) | 1 << i)
            depth.append(depth[parent] + 1 if parent >= 0 else 0)
        masks += mine
        pos += [[start + x] * axes for x in depth]
    cb = lambda m: _normal(gen, (hkv, m, WORDS, HEAD_DIM), m ** -0.5, bf16)
    codes = lambda m: torch.randint(0, WORDS, (pool, hkv, block, m), generator=gen, device="cuda", dtype=torch.uint8)
    total = sum(nodes)
    return {"lens": lens, "nodes": nodes, "pool": pool, "table": table, "seq_lens": _int32(lens), "cu_nodes": _int32(_running(nodes)),
            "mask": torch.tensor([m - (1 << 64) if m >> 63 else m for m in masks], dtype=torch.int64, device="cuda"), "node_pos": _int32(pos), "key_pos": key_pos,
            "q": _normal(gen, (total, hq, HEAD_DIM), 1.0, bf16), "node_k": _normal(gen, (total, hkv, HEAD_DIM), 1.0, bf16),
            "node_v": _normal(gen, (total, hkv, HEAD_DIM), 1.0, bf16), "key_cb": cb(case["m_key"]), "val_cb": cb(case["m_val"]),
            "key_pages": codes(case["m_key"]), "val_pages": codes(case["m_val"])}


_INPUTS = {"tables": _inputs_tables, "store": _inputs_store, "tree": _inputs_tree}


def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return _INPUTS[case["what"]](case, gen)


def _pair_axis(axes):
    return [a for a, n in enumerate(SECTIONS[axes]) for _ in range(n)]


class _Handle:
    """A library handle that goes with the state that uses it."""

    def __init__(self, cv, case):
        kind = cv.COMMVQ_F32 if case.get("storage") == "f32" else cv.COMMVQ_BF16
        self.cv = cv
        self.ptr = cv.commvq_create(cv.Config(case.get("q_heads", case["kv_heads"]), case["kv_heads"], HEAD_DIM, case["m_key"], case["m_val"], WORDS,
                                              kind, kind, ROPE_BASE, 0.0, MAX_POSITION, cv.COMMVQ_KEYS_INDEXED, 0, 0, cv.COMMVQ_VALUES_INDEXED, 0))

    def __del__(self):
        self.cv.commvq_destroy(self.ptr)


def _stream():
    return torch.cuda.current_stream().cuda_stream


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if case["what"] == "tables":  # what the call fills in
        s["seq_lens"] = torch.zeros(case["batch"], dtype=torch.int32, device="cuda")
        s["cu_new"] = torch.zeros(case["batch"] + 1, dtype=torch.int32, device="cuda")
        s["slots"], s["token_pos"] = (torch.zeros(s["total"], dtype=torch.int32, device="cuda") for _ in range(2))
        s["taken"] = torch.zeros(2, dtype=torch.int32, device="cuda")
    if case["what"] == "tree":
        s["out"] = torch.empty_like(s["q"])
        s["theta"] = ROPE_BASE ** (-torch.arange(PAIRS, device="cuda", dtype=torch.float64) / PAIRS)
        s["axis"] = torch.tensor(_pair_axis(case["axes"]), device="cuda")
    if not own:
        return s
    import paper_2506_18879_amd as cv

    s["cv"] = cv
    s["pages"] = cv.make_pages(case["block"], s["pool"], s["table"].shape[1] if "table" in s else 1, case.get("axes", 1))
    if case["what"] != "tables":
        s["handle"] = _Handle(cv, case)
    if case["what"] == "tree":
        h = s["handle"].ptr
        s["tree"] = cv.make_tree(case["batch"], sum(s["nodes"]), max(s["nodes"]), max(s["lens"]), s["seq_lens"], s["table"], s["cu_nodes"], s["node_pos"],
                                 s["mask"], s["key_pos"], _pair_axis(case["axes"]) if case["axes"] > 1 else None)
        s["workspace"] = torch.empty(cv.commvq_tree_workspace_bytes(h, case["batch"], sum(s["nodes"]), max(s["nodes"]), max(s["lens"])),
                                     dtype=torch.uint8, device="cuda")
        s["tables"] = None
        if case["storage"] == "bf16":  # the codebooks are a layer's constants: laid out once
            s["tables"] = torch.empty(cv.commvq_tree_table_bytes(h), dtype=torch.uint8, device="cuda")
            cv.commvq_tree_prepare(h, s["key_cb"], s["val_cb"], s["tables"], _stream())
    return s


# ------------------------------------------------------------------ one pass
def _own_tables(s):
    s["cv"].commvq_page_tables(s["pages"], s["case"]["batch"], s["cached"], s["new"], s["free"], s["free"].numel(), s["table"], s["seq_lens"], s["cu_new"],
                               s["slots"], s["token_pos"], s["total"], s["taken"], _stream())
    return {k: s[k] for k in ("table", "seq_lens", "cu_new", "slots", "token_pos", "taken")}


def _plain_tables(s):
    block, cached, new, table = s["case"]["block"], s["cached"], s["new"], s["table"]
    widest = table.shape[1]
    held, after = (cached + block - 1) // block, (cached + new + block - 1) // block
    fits = after <= widest
    need = torch.where(fits, after - held, torch.zeros_like(held))
    ends = torch.cumsum(need, 0)
    granted = fits & ((ends <= s["free"].numel()) | (need == 0))
    column = torch.arange(widest, device=table.device)[None, :]
    fresh = granted[:, None] & (column >= held[:, None]) & (column < after[:, None])
    at = (ends - need)[:, None] + column - held[:, None]
    table = torch.where(fresh, s["free"][at.clamp(0, s["free"].numel() - 1)], table)
    cu = torch.cat((torch.zeros(1, dtype=torch.int64, device=table.device), torch.cumsum(new, 0)))
    token = torch.arange(s["total"], device=table.device)
    request = torch.searchsorted(cu[1:].contiguous(), token, right=True)
    pos = cached[request] + token - cu[request]
    page = table[request, (pos // block).clamp(max=widest - 1)]
    slots = torch.where(granted[request] & (page >= 0) & (page < s["pool"]), page * block + pos % block, torch.full_like(page, -1))
    taken = torch.stack((torch.where(granted, need, torch.zeros_like(need)).sum(), (~granted).sum()))
    return {"table": table, "seq_lens": torch.where(granted, cached + new, cached), "cu_new": cu.to(torch.int32), "slots": slots.to(torch.int32),
            "token_pos": pos.to(torch.int32), "taken": taken.to(torch.int32)}


def _own_store(s):
    s["cv"].commvq_store_pages(s["handle"].ptr, s["pages"], s["case"]["tokens"], s["slots"], s["key_codes"], s["val_codes"], s["pos"], s["key_pages"],
                               s["val_pages"], s["page_pos"], _stream())
    return {k: s[k] for k in ("key_pages", "val_pages", "page_pos")}


def _plain_store(s):
    block, keep = s["case"]["block"], s["slots"] >= 0
    slots = s["slots"][keep].long()
    s["key_pages"][slots // block, :, slots % block] = s["key_codes"][keep]
    s["val_pages"][slots // block, :, slots % block] = s["val_codes"][keep]
    s["page_pos"][slots] = s["pos"][keep]
    return {k: s[k] for k in ("key_pages", "val_pages", "page_pos")}


def _own_tree(s):
    s["cv"].commvq_tree_attn(s["handle"].ptr, s["pages"], s["tree"], s["q"], s["node_k"], s["node_v"], s["key_pages"], s["val_pages"], s["key_cb"],
                             s["val_cb"], s["tables"], s["out"], s["workspace"], s["workspace"].numel(), _stream())
    return s["out"]


def _turn(x, pos, theta, axis):
    """x R_p: pairs (x, y) -> (x cos + y sin, y cos - x sin), every pair by the position on its own axis."""
    angle = pos.double()[:, axis] * theta
    c, n = (f(angle).float()[:, None, :] for f in (torch.cos, torch.sin))
    x = x.float()
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack((a * c + b * n, b * c - a * n), -1).flatten(-2)


def _decoded(codes, book):
    """Sums of the selected rows: codes [tokens][heads][M], book [heads][M][256][d]."""
    heads, m = book.shape[:2]
    rows = book.float().view(-1, HEAD_DIM)
    base = torch.arange(heads, device=codes.device) * (m * WORDS)
    out = torch.zeros(codes.shape[:2] + (HEAD_DIM,), device=codes.device)
    for i in range(m):
        out += rows[codes[:, :, i].long() + base + i * WORDS]
    return out


def _plain_tree(s):
    case = s["case"]
    block, hkv, hq = case["block"], case["kv_heads"], case["q_heads"]
    group = hq // hkv
    parts, first = [], 0
    bit = torch.arange(64, device=s["q"].device)
    for b, (n, k) in enumerate(zip(s["lens"], s["nodes"])):
        mine = slice(first, first + k)
        first += k
        i = torch.arange(n, device=s["q"].device)
        slot = s["table"][b].long()[i // block] * block + i % block
        pos = s["key_pos"][slot] if s["key_pos"] is not None else i[:, None]
        keys = _decoded(s["key_pages"][slot // block, :, slot % block], s["key_cb"])
        keys = torch.cat((_turn(keys, pos, s["theta"], s["axis"]), _turn(s["node_k"][mine], s["node_pos"][mine], s["theta"], s["axis"])))
        values = torch.cat((_decoded(s["val_pages"][slot // block, :, slot % block], s["val_cb"]), s["node_v"][mine].float()))
        q = _turn(s["q"][mine], s["node_pos"][mine], s["theta"], s["axis"]).view(k, hkv, group, HEAD_DIM).permute(1, 0, 2, 3).reshape(hkv, k * group, HEAD_DIM)
        logits = torch.bmm(q, keys.permute(1, 2, 0).contiguous()).view(hkv, k, group, n + k) * HEAD_DIM ** -0.5
        seen = (s["mask"][mine, None] >> bit[None, :k] & 1) != 0
        seen = torch.cat((torch.ones((k, n), dtype=torch.bool, device=seen.device), seen), 1)[None, :, None, :]
        logits = torch.where(seen, logits, torch.full_like(logits, -math.inf))
        top = logits.amax(-1, keepdim=True)
        weight = torch.where(seen, torch.exp(logits - top), torch.zeros_like(logits))
        out = torch.bmm(weight.view(hkv, k * group, n + k), values.permute(1, 0, 2).contiguous()).view(hkv, k, group, HEAD_DIM) / weight.sum(-1, keepdim=True)
        parts.append(out.permute(1, 0, 2, 3).reshape(k, hq, HEAD_DIM))
    return torch.cat(parts).to(s["q"].dtype)


def run(state):
    what = state["case"]["what"]
    if own:
        return {"tables": _own_tables, "store": _own_store, "tree": _own_tree}[what](state)
    return {"tables": _plain_tables, "store": _plain_store, "tree": _plain_tree}[what](state)


# ------------------------------------------------------------------ the definition in 64 bits
def _exact_tables(case, s):
    """Request by request and page by page, as a scheduler on the host does it."""
    block, free = case["block"], s["free"].tolist()
    cached, new = _table_lengths(case)
    table, next_page = s["table"].tolist(), 0
    slots, where, lens, cu = [], [], [], [0]
    for row, c, n in zip(table, cached, new):
        for page in range(_pages_of(c, block), _pages_of(c + n, block)):
            row[page] = free[next_page]
            next_page += 1
        for t in range(c, c + n):
            slots.append(row[t // block] * block + t % block)
            where.append(t)
        lens.append(c + n)
        cu.append(cu[-1] + n)
    return {"table": _int32(table), "seq_lens": _int32(lens), "cu_new": _int32(cu), "slots": _int32(slots), "token_pos": _int32(where), "taken": _int32([next_page, 0])}


def _exact_store(case, s):
    """Token by token into copies on the host; a token without a slot goes nowhere."""
    block = case["block"]
    out = {k: s[k].cpu().numpy() for k in ("key_pages", "val_pages", "page_pos")}
    keys, values, pos = (s[k].cpu().numpy() for k in ("key_codes", "val_codes", "pos"))
    for t, slot in enumerate(s["slots"].tolist()):
        if slot >= 0:
            out["key_pages"][slot // block, :, slot % block] = keys[t]
            out["val_pages"][slot // block, :, slot % block] = values[t]
            out["page_pos"][slot] = pos[t]
    return out


def _exact_tree(case, s):
    """Sequence by sequence and KV head by KV head, keys and queries as complex numbers: Re(q conj(k) exp(-i (t - p) theta))."""
    block, hkv, group = case["block"], case["kv_heads"], case["q_heads"] // case["kv_heads"]
    device = s["q"].device
    theta = torch.pow(torch.tensor(ROPE_BASE, dtype=torch.float64, device=device), -2.0 * torch.arange(PAIRS, dtype=torch.float64, device=device) / HEAD_DIM)
    axis = torch.tensor(_pair_axis(case["axes"]), device=device)
    paired = lambda x: torch.view_as_complex(x.double().reshape(x.shape[:-1] + (PAIRS, 2)).contiguous())
    out = torch.zeros((sum(s["nodes"]), case["q_heads"], HEAD_DIM), dtype=torch.float64, device=device)
    first = 0
    for b, (n, k) in enumerate(zip(s["lens"], s["nodes"])):
        token = torch.arange(n, device=device)
        page, within = s["table"][b].long()[token // block], token % block
        pos = token[:, None].expand(n, case["axes"]) if s["key_pos"] is None else s["key_pos"][page * block + within]
        pos = torch.cat((pos.double(), s["node_pos"][first:first + k].double()))
        back = torch.polar(torch.ones((n + k, PAIRS), dtype=torch.float64, device=device), -pos[:, axis] * theta)
        masks = s["mask"][first:first + k].tolist()
        seen = torch.tensor([[m >> j & 1 for j in range(k)] for m in masks], dtype=torch.bool, device=device).view(k, k)
        for g in range(hkv):
            key = torch.zeros((n, HEAD_DIM), dtype=torch.float64, device=device)
            value = torch.zeros_like(key)
            for total, codes, book in ((key, s["key_pages"], s["key_cb"]), (value, s["val_pages"], s["val_cb"])):
                chosen = codes[page, g, within].long()
                for m in range(book.shape[1]):
                    total += book[g, m].double().index_select(0, chosen[:, m])
            turned = paired(torch.cat((key, s["node_k"][first:first + k, g].double()))) * back
            value = torch.cat((value, s["node_v"][first:first + k, g].double()))
            for h in range(g * group, (g + 1) * group):
                q = paired(s["q"][first:first + k, h]) * back[n:]
                logits = (torch.matmul(q.real, turned.real.T) + torch.matmul(q.imag, turned.imag.T)) / math.sqrt(HEAD_DIM)
                logits[:, n:].masked_fill_(~seen, -math.inf)
                out[first:first + k, h] = torch.matmul(torch.softmax(logits, -1), value)
        first += k
    return out


def exact(case, seed):
    s = _inputs(case, seed)
    return {"tables": _exact_tables, "store": _exact_store, "tree": _exact_tree}[case["what"]](case, s)


def work(case):
    """Bytes: every input read once, every output written once.  Operations of attention: the codewords' sums, the keys' turns and
    the two products of every row with every token; none are counted for tables and copies."""
    if case["what"] == "tables":
        cached, new = _table_lengths(case)
        block, total = case["block"], sum(new)
        fresh = sum(_pages_of(c + n, block) - _pages_of(c, block) for c, n in zip(cached, new))
        # lengths in, lengths and offsets out, pages from the free list into the tables, slots and positions out
        return {"bytes": 4 * (4 * case["batch"] + 1 + 2 * fresh + 2 * total), "flops": 0}
    if case["what"] == "store":
        n = case["tokens"]
        kept = n - (_pages_of(n, case["skipped"]) if case["skipped"] else 0)
        return {"bytes": 4 * n + 2 * kept * (case["kv_heads"] * (case["m_key"] + case["m_val"]) + 4 * case["axes"]), "flops": 0}
    lens, nodes = _tree_lengths(case)
    hq, hkv, d, size = case["q_heads"], case["kv_heads"], HEAD_DIM, 2 if case["storage"] == "bf16" else 4
    tokens, total = sum(lens), sum(nodes)
    record = hkv * (case["m_key"] + case["m_val"]) + (4 * case["axes"] if case["axes"] > 1 else 0)
    nbytes = tokens * record + size * d * (total * (2 * hq + 2 * hkv) + hkv * WORDS * (case["m_key"] + case["m_val"]))
    pairs = sum(n * k for n, k in zip(lens, nodes))
    return {"bytes": nbytes, "flops": tokens * hkv * d * (case["m_key"] + case["m_val"] + 3) + 4 * pairs * hq * d}
