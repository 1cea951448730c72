"""Attention of drafted trees over a paged cache, against the definition in 64 bits (decode, turn, softmax, sum, row by row of the tables).

Tolerances.  u = eps / 2 is a rounding's largest relative error.  bf16 results are rounded once to bf16 (u = 2^-8); on the way turned queries and
keys, weights and values are rounded to fp16 (h = 2^-11) or to two bf16 parts (less).  Errors of queries and keys enter a logit with at most
2h Sum_d |q_d k_d| scale =: D, a normalised weight is then off by at most the factor exp(2 D) (1 + h)^2 (and 2^-32 of the largest weight a token, less than another
h for the 70 001 tokens here), an element before its last rounding by E = (exp(2 D) (1 + h)^3 - 1) Sum p |v|, after it by E + u (|out| + E).
Taken together the errors are independent, u / sqrt(3) and h / sqrt(3) each in the root mean square if evenly spread: sqrt(u^2 + 4 h^2) / sqrt(3) = 2.33e-3 of the
results' norm (logits are of unit variance here); twice that is the bound of the norm.  fp32 results: sums of at most 128 + 32 terms a logit and 2^13
terms a result, 2^-24 each and random in sign, stay below 2^-24 (13 * 8 + 91) = 1.2e-5 of the norm, and four times that in any element relative to Sum p |v|."""
import math

import pytest
import torch

import paper_2506_18879_amd as cv

pytestmark = pytest.mark.gpu
D, U, H = 128, 2.0 ** -8, 2.0 ** -11
NORM = 2 * math.sqrt((U * U + 4 * H * H) / 3)


def _axis_map(axes):
    return [0] * 64 if axes == 1 else [j * axes // 64 for j in range(64)]


class Case:
    """A batch: lens[b] cached tokens and masks[b] = the node masks (Python ints) of sequence b."""

    def __init__(self, lens, masks, Hkv=2, G=4, Mk=16, Mv=16, block=16, axes=1, q="bf16", cb="bf16", key_pos=None, position_free=False, seed=0, spare=3, base=5e5,
                 max_position=1 << 15, node_pos=None, tables=True):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        kind = {"bf16": torch.bfloat16, "f32": torch.float32}
        self.lens, self.masks, self.Hkv, self.G, self.block, self.axes, self.base = list(lens), masks, Hkv, G, block, axes, base
        self.nodes = [len(m) for m in masks]
        self.B, self.N, self.turn = len(lens), sum(self.nodes), not position_free
        dtype = lambda s: cv.COMMVQ_BF16 if s == "bf16" else cv.COMMVQ_F32
        self.cfg = cv.Config(Hkv * G, Hkv, D, Mk, Mv, 256, dtype(q), dtype(cb), base, 0.0, max_position, cv.COMMVQ_KEYS_INDEXED, 0, int(position_free),
                             cv.COMMVQ_VALUES_INDEXED, 0)
        held = [-(-n // block) for n in self.lens]
        self.pool, self.width = sum(held) + spare, max(1, max(held))
        order = torch.randperm(self.pool, generator=gen, device="cuda").int().cpu()
        self.table = torch.full((self.B, self.width), -1, dtype=torch.int32)
        at = 0
        for b, h in enumerate(held):
            self.table[b, :h] = order[at:at + h]
            at += h
        normal = lambda shape, t, std=1.0: (torch.randn(shape, generator=gen, device="cuda") * std).to(kind[t])
        codes = lambda m: torch.randint(0, 256, (self.pool, Hkv, block, m), generator=gen, device="cuda", dtype=torch.uint8)
        self.key_pages, self.val_pages = codes(Mk), codes(Mv)
        self.key_cb, self.val_cb = (normal((Hkv, m, 256, D), cb, m ** -0.5) for m in (Mk, Mv))
        self.q = normal((max(1, self.N), Hkv * G, D), q)
        self.node_k, self.node_v = (normal((max(1, self.N), Hkv, D), q) for _ in range(2))
        self.out = torch.full_like(self.q, 77.0)
        self.key_pos = None if key_pos is None else key_pos(gen, self.pool * block, axes)
        if node_pos is None:
            node_pos = [[n + bin(m & ((1 << i) - 1)).count("1")] * axes for n, ms in zip(self.lens, masks) for i, m in enumerate(ms)]
        self.node_pos = torch.tensor(node_pos, dtype=torch.int32).view(-1, axes)
        self.tables_wanted = tables and q == cb == "bf16"
        self.q_stride = self.node_stride = 0
        self.more = {}

    def call(self, handle=None, mask="own", total=None, max_len=None):
        h = handle or cv.commvq_create(self.cfg)
        dev = lambda x: torch.as_tensor(x, dtype=torch.int32).cuda()
        cu = [0]
        for n in self.nodes:
            cu.append(cu[-1] + n)
        flat = [m - (1 << 64) if m >> 63 else m for ms in self.masks for m in ms]
        self.d = {"lens": dev(self.lens), "table": self.table.cuda(), "cu": dev(cu), "pos": self.node_pos.cuda(), "mask": torch.tensor(flat or [0], dtype=torch.int64).cuda()}
        total, max_len = total or self.N, max(self.lens) if max_len is None else max_len
        pages = cv.make_pages(self.block, self.pool, self.width, self.axes)
        tree = cv.make_tree(self.B, total, max(self.nodes), max_len, self.d["lens"], self.d["table"], self.d["cu"], self.d["pos"],
                            self.d["mask"] if mask == "own" else None, self.key_pos, _axis_map(self.axes) if self.axes > 1 else None, self.q_stride, self.node_stride, **self.more)
        tables = None
        if self.tables_wanted:
            tables = torch.empty(cv.commvq_tree_table_bytes(h), dtype=torch.uint8, device="cuda")
            cv.commvq_tree_prepare(h, self.key_cb, self.val_cb, tables, torch.cuda.current_stream().cuda_stream)
        ws = torch.full((cv.commvq_tree_workspace_bytes(h, self.B, total, max(self.nodes), max_len),), 255, dtype=torch.uint8, device="cuda")
        self.kept = (tables, ws, tree, pages, h)
        self.again = lambda stream=None: cv.commvq_tree_attn(h, pages, tree, self.q, self.node_k, self.node_v, self.key_pages, self.val_pages, self.key_cb,
                                                             self.val_cb, tables, self.out, ws, ws.numel(), stream or torch.cuda.current_stream().cuda_stream)
        self.again()
        torch.cuda.synchronize()
        if handle is None:
            cv.commvq_destroy(h)
        return self.out

    def plain(self, masks=None):
        """(result, Sum p |v|, D of the head comment), all [N][Hq][d] in float64; D is [N][Hq][1]."""
        theta = self.base ** (-torch.arange(64, dtype=torch.float64, device="cuda") / 64)
        axis = torch.tensor(_axis_map(self.axes), device="cuda")
        shape = (self.N, self.Hkv * self.G, D)
        out, mass, slack = torch.zeros(shape, dtype=torch.float64, device="cuda"), torch.zeros(shape, dtype=torch.float64, device="cuda"), torch.zeros(shape[:2] + (1,), dtype=torch.float64, device="cuda")

        def turn(x, pos):
            if not self.turn:
                return x
            angle = pos.double().cuda()[:, axis] * theta
            c, s = angle.cos()[:, None], angle.sin()[:, None]
            a, b = x[..., 0::2], x[..., 1::2]
            return torch.stack((a * c + b * s, b * c - a * s), -1).flatten(-2)

        first = 0
        for b, n in enumerate(self.lens):
            k = self.nodes[b]
            tok = torch.arange(n)
            page = self.table[b].long()[tok // self.block]
            keep = (page >= 0) & (page < self.pool)
            tok, page = tok[keep], page[keep].cuda()
            within = (tok % self.block).cuda()
            def decode(pages, cb):
                c = pages[page, :, within].long()                                                # [n][Hkv][M]
                x = torch.zeros(c.shape[:2] + (D,), dtype=torch.float64, device="cuda")
                for g in range(self.Hkv):
                    for m in range(cb.shape[1]):
                        x[:, g] += cb[g, m].double()[c[:, g, m]]
                return x
            mine = slice(first, first + k)
            first += k
            pos = tok[:, None].expand(-1, self.axes) if self.key_pos is None else self.key_pos[page * self.block + within].cpu()
            keys = torch.cat((turn(decode(self.key_pages, self.key_cb), pos), turn(self.node_k[mine].double(), self.node_pos[mine])))
            vals = torch.cat((decode(self.val_pages, self.val_cb), self.node_v[mine].double()))
            q = turn(self.q[mine].double(), self.node_pos[mine])
            c = len(tok)
            for i, bits in enumerate((masks or self.masks)[b]):
                see = [j for j in range(k) if bits >> j & 1]
                if c + len(see) == 0:
                    continue
                at = torch.tensor(list(range(c)) + [c + j for j in see], device="cuda")
                for h in range(self.Hkv * self.G):
                    kk, vv = keys[at, h // self.G], vals[at, h // self.G]
                    p = torch.softmax(kk @ q[i, h] / math.sqrt(D), 0)
                    out[mine][i, h] = p @ vv
                    mass[mine][i, h] = p @ vv.abs()
                    slack[mine][i, h] = (kk.abs() @ q[i, h].abs()).max() / math.sqrt(D)
        return out, mass, 2 * H * slack

    def check(self, got=None, masks=None):
        got = (self.out if got is None else got)[:self.N].double()
        want, mass, d = self.plain(masks)
        err = (got - want).abs()
        norm = float((got - want).norm() / want.norm().clamp(min=1e-300)) if float(want.norm()) else float(err.max())
        if self.out.dtype == torch.bfloat16:
            before = ((2 * d).exp() * (1 + H) ** 3 - 1) * mass
            fits = bool((err <= before + U * (want.abs() + before)).all())
            assert fits, float((err / mass.clamp(min=1e-30)).max())
            assert norm <= NORM, norm
        else:
            fits = bool((err <= 4 * 1.2e-5 * mass + 1e-30).all())
            assert fits, float((err / mass.clamp(min=1e-30)).max())
            assert norm <= 1.2e-5, norm


def chain(n):
    return [(1 << (i + 1)) - 1 for i in range(n)]


def tree(n, seed=0):
    import random
    r, out = random.Random(seed * 100 + n), []
    for i in range(n):
        out.append((out[r.randrange(i)] if i else 0) | 1 << i)
    return out


@pytest.mark.parametrize("G", [1, 2, 4, 8])
@pytest.mark.parametrize("Mk,Mv", [(16, 16), (32, 16), (16, 32), (32, 32)])
def test_heads_and_codebooks(G, Mk, Mv):
    c = Case([0, 1, 77, 300], [tree(3), tree(9), tree(1), tree(17)], G=G, Mk=Mk, Mv=Mv, seed=G + Mk + Mv)
    c.call()
    c.check()


@pytest.mark.parametrize("n", [1, 15, 16, 17, 31, 32, 33, 64, 65, 511, 512, 513, 1023, 1025, 2049, 4097])
@pytest.mark.parametrize("k", [1, 5, 64])
def test_lengths(n, k):
    c = Case([n], [tree(k)], Hkv=1, G=2, seed=n + k)
    c.call()
    c.check()


@pytest.mark.parametrize("k,G", [(4, 4), (5, 4), (8, 4), (9, 4), (16, 4), (17, 4), (32, 4), (33, 4), (64, 4), (33, 8), (64, 8)])
def test_rows_of_workgroups(k, G):
    c = Case([200, 40], [tree(k), tree(max(1, k // 3))], Hkv=1, G=G, seed=k * G)
    c.call()
    c.check()


@pytest.mark.parametrize("block", [16, 32, 256, 1024])
def test_page_sizes(block):
    c = Case([1500, 3, 0, 999], [tree(4), tree(2), tree(3), tree(8)], block=block, Mk=32, seed=block)
    c.call()
    c.check()


@pytest.mark.parametrize("q,cb", [("f32", "f32"), ("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("lens,ks", [([700], [5]), ([0, 33, 16], [1, 20, 3])])
def test_types(q, cb, lens, ks):
    c = Case(lens, [tree(k) for k in ks], Hkv=2, G=4, Mk=32, Mv=16, q=q, cb=cb, seed=len(lens))
    c.call()
    c.check()


@pytest.mark.parametrize("q", ["bf16", "f32"])
@pytest.mark.parametrize("axes", [2, 3, 4])
def test_positions_of_several_axes(axes, q):
    where = lambda gen, n, a: torch.randint(-3000, 3000, (n, a), generator=gen, device="cuda", dtype=torch.int32)
    pos = [[(7 * i + 100 * a) - 900 for a in range(axes)] for i in range(9 + 2)]
    for key_pos in (where, None):
        c = Case([500, 90], [tree(9), tree(2)], axes=axes, q=q, cb=q, key_pos=key_pos, node_pos=pos, seed=axes)
        c.call()
        c.check()


@pytest.mark.parametrize("q", ["bf16", "f32"])
def test_explicit_positions_on_both_sides_of_the_nodes(q):
    c = Case([700], [tree(6)], q=q, cb=q, key_pos=lambda gen, n, a: torch.randint(0, 30000, (n, a), generator=gen, device="cuda", dtype=torch.int32),
             node_pos=[[15000 + 3 * i] for i in range(6)], seed=5)
    c.call()
    c.check()


def test_far_positions():
    # positions near 2^31: only distances matter
    top = 2 ** 31 - 1 - 5000
    c = Case([300], [chain(4)], key_pos=lambda gen, n, a: top + torch.randint(0, 4000, (n, a), generator=gen, device="cuda", dtype=torch.int32),
             node_pos=[[top + 4000 + i] for i in range(4)], seed=6)
    c.call()
    c.check()


@pytest.mark.parametrize("n", [40, 1500])
def test_position_free(n):
    c = Case([n], [tree(7)], position_free=True, seed=n)
    c.call()
    c.check()


def test_no_mask_is_a_chain():
    c = Case([100, 0], [chain(64), chain(3)], seed=8)
    c.call(mask=None)
    c.check()


def test_masks_that_leave_rows_empty_and_sequences_without_nodes():
    c = Case([0, 50, 0, 20], [[0, 2, 1], [], [0], [0, 0]], seed=9)
    c.call()
    c.check()
    assert not c.out[0].any() and not c.out[3].any()   # nothing cached, nothing named: zeros
    c.masks = [[m | ~0 << 3 & (1 << 64) - 1 for m in c.masks[0]]] + c.masks[1:]
    before = c.out.clone()
    c.call()                                           # bits past the last node
    assert torch.equal(before, c.out)


def test_what_masked_nodes_hold_does_not_matter():
    c = Case([33, 0], [tree(9), [1, 2, 4]], seed=10)
    c.call()
    want = c.out.clone()
    hidden = [i for i in range(9) if all(not m >> i & 1 for j, m in enumerate(c.masks[0]) if j != i)]
    i = hidden[-1]
    c.node_k[i], c.node_v[i] = float("nan"), float("inf")
    c.node_k[9 + 1], c.node_v[9 + 1] = float("-inf"), float("nan")
    c.call()
    rows = [r for r in range(12) if r not in (i, 10)]
    assert torch.equal(want[rows], c.out[rows])
    assert not torch.isfinite(c.out[i]).any() and not torch.isfinite(c.out[10]).any()


@pytest.mark.parametrize("n", [70, 77, 1500, 5001])
def test_codewords_that_no_counted_token_selects(n):
    # tails of pages, pages that are not there and rows past the context select infinities; no weight may touch them
    c = Case([n], [tree(5)], Hkv=1, seed=n, spare=1)
    c.key_cb[:, :, 0], c.val_cb[:, :, 0] = float("nan"), float("inf")
    c.key_pages.clamp_(min=1)
    c.val_pages.clamp_(min=1)
    last = int(c.table[0, (n - 1) // 16])
    c.key_pages[last, :, n % 16 or 16:], c.val_pages[last, :, n % 16 or 16:] = 0, 0
    c.key_pages[0], c.val_pages[0] = 0, 0
    c.table[0][c.table[0] == 0] = -1
    c.table[0, 1], c.table[0, 3] = c.pool, 2 ** 31 - 1
    c.call()
    c.check()


def test_context_without_a_single_page():
    c = Case([100, 700], [tree(3), tree(2)], seed=12)
    c.table[:] = -1
    c.call()
    c.check()


def test_strides_and_rows_behind_the_last_sequence():
    c = Case([100, 31], [tree(4), tree(3)], Hkv=2, G=4, seed=13)
    wide = torch.full((c.N + 2, 8 + 2 + 2, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:c.N, :8], wide[:c.N, 8:10], wide[:c.N, 10:] = c.q, c.node_k, c.node_v
    c.q, c.node_k, c.node_v = wide, wide.view(-1)[8 * D:], wide.view(-1)[10 * D:]
    c.q_stride = c.node_stride = 12 * D
    c.out = torch.full((c.N + 2, 8, D), 77.0, dtype=torch.bfloat16, device="cuda")
    c.call(total=7 + 1)                                # one row more than the sequences have
    assert bool((c.out[c.N:] == 77).all())
    c.q, c.node_k, c.node_v = wide[:, :8], wide[:, 8:10], wide[:, 10:]
    c.check()


def test_lengths_and_offsets_beyond_what_the_host_said_are_cut():
    """Device arrays that contradict the host's sizes: nothing outside the described buffers is touched."""
    c = Case([64, 10], [tree(3), tree(2)], seed=14)
    h = cv.commvq_create(c.cfg)
    want = c.call(handle=h).clone()
    c.d["lens"][0] = 1 << 30                           # counts as 64
    c.again()
    torch.cuda.synchronize()
    assert torch.equal(want, c.out)
    c.d["lens"][0], c.d["lens"][1], c.d["cu"][2] = 64, -5, 1 << 30   # no tokens; still two nodes
    c.again()
    torch.cuda.synchronize()
    c.lens[1] = 0
    c.check()
    cv.commvq_destroy(h)


@pytest.mark.parametrize("n,Hkv,k", [(900, 2, 6), (12400, 8, 3), (12400, 8, 7)])
def test_large_logits(n, Hkv, k):
    c = Case([n], [tree(k)], Hkv=Hkv, seed=15)
    c.q *= 30
    c.call()
    want, mass, d = c.plain()
    before = ((2 * d).exp() * (1 + H) ** 3 - 1) * mass
    fits = bool(((c.out.double() - want).abs() <= before + U * (want.abs() + before)).all())
    assert fits


def test_the_same_bits_from_call_to_call_and_on_another_stream():
    c = Case([3000, 200], [tree(20), tree(64)], Mk=32, seed=16)
    h = cv.commvq_create(c.cfg)
    want = c.call(handle=h).clone()
    side = torch.cuda.Stream()
    for _ in range(3):
        c.out.zero_()
        torch.cuda.synchronize()
        c.again(side.cuda_stream)
        side.synchronize()
        assert torch.equal(want, c.out)
    cv.commvq_destroy(h)


def test_captured_and_replayed():
    c = Case([1200, 7], [tree(10), tree(3)], seed=17)
    h = cv.commvq_create(c.cfg)
    want = c.call(handle=h).clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.again()
    for i in range(4):
        c.out.zero_()
        c.kept[1].fill_(i)                             # (nothing is expected of the workspace)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(want, c.out)
        c.again()
        torch.cuda.synchronize()
        assert torch.equal(want, c.out)
    c.d["lens"][0] = 300                               # what the graph reads may change between replays
    graph.replay()
    torch.cuda.synchronize()
    c.lens[0] = 300
    c.check()
    cv.commvq_destroy(h)


def test_single_nodes_agree_with_decode_attention_of_the_flat_cache():
    """A node that attends to the cache alone is commvq_decode_attn's query."""
    from paper_2506_18879_amd import synth
    from paper_2506_18879_amd.device import DecodeAttention, DeviceWorkload
    lens = [1000, 33, 1]
    w = synth.make_workload("paged", B=3, Hq=8, Hkv=2, seqlens=lens, Mk=16, Mv=16, dtype="bf16", seed=3)
    dw, op = DeviceWorkload(w), DecodeAttention(w, max_position=1 << 15)
    flat = op(dw).clone()
    c = Case(lens, [[0]] * 3, Hkv=2, G=4, node_pos=[[int(p)] for p in w.q_pos], seed=18)
    c.q, c.key_cb, c.val_cb = dw.q, dw.key_codebooks.view(2, 16, 256, D), dw.val_codebooks.view(2, 16, 256, D)
    at = 0
    for b, n in enumerate(lens):
        for pages, codes in ((c.key_pages, dw.key_codes), (c.val_pages, dw.val_codes)):
            mine = codes[at * 32:(at + n) * 32].view(2, n, 16)
            for i in range(n):
                pages[int(c.table[b, i // 16]), :, i % 16] = mine[:, i]
        at += n
    c.base = w.rope_base
    c.call()
    c.check()
    assert float((c.out.double() - flat.double()).norm() / flat.double().norm()) <= NORM
    op.close()


# ---- contexts long enough for the kernels that stream whole codebooks (up to 16 rows a KV head: in one go; more: decoded ahead, in passes)
@pytest.mark.parametrize("k,G", [(1, 1), (1, 8), (4, 4), (2, 8), (5, 4), (33, 1), (9, 8), (17, 8), (35, 8)])
def test_long_rows(k, G):
    c = Case([12300], [tree(k)], Hkv=8, G=G, seed=100 + k + G)
    c.call()
    c.check()


@pytest.mark.parametrize("k", [3, 20])
@pytest.mark.parametrize("Mk,Mv", [(32, 16), (16, 32), (32, 32)])
def test_long_codebooks(Mk, Mv, k):
    c = Case([12289], [tree(k)], Hkv=8, G=4, Mk=Mk, Mv=Mv, seed=Mk + Mv + k)
    c.call()
    c.check()


@pytest.mark.parametrize("most", [4, 12])
@pytest.mark.parametrize("block", [16, 1024])
def test_long_ragged(most, block):
    import random
    r = random.Random(most + block)
    lens = [0, 1, 2047, 2048, 2049, 4096, 4097, 0, 6143] + [r.randrange(5000) for _ in range(70)]
    ks = [r.randrange(0, most + 1) for _ in lens]
    ks[3] = most
    for sizes in ({}, {"total_tokens": sum(lens)}):
        c = Case(lens, [tree(k, i) for i, k in enumerate(ks)], Hkv=2, G=4, block=block, seed=most + block)
        c.more = sizes
        c.call()
        c.check()


@pytest.mark.parametrize("axes", [1, 2])
@pytest.mark.parametrize("k", [0, 40])
def test_long_sequences_without_nodes_at_either_end(k, axes):
    # (their first node's position would be in front of, or behind, what is there)
    kw = {} if axes == 1 else dict(axes=2, key_pos=lambda gen, n, a: torch.randint(0, 9000, (n, a), generator=gen, device="cuda", dtype=torch.int32))
    c = Case([5000, 9000, 3000, 0, 12000], [[], tree(5), tree(k), tree(3), []], Hkv=8, G=4, seed=k, **kw)
    c.call()
    c.check()


@pytest.mark.parametrize("k", [4, 10, 40])
def test_long_sequences_over_several_passes(k):
    # 16 tiles of 2048 tokens a pass for 8 heads: the first and the last sequence are in several
    c = Case([70001, 3000, 40000], [tree(k), tree(2), tree(min(3, k))], Hkv=8, G=1 if k == 40 else 2, block=64, max_position=1 << 17, seed=k)
    c.call()
    c.check()


@pytest.mark.parametrize("axes", [1, 3])
@pytest.mark.parametrize("k", [2, 30])
def test_long_explicit_positions(k, axes):
    where = lambda gen, n, a: torch.randint(-9000, 30000, (n, a), generator=gen, device="cuda", dtype=torch.int32)
    c = Case([13000], [tree(k)], Hkv=8, G=4, axes=axes, key_pos=where, node_pos=[[4000 + i + 50 * a for a in range(axes)] for i in range(k)], seed=k + axes)
    c.call()
    c.check()


@pytest.mark.parametrize("k", [3, 18])
@pytest.mark.parametrize("how", ["axes without stored positions", "far", "before the context", "position free"])
def test_long_positions(how, k):
    kw = {"axes without stored positions": dict(axes=2), "far": {}, "before the context": dict(node_pos=[[i - 500] for i in range(k)]), "position free": dict(position_free=True)}[how]
    if how == "far":
        top = 2 ** 31 - 1 - 20000
        kw = dict(key_pos=lambda gen, n, a: top + torch.randint(0, 14000, (n, a), generator=gen, device="cuda", dtype=torch.int32), node_pos=[[top + 14000 + i] for i in range(k)])
    c = Case([12500], [tree(k)], Hkv=8, G=4, seed=k, **kw)
    c.call()
    c.check()


@pytest.mark.parametrize("k", [3, 18])
def test_long_codewords_that_no_counted_token_selects(k):
    c = Case([13001, 20], [tree(k), tree(2)], Hkv=8, seed=k, spare=1)
    c.key_cb[:, :, 0], c.val_cb[:, :, 0] = float("nan"), float("inf")
    c.key_pages.clamp_(min=1)
    c.val_pages.clamp_(min=1)
    last = int(c.table[0, 13000 // 16])
    c.key_pages[last, :, 13001 % 16:], c.val_pages[last, :, 13001 % 16:] = 0, 0
    c.key_pages[0], c.val_pages[0] = 0, 0
    c.table[0][c.table[0] == 0] = -1
    c.table[0, 1], c.table[0, 300], c.table[0, 500:640] = c.pool, 2 ** 31 - 1, -5
    c.call()
    c.check()


@pytest.mark.parametrize("n,k", [(300, 3), (12500, 3), (12500, 18)])
@pytest.mark.parametrize("keys,vals", [(2.0 ** 100, 2.0 ** -110), (2.0 ** -90, 2.0 ** 60), (1.0, 2.0 ** 30)])
def test_codebooks_of_any_magnitude(n, k, keys, vals):
    """Sizes that only bf16's exponents hold; queries make up for the keys'."""
    c = Case([n], [tree(k)], Hkv=8, seed=k)
    c.key_cb, c.node_k, c.q = c.key_cb * keys, c.node_k * keys, c.q / keys
    c.val_cb, c.node_v = c.val_cb * vals, c.node_v * vals
    c.call()
    c.check()


@pytest.mark.parametrize("k", [3, 18])
def test_long_contexts_without_a_single_page(k):
    c = Case([12500, 700], [tree(k), tree(2)], Hkv=8, seed=k)
    c.table[:] = -1
    c.call()
    c.check()


@pytest.mark.parametrize("k", [4, 40])
def test_long_captured_and_replayed(k):
    c = Case([40000, 100], [tree(k), tree(3)], Hkv=8, G=2, block=64, max_position=1 << 16, seed=k)
    h = cv.commvq_create(c.cfg)
    want = c.call(handle=h).clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.again()
    for i in range(4):
        c.out.zero_()
        c.kept[1].fill_(255 - i)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(want, c.out)
        c.again()
        torch.cuda.synchronize()
        assert torch.equal(want, c.out)
    c.d["lens"][0] = c.lens[0] = 30000
    graph.replay()
    torch.cuda.synchronize()
    c.check()
    cv.commvq_destroy(h)


def test_codes_beyond_32_bit_offsets():
    """Pages past 4 GiB of the pool, short and long contexts."""
    for lens, k in (([500], 3), ([12400], 3), ([12400], 9)):
        c = Case(lens, [tree(k)], Hkv=8, G=4, Mk=32, Mv=32, block=1024, spare=(9 << 29) // (1024 * 8 * 32) + 1, seed=k)
        held = -(-lens[0] // 1024)
        c.table[0, :held] = torch.arange(c.pool - held, c.pool, dtype=torch.int32)
        assert c.key_pages.numel() > 1 << 32
        c.call()
        c.check()
        del c
        torch.cuda.empty_cache()


def test_random_batches():
    import random
    for seed in range(12):
        r = random.Random(seed)
        B = r.choice((1, 2, 5))
        lens = [r.choice((0, 1, r.randrange(40), r.randrange(400), r.randrange(3000))) for _ in range(B)]
        ks = [r.choice((0, 1, r.randrange(1, 65))) for _ in range(B)]
        ks[r.randrange(B)] = r.randrange(1, 65)
        axes = r.choice((1, 1, 3))
        c = Case(lens, [[r.getrandbits(64) for _ in range(k)] for k in ks], Hkv=r.choice((1, 2, 3)), G=r.choice((1, 2, 4, 8)), Mk=r.choice((16, 32)), Mv=r.choice((16, 32)),
                 block=r.choice((16, 64, 512)), axes=axes, tables=r.random() < 0.8, seed=seed,
                 key_pos=None if axes == 1 and r.random() < 0.5 else lambda gen, n, a: torch.randint(0, 9000, (n, a), generator=gen, device="cuda", dtype=torch.int32))
        c.call()
        c.check()
