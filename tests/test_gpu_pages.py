"""Block tables and slots from the requests' lengths, and stores into pages: whole numbers and bytes, equal to a scheduler written out on the host."""
import random

import pytest
import torch

import paper_2506_18879_amd as cv

pytestmark = pytest.mark.gpu


def plain(block, n_blocks, cached, new, free, table, n_slots):
    table = [list(r) for r in table]
    width = len(table[0])
    asked = first = 0
    lens, cu, slots, pos, taken, refused = [], [0], [], [], 0, 0
    for b, (c, n) in enumerate(zip(cached, new)):
        c, n = max(c, 0), max(n, 0)
        held, after = -(-c // block), -(-(c + n) // block)
        fits = after <= width and c + n < 2 ** 31
        need = after - held if fits else 0
        ok = fits and (need == 0 or asked + need <= len(free)) and first + n <= n_slots
        if ok:
            for i in range(need):
                table[b][held + i] = free[asked + i]
            taken += need
        refused += not ok
        asked += need
        for t in range(c, min(c + n, c + max(0, n_slots - first))):
            page = table[b][t // block] if ok else -1
            slots.append(page * block + t % block if 0 <= page < n_blocks else -1)
            pos.append(min(t, 2 ** 31 - 1))
        first += n
        lens.append(c + n if ok else c)
        cu.append(first)
    return table, lens, cu, slots + [-1] * (n_slots - len(slots)), pos, [taken, refused]


def run(block, n_blocks, cached, new, free, table, n_slots, want_pos=True):
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    B, width = len(cached), len(table[0])
    d = {"table": dev(table), "lens": torch.full((B,), 99, dtype=torch.int32, device="cuda"), "cu": torch.full((B + 1,), 99, dtype=torch.int32, device="cuda"),
         "slots": torch.full((n_slots + 1,), 99, dtype=torch.int32, device="cuda"), "pos": torch.full((n_slots + 1,), 99, dtype=torch.int32, device="cuda"),
         "taken": dev([99, 99]), "cached": dev(cached), "new": dev(new), "free": dev(free)}
    def call():
        cv.commvq_page_tables(cv.make_pages(block, n_blocks, width), B, d["cached"], d["new"], d["free"] if free else None, len(free), d["table"], d["lens"], d["cu"],
                              d["slots"] if n_slots else None, d["pos"] if want_pos else None, n_slots, d["taken"], torch.cuda.current_stream().cuda_stream)
    call()
    torch.cuda.synchronize()
    want = plain(block, n_blocks, cached, new, free, table, n_slots)
    check(d, want, n_slots, want_pos)
    return d, call, want


def check(d, want, n_slots, want_pos=True):
    table, lens, cu, slots, pos, taken = want
    assert d["table"].tolist() == table and d["lens"].tolist() == lens and d["cu"].tolist() == cu and d["taken"].tolist() == taken
    assert d["slots"].tolist() == slots + [99]
    assert d["pos"].tolist() == (pos if want_pos else []) + [99] * (n_slots + 1 - (len(pos) if want_pos else 0))


def start(r, B, block, most, width=None):
    cached = [r.choice((0, 1, block - 1, block, r.randrange(most + 1))) for _ in range(B)]
    held = [-(-c // block) for c in cached]
    width = width or max(held) + 4
    ids = list(range(sum(held) + 4000))
    r.shuffle(ids)
    table, at = [], 0
    for h in held:
        table.append(ids[at:at + h] + [-7] * (width - h))
        at += h
    return cached, table, ids[at:], len(ids)


@pytest.mark.parametrize("block", [16, 64, 1024])
@pytest.mark.parametrize("B", [1, 2, 63, 65, 1023, 1024, 1025, 2500])
def test_tables(B, block):
    r = random.Random(B + block)
    cached, table, free, pool = start(r, B, block, 3 * block)
    new = [r.choice((0, 0, 1, 1, 5, r.randrange(2 * block))) for _ in range(B)]
    run(block, pool, cached, new, free, table, sum(new) + r.choice((0, 1, 3000)))


def test_prompts_of_many_workgroups():
    run(16, 5000, [0, 7, 0], [30001, 0, 20000], list(range(4999, 0, -1)), [[0] + [-1] * 2000] * 3, 50001)
    run(16, 5000, [0], [1], [3], [[-1]], 1)
    run(16, 5000, [15], [1], [], [[4]], 1)
    run(16, 5000, [16], [0], [], [[4]], 0)


def test_requests_that_do_not_fit():
    r = random.Random(4)
    for trial in range(20):
        B = r.choice((3, 40, 1100))
        cached, table, free, pool = start(r, B, 16, 60, width=6)
        new = [r.choice((0, 1, 17, 60, -3)) for _ in range(B)]
        total = sum(max(n, 0) for n in new)
        run(16, pool, cached, new, free[:r.choice((0, 1, 5, B))], table, r.choice((total, total // 2, 0)))


def test_pages_outside_the_pool_and_lengths_that_overflow():
    run(16, 10, [16, 0, 3], [4, 20, 1], [9, 10, -1, 11, 2], [[3, 0, 0], [0, 0, 0], [-5, 0, 0]], 30)
    big = 2 ** 31 - 1
    d, _, want = run(16, 10, [big - 3, 5, big], [0, 2, 0], [1], [[1, 2]] * 3, 4)
    assert d["lens"].tolist() == [big - 3, 7, big]
    run(1024, 10, [big - 5, 5], [10, 2], [1, 2], [[0] * (2 ** 21 + 1)] * 2, 16)   # a length that 32 bits do not hold, in a row that is long enough


def test_positions_are_optional_and_calls_repeat():
    r = random.Random(9)
    cached, table, free, pool = start(r, 50, 32, 100)
    new = [r.randrange(70) for _ in range(50)]
    n = sum(new) + 5
    d, call, want = run(32, pool, cached, new, free, table, n, want_pos=False)
    d, call, want = run(32, pool, cached, new, free, table, n)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):                                 # the same inputs, the same outputs
        d["slots"][:n], d["lens"][:], d["taken"][:] = 5, 5, 5
        graph.replay()
        torch.cuda.synchronize()
        check(d, want, n)


@pytest.mark.parametrize("Hkv,Mk,Mv,axes", [(8, 16, 16, 1), (8, 32, 16, 3), (1, 16, 16, 4), (3, 16, 32, 2)])
@pytest.mark.parametrize("n,block", [(1, 16), (5, 16), (1000, 64), (3001, 1024)])
def test_stores(Hkv, Mk, Mv, axes, n, block):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(n + Hkv)
    pool = n // block + 3
    slots = torch.randperm(pool * block, generator=gen, device="cuda")[:n].int()
    slots[::7], slots[3::11] = -1, pool * block
    slots[n - 1] = pool * block - 1 if not bool((slots == pool * block - 1).any()) else slots[n - 1]
    codes = lambda *s: torch.randint(0, 256, s, generator=gen, device="cuda", dtype=torch.uint8)
    keys, vals, kp, vp = codes(n, Hkv, Mk), codes(n, Hkv, Mv), codes(pool, Hkv, block, Mk), codes(pool, Hkv, block, Mv)
    pos = torch.randint(-9, 9, (n, axes), generator=gen, device="cuda", dtype=torch.int32)
    pp = torch.full((pool * block, axes), 99, dtype=torch.int32, device="cuda")
    wk, wv, wp = kp.clone(), vp.clone(), pp.clone()
    for t, s in enumerate(slots.tolist()):
        if 0 <= s < pool * block:
            wk[s // block, :, s % block], wv[s // block, :, s % block], wp[s] = keys[t], vals[t], pos[t]
    h = cv.commvq_create(cv.Config(Hkv, Hkv, 128, Mk, Mv, 256, 1, 1, 5e5, 0.0, 1000, 0, 0, 0, 0, 0))
    pages, st = cv.make_pages(block, pool, 1, axes), torch.cuda.current_stream().cuda_stream
    k2, v2 = kp.clone(), vp.clone()
    cv.commvq_store_pages(h, pages, n, slots, keys, vals, None, k2, v2, None, st)
    cv.commvq_store_pages(h, pages, n, slots, keys, vals, pos, kp, vp, pp, st)
    torch.cuda.synchronize()
    cv.commvq_destroy(h)
    assert torch.equal(kp, wk) and torch.equal(vp, wv) and torch.equal(pp, wp) and torch.equal(k2, wk) and torch.equal(v2, wv)


def test_stores_beyond_32_bit_offsets():
    """Pages past 4 GiB of the pool."""
    block, Hkv, M = 1024, 8, 32
    pool = (5 << 30) // (block * Hkv * M)
    kp, vp = (torch.zeros((pool, Hkv, block, M), dtype=torch.uint8, device="cuda") for _ in range(2))
    slots = torch.tensor([pool * block - 1, pool * block - 1024, 0, (pool - 30) * block + 5], dtype=torch.int32, device="cuda")
    keys = torch.randint(0, 256, (4, Hkv, M), device="cuda", dtype=torch.uint8)
    h = cv.commvq_create(cv.Config(Hkv, Hkv, 128, M, M, 256, 1, 1, 5e5, 0.0, 1000, 0, 0, 0, 0, 0))
    cv.commvq_store_pages(h, cv.make_pages(block, pool, 1), 4, slots, keys, keys, None, kp, vp, None, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    cv.commvq_destroy(h)
    for t, s in enumerate(slots.tolist()):
        assert torch.equal(kp[s // block, :, s % block], keys[t]) and torch.equal(vp[s // block, :, s % block], keys[t])
    assert int(kp.view(-1).count_nonzero()) == int(keys.count_nonzero())
