"""Steps of speculative decoding as a server makes them: prompts encoded and put into pages, drafted trees attended, the accepted path encoded
and appended, and again; every result against the definition in 64 bits over the codes that the encoder chose."""
import math

import pytest
import torch

import paper_2506_18879_amd as cv
from paper_2506_18879_amd.device import PagedCache, TreeAttention

from test_gpu_tree import D, NORM, tree

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("axes", [1, 3])
@pytest.mark.parametrize("prompts,drafts", [([40, 3, 129], [6, 1, 9]), ([9000, 20, 5100, 700], [3, 4, 2, 1]), ([6000, 50, 8000], [17, 20, 5])])
def test_prompts_drafts_and_accepted_paths(prompts, drafts, axes):
    Hkv, G, M = 4, 4, 16
    gen = torch.Generator(device="cuda")
    gen.manual_seed(sum(prompts))
    normal = lambda *s, std=1.0: (torch.randn(s, generator=gen, device="cuda") * std).to(torch.bfloat16)
    cfg = cv.Config(Hkv * G, Hkv, D, M, M, 256, 1, 1, 5e5, 0.0, 1 << 15, cv.COMMVQ_KEYS_INDEXED, 0, 0, cv.COMMVQ_VALUES_INDEXED, 0)
    h = cv.commvq_create(cfg)
    st = torch.cuda.current_stream().cuda_stream
    kcb, vcb = normal(Hkv, M, 256, D, std=M ** -0.5), normal(Hkv, M, 256, D, std=M ** -0.5)
    ktab, vtab = (torch.empty(f(h), dtype=torch.uint8, device="cuda") for f in (cv.commvq_encoder_table_bytes, cv.commvq_value_encoder_table_bytes))
    cv.commvq_encoder_prepare(h, kcb, ktab, st)
    cv.commvq_value_encoder_prepare(h, vcb, vtab, st)

    def encode(keys, vals):
        out = []
        for x, f, cb, tab in ((keys, cv.commvq_encode_keys, kcb, ktab), (vals, cv.commvq_encode_values, vcb, vtab)):
            codes = torch.empty((len(x), Hkv, M), dtype=torch.uint8, device="cuda")
            f(h, x, len(x), cb, tab, codes, Hkv * M, M, st)
            out.append(codes)
        return out

    B = len(prompts)
    blocks = sum(-(-(n + 40) // 16) for n in prompts) + 2
    cache = PagedCache(cfg, h, blocks, 16, B, max(-(-(n + 40) // 16) for n in prompts), axes)
    attn = TreeAttention(cfg, h, kcb, vcb)
    axis = None if axes == 1 else [0] * 16 + [1] * 24 + [2] * 24
    place = lambda n, first: torch.stack([torch.arange(first, first + n) // (1, 3, 2)[a] + 7 * a for a in range(axes)], 1).int()
    theta = 5e5 ** (-torch.arange(64, dtype=torch.float64, device="cuda") / 64)
    which = torch.tensor(axis or [0] * 64, device="cuda")

    def turn(x, pos):
        a = pos.double().cuda()[:, which] * theta
        c, s = a.cos()[:, None], a.sin()[:, None]
        u, v = x[..., 0::2], x[..., 1::2]
        return torch.stack((u * c + v * s, v * c - u * s), -1).flatten(-2)

    def decode(codes, cb):
        x = torch.zeros(codes.shape[:2] + (D,), dtype=torch.float64, device="cuda")
        for g in range(Hkv):
            for m in range(M):
                x[:, g] += cb[g, m].double()[codes[:, g, m].long()]
        return x

    held = [[torch.empty((0, Hkv, M), dtype=torch.uint8, device="cuda")] * 2 + [torch.empty((0, axes), dtype=torch.int32)] for _ in range(B)]

    def append(parts):                                 # parts[b] = keys, values, positions of its new tokens
        keys, vals = (torch.cat([p[i] for p in parts]) for i in range(2))
        pos = torch.cat([p[2] for p in parts])
        if len(keys):
            kc, vc = encode(keys, vals)
            at = 0
            for b, p in enumerate(parts):
                n = len(p[0])
                held[b] = [torch.cat((held[b][0], kc[at:at + n])), torch.cat((held[b][1], vc[at:at + n])), torch.cat((held[b][2], p[2]))]
                at += n
            cache.append([len(p[0]) for p in parts], kc, vc, pos.cuda())

    append([(normal(n, Hkv, D), normal(n, Hkv, D), place(n, 0)) for n in prompts])
    for step in range(3):
        masks = [tree(k, step + b) for b, k in enumerate(drafts)]
        N = sum(drafts)
        q, nk, nv = normal(N, Hkv * G, D), normal(N, Hkv, D), normal(N, Hkv, D)
        pos = torch.cat([torch.cat([place(1, n + bin(m).count("1") - 1) for m in ms]) for n, ms in zip(cache.lens, masks)])
        out = attn(cache, q, nk, nv, drafts, pos.cuda(), torch.tensor([m for ms in masks for m in ms], dtype=torch.int64, device="cuda"), axis)
        torch.cuda.synchronize()
        assert cache.seq_lens.tolist() == cache.lens == [len(x[0]) for x in held]
        want = torch.zeros((N, Hkv * G, D), dtype=torch.float64, device="cuda")
        first, accepted = 0, []
        for b, ms in enumerate(masks):
            mine = slice(first, first + len(ms))
            # (with one axis the cache keeps no positions: token i is at i, as place() has it)
            keys = torch.cat((turn(decode(held[b][0], kcb), held[b][2]), turn(nk[mine].double(), pos[mine])))
            vals = torch.cat((decode(held[b][1], vcb), nv[mine].double()))
            tq, c = turn(q[mine].double(), pos[mine]), len(held[b][0])
            for i, m in enumerate(ms):
                at = torch.tensor(list(range(c)) + [c + j for j in range(len(ms)) if m >> j & 1], device="cuda")
                logits = torch.bmm(tq[i].view(Hkv, G, D), keys[at].permute(1, 2, 0).contiguous()) / math.sqrt(D)
                want[first + i] = torch.bmm(torch.softmax(logits, -1), vals[at].permute(1, 0, 2).contiguous()).view(Hkv * G, D)
            path = [j for j in range(len(ms)) if ms[-1] >> j & 1]   # what the last node attends to is accepted
            rows = torch.tensor([first + j for j in path], device="cuda")
            accepted.append((nk[rows], nv[rows], pos[rows.cpu()]))
            first += len(ms)
        assert float((out.double() - want).norm() / want.norm()) <= NORM
        append(accepted)
        if step == 1:                                  # the first sequence ends, another one takes its place and its pages
            cache.release(0)
            held[0] = [x[:0] for x in held[0]]
            append([(normal(n, Hkv, D), normal(n, Hkv, D), place(n, 0)) for n in [prompts[0] // 2] + [0] * (B - 1)])
    with pytest.raises(RuntimeError):
        cache.append([10 ** 6] + [0] * (B - 1), None, None)
    codes = torch.zeros((2, Hkv, M), dtype=torch.uint8, device="cuda")
    one = [1] + [0] * (B - 1)
    for new, k, v in (([-1] + [0] * (B - 1), None, None), (one, codes, codes), (one, codes[:1], None), (one, codes[:1].int(), codes[:1]), ([1], codes[:1], codes[:1])):
        with pytest.raises(ValueError):
            cache.append(new, k, v, place(1, 0).cuda())
    assert attn(cache, q[:0], nk[:0], nv[:0], [0] * B, pos[:0].cuda()).shape == (0, Hkv * G, D)
    for bad in (q.float(), q[:-1], q.transpose(0, 1).contiguous().transpose(0, 1), q.cpu()):
        with pytest.raises(ValueError):
            attn(cache, bad, nk, nv, drafts, pos.cuda())
    cv.commvq_destroy(h)
