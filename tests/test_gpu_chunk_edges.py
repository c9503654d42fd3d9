"""Calls with several new tokens per sequence on the GPU, at the edges of their launches: refused
chunks, more key blocks than a wave holds page ids for, more heads and more vocabulary than one
wave's sums, and the bits of short chunks."""
import math

import numpy as np
import pytest
import torch

import oracle.chunk_oracle as CO
from hk_testlib import np64, np_i
from test_gpu_chunk import DEV, I32, Cache, _attend, _bound, _check_attn, _chunks, _reserve, _verify

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ refused chunks
@pytest.mark.parametrize("graph", [False, True])
def test_a_refused_chunk_takes_nothing_back(graph):
    """Drafts whose slots were refused (pool too small, a row full, starts out of bounds) are not
    trimmed: tables, masks, counts and free list stay, no token is drawn.  A granted chunk of the same
    loop before, between and after them is tested and trimmed as ever."""
    import paper_2606_28831_amd as hk
    from paper_2606_28831_amd.pipeline import DecodeLoop, Verifier
    L, B, Hkv, G, D, V, T = 2, 3, 2, 2, 64, 33, 60
    Hq, bf = Hkv * G, torch.bfloat16
    c = Cache([30 + 3 * h for h in range(L * B * Hkv)], D, "bf16", seed=2, width=6, spare=14)
    loop = DecodeLoop(L, B, Hq, Hkv, D, 8, c.kv, c.alloc, 0.9, 32, max_tokens=T, max_len=50)
    ver = Verifier(B, V, DEV)
    start = torch.zeros(B + 1, dtype=I32, device=DEV)
    ch = hk.Chunks(start, T, 50)
    q, o = (torch.randn(L, T, Hq, D, device=DEV).to(bf) for _ in "qo")
    k, v = (torch.randn(L, T, Hkv, D, device=DEV).to(bf) for _ in "kv")
    lse = torch.zeros(L, T, Hq, device=DEV)
    p = torch.zeros(T, V, device=DEV)
    p[:, 5] = 1.0
    tok, u = torch.full((T,), 5, dtype=I32, device=DEV), torch.full((T,), 0.5, device=DEV)
    out = [torch.full((B,), -77, dtype=I32, device=DEV) for _ in range(3)]

    def step():
        loop.extend(ch, q, k, v, o, lse)
        loop.accept(ver, ch, tok, p, u, *out)
    if graph:
        captured = torch.cuda.CUDAGraph()
        with torch.cuda.graph(captured):
            step()
    for starts, flag in (([0, 3, 4, 6], 0), ([0, 20, 40, 59], hk.FLAG_NOSPACE), ([0, 2, 6, 7], 0),
                         ([0, 0, 0, 50], hk.FLAG_NOSPACE), ([0, 9, 5, 8], hk.FLAG_CHUNK), ([0, 1, 61, 62], hk.FLAG_CHUNK),
                         ([0, 4, 8, 12], 0)):
        start.copy_(torch.tensor(starts, device=DEV).to(I32))
        loop.status.zero_()
        tok.fill_(5)
        tok[2], tok[5], tok[11] = 4, 4, 4                # some drafts are rejected
        captured.replay() if graph else step()
        torch.cuda.synchronize()
        assert int(loop.status.item()) == flag, starts
        got = [np_i(x).tolist() for x in out]
        if flag:
            assert got == [[0] * B, [-1] * B, [0] * B], starts
        else:
            lens = [b - a for a, b in zip(starts, starts[1:])]
            want = [CO.verify(np_i(tok)[a:b], np64(p)[a:b], None, np_i(u)[a:b]) for a, b in zip(starts, starts[1:])]
            assert [tuple(x) for x in zip(*got)] == want, starts
            ok, c.t, c.m, c.n, c.top, _ = CO.reserve(c.t, c.m, c.n, c.free, c.top, lens, Hkv)
            assert ok
            c.t, c.m, c.n, c.free, c.top = CO.trim(c.t, c.m, c.n, c.free, c.top, got[2], Hkv)
        c.check(starts)


# ------------------------------------------------------------------ the bits of short chunks
@pytest.mark.parametrize("D,G,lens,ctx", [
    (128, 4, [1, 8, 3, 0], [0, 1, 500, 20]), (64, 8, [4, 1, 2], [3, 0, 900]),
    (128, 1, [1, 32, 1], [0, 2, 1500]), (64, 3, [10, 1], [0, 40])])
def test_short_chunks_keep_the_bits_of_their_probabilities(D, G, lens, ctx):
    """Drafts and single tokens of a bf16 cache are off by the rounding of their output and little else,
    as the framework's decode is: probabilities enter the product with V in two bf16 parts, off by half a
    step of the second, 2^-8 of the 2^-8 that the first leaves.  A query that sees one key has its V."""
    rows = [a + n for a, n in zip(ctx, lens) for _ in range(2)]
    c = Cache(rows, D, "bf16", holes=0.2, seed=40 + G, keep_last=max(lens))
    q, o, lse = _attend(c, lens, 2, G, D, "bf16")
    first = [sum(lens[:s]) for s in range(len(lens))]
    qn, on = np64(q), np64(o)
    for h in range(len(rows)):
        s, kv = divmod(h, 2)
        n, a, g = lens[s], first[s], slice(kv * G, kv * G + G)
        if n == 0:
            continue
        k, v, valid, end = c.head(h)
        ro, rl, zabs, absv = CO.chunk_attn_head(qn[a:a + n, g], k, v, valid, end, 1 / math.sqrt(D))
        dz, rest = (D + 8) * 2.0 ** -23 * zabs, (len(valid) / 32 + 64) * 2.0 ** -23
        bo = 2.0 ** -8 * np.abs(ro) * 1.01 + (2.0 ** -16 + 2 * dz[..., None] + 2 * rest) * 1.05 * absv
        assert (np.abs(on[a:a + n, g] - ro) <= bo).all(), h
        if valid[:end - n + 1].sum() == 1:
            assert (on[a, g] == v[np.nonzero(valid)[0][0]]).all()
