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
