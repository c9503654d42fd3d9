"""Calls with several new tokens per sequence, on the CPU: the oracle's own pins, and what the C
entry points and their wrappers refuse before any launch."""
import ctypes as C
import math
from fractions import Fraction

import numpy as np
import pytest
import torch
from scipy.special import logsumexp, softmax

import oracle.chunk_oracle as CO


@pytest.fixture(scope="module")
def hk():
    import paper_2606_28831_amd as hk
    return hk


# ------------------------------------------------------------------ the oracle
def _cache(rng, H, width, pool):
    perm = rng.permutation(pool)
    t, m, n, at = np.full((H, width), -1, np.int64), np.zeros((H, width), np.int64), np.zeros(H, np.int64), 0
    for h in range(H):
        n[h] = rng.integers(0, width - 1)
        t[h, :n[h]] = perm[at:at + n[h]]
        m[h, :n[h]] = rng.integers(0, 1 << 16, n[h])
        at += n[h]
    free = np.zeros(pool, np.int64)
    free[:pool - at] = perm[at:]
    return t, m, n, free, pool - at


@pytest.mark.parametrize("seed", range(6))
def test_reserve_then_trim_is_nothing(seed):
    rng = np.random.default_rng(seed)
    Hkv, lens = 2, [int(x) for x in rng.integers(0, 40, 3)]
    t, m, n, free, top = _cache(rng, 12, 8, 400)
    ok, t1, m1, n1, top1, slots = CO.reserve(t, m, n, free, top, lens, Hkv)
    assert ok == (n1 != n).any() or ok
    if not ok:
        assert (t1 == t).all() and top1 == top
        return
    flat = [x for s in slots for x in s]
    assert len(set(flat)) == len(flat)
    for h in range(12):
        k = lens[(h // Hkv) % 3]
        assert bin(int(m1[h].sum() and sum(int(x) << (16 * i) for i, x in enumerate(m1[h])))).count("1") - \
            sum(bin(int(x)).count("1") for x in m[h]) == k == len(slots[h])
    live = {int(x) for h in range(12) for x in t1[h, :n1[h]]}
    assert len(live) == n1.sum() and live.isdisjoint(int(x) for x in free[:top1])
    if all(m[h, n[h] - 1] for h in range(12) if n[h]):       # (an empty newest page leaves with the trim)
        t2, m2, n2, free2, top2 = CO.trim(t1, m1, n1, free, top1, lens, Hkv)
        assert (t2 == t).all() and (m2 == m).all() and (n2 == n).all() and top2 == top and (free2[:top] == free[:top]).all()


def test_chunk_attention_against_scipy():
    rng = np.random.default_rng(3)
    S, n, G, D = 37, 5, 3, 8
    k, v, q = rng.normal(size=(S, D)), rng.normal(size=(S, D)), rng.normal(size=(n, G, D))
    valid = rng.random(S) < 0.8
    valid[-5:] = True
    o, lse, zabs, absv = CO.chunk_attn_head(q, k, v, valid, S, 0.3)
    for i in range(n):
        see = valid & (np.arange(S) <= S - n + i)
        z = np.where(see, 0.3 * q[i] @ k.T, -np.inf)
        np.testing.assert_allclose(lse[i], logsumexp(z, axis=1), rtol=1e-13)
        np.testing.assert_allclose(o[i], softmax(z, axis=1) @ v, rtol=1e-12, atol=1e-14)
    assert (absv >= np.abs(o) - 1e-15).all() and (zabs > 0).all()
    o, lse, _, _ = CO.chunk_attn_head(q, k[:2], v[:2], np.ones(2, bool), 2, 0.3)   # more queries than slots
    assert (o[:3] == 0).all() and np.isneginf(lse[:3]).all() and (o[3] == v[0]).all()


def test_draft_rule_draws_from_the_target():
    """Over all pairs of a fine grid of random numbers one draft's token follows p exactly: q's draws kept
    or replaced by the rest's."""
    p, q = [Fraction(a, 8) for a in (1, 4, 3)], [Fraction(a, 8) for a in (4, 1, 3)]
    out = [Fraction(0)] * 3
    n = 16
    for x in range(3):
        for a in range(n):
            for b in range(n):
                u = [b / n, a / n]
                kept, nxt, drop = CO.verify([0, x], [[float(y) for y in p]] * 2, [None, [float(y) for y in q]], u)
                assert kept + drop == 1
                out[x if kept else nxt] += q[x] / (n * n)
    assert out == p


@pytest.mark.parametrize("case,want", [
    (([5], [[0.0, 0.5, 0.5]], None, [0.0]), (0, 1, 0)),
    (([5], [[0.0, 0.5, 0.5]], None, [0.5]), (0, 2, 0)),
    (([5], [[0.0, 0.0, 0.0]], None, [0.5]), (0, -1, 0)),
    (([5, 1], [[0.0, 1.0, 0.0], [1.0, 0.0, 0.0]], None, [0.9, 0.999]), (1, 0, 0)),
    (([5, 2], [[0.25, 0.75, 0.0], [1.0, 0.0, 0.0]], None, [0.5, 0.0]), (0, 1, 1)),
    (([5, -1, 0], [[1.0, 0.0, 0.0]] * 3, None, [0.0, 0.0, 0.0]), (0, 0, 2)),
    (([5, 1], [[0.5, 0.5, 0.0]] * 2, [None, [0.5, 0.5, 0.0]], [0.0, 0.5]), (1, 0, 0)),
    # the draft's own distribution leaves nothing: the target's is drawn from
    (([5, 2], [[0.25, 0.25, 0.0]] * 2, [None, [0.5, 0.5, 0.0]], [0.5, 0.5]), (0, 1, 1)),
    (([], [], None, []), (0, -1, 0))])
def test_draft_rule_by_hand(case, want):
    assert CO.verify(*case) == want


# ------------------------------------------------------------------ refusals
P = 1 << 20


def _kv(hk, dtype=1, max_pages=4):
    return hk.hk_paged_kv(P, P, P, P, P, 64, max_pages, dtype)


def test_reserve_write_trim_refusals(hk):
    L = hk.lib()
    d, kv, al = hk.dims(4, 8, 2, 128), _kv(hk), hk.hk_allocator(P, P, 64)
    ch = lambda start=P, n=2, t=16, m=8: hk.hk_chunks(start, n, t, m)  # noqa: E731
    need = L.hk_workspace_size(hk.OP_RESERVE, C.byref(d), 4)
    assert need >= 3 * 8 * 4

    def reserve(d=d, kv=kv, c=ch(), al=al, ws=P, n=need):
        return L.hk_reserve_slots(C.byref(d), C.byref(kv), C.byref(c), C.byref(al), P, P, ws, n, None)
    assert reserve(c=ch(start=None)) == 1 and reserve(c=ch(n=0)) == 1
    assert reserve(c=ch(t=0)) == 1 and reserve(c=ch(m=0)) == 1
    assert reserve(c=ch(n=3)) == 3                            # 4 sequences of the cache, 3 of the batch
    assert reserve(c=ch(t=(1 << 24) + 1)) == 3 and reserve(c=ch(m=(1 << 24) + 1)) == 3
    assert reserve(d=hk.dims(65000, 1, 1, 128), c=ch(n=1, m=1 << 24), n=1 << 30) == 3   # too many threads
    assert reserve(al=hk.hk_allocator(None, P, 64)) == 1 and reserve(al=hk.hk_allocator(P, P, 0)) == 1
    assert reserve(ws=None) == 5 and reserve(n=need - 1) == 5 and reserve(ws=P + 16) == 4
    assert reserve(kv=_kv(hk, dtype=5)) == 2 and reserve(kv=_kv(hk, max_pages=3)) == 3
    assert L.hk_reserve_slots(C.byref(d), C.byref(kv), None, C.byref(al), P, P, P, need, None) == 1

    def write(layers=1, T=8, m=P, k=P, kr=256, v=P, vr=256, ls=0):
        return L.hk_write_kv(C.byref(d), C.byref(kv), layers, T, m, k, ls, kr, v, ls, vr, None)
    assert write(layers=0) == 1 and write(T=0) == 1 and write(m=None) == 1 and write(k=None) == 1
    assert write(kr=255) == 1 and write(vr=128) == 1          # rows shorter than the heads
    assert write(k=P + 8) == 4 and write(kr=260) == 4 and write(layers=2, ls=100) == 4
    assert write(layers=1 << 20, T=1 << 20, ls=1 << 24) == 3

    def trim(n=2, drop=P, al=al, ws=P, b=need):
        return L.hk_trim_slots(C.byref(d), C.byref(kv), n, drop, C.byref(al), ws, b, None)
    assert trim(n=0) == 1 and trim(drop=None) == 1 and trim(n=3) == 3
    assert trim(al=hk.hk_allocator(P, P, 63)) == 1            # the stack must hold the pool
    assert trim(b=need - 1) == 5 and trim(ws=P + 4) == 4


def test_chunk_attn_refusals(hk):
    L = hk.lib()
    d, kv = hk.dims(2, 8, 2, 128), _kv(hk)
    ch = hk.hk_chunks(P, 2, 16, 8)
    need = L.hk_chunk_attn_workspace_size(C.byref(d), C.byref(ch), 4)

    def attn(d=d, kv=kv, c=ch, q=P, row=1024, scale=0.1, o=P, ws=P, n=need):
        return L.hk_chunk_attn(C.byref(d), C.byref(kv), C.byref(c), q, row, scale, o, None, ws, n, None)
    assert attn(d=hk.dims(2, 8, 2, 96)) == 3 and attn(d=hk.dims(2, 9, 2, 128)) == 3
    assert attn(d=hk.dims(2, 130, 2, 128), row=130 * 128) == 3      # 65 query heads per KV head
    assert attn(c=hk.hk_chunks(P, 1, 16, 8)) == 3                   # sequences differ
    assert attn(scale=0.0) == 1 and attn(scale=math.inf) == 1 and attn(scale=math.nan) == 1
    assert attn(q=None) == 1 and attn(o=None) == 1 and attn(row=1023) == 1
    assert attn(q=P + 2) == 4 and attn(row=1028) == 4 and attn(o=P + 8) == 4
    if need:
        assert attn(n=need - 1) == 5 and attn(ws=None) == 5 and attn(ws=P + 16) == 4
    assert attn(kv=_kv(hk, dtype=9)) == 2
    # a workspace for more tokens serves fewer
    size = lambda t, m: L.hk_chunk_attn_workspace_size(  # noqa: E731
        C.byref(d), C.byref(hk.hk_chunks(P, 2, t, m)), 2048)
    sizes = [size(t, t) for t in (1, 2, 7, 31, 64, 300, 1000, 5000, 40000)]
    assert sizes == sorted(sizes) and size(5000, 1) <= size(5000, 5000)
    assert L.hk_chunk_attn_workspace_size(C.byref(d), None, 4) == 0


def test_chunk_attn_refuses_more_queries_than_a_launch_takes(hk):
    L = hk.lib()
    d, kv = hk.dims(1, 64 * 1000, 1000, 128), _kv(hk)
    for tokens, want in ((1 << 24, 3), (1 << 19, 3), (1 << 18, 5)):              # the last: no workspace
        c = hk.hk_chunks(P, 1, tokens, 8)
        assert L.hk_chunk_attn(C.byref(d), C.byref(kv), C.byref(c), P, 64 * 1000 * 128, 0.1, P, None, None, 0, None) == want


def test_verify_refusals(hk):
    L = hk.lib()
    ch, need = hk.hk_chunks(P, 2, 16, 8), L.hk_verify_workspace_size(2, 1000)
    assert need > 0 and L.hk_verify_workspace_size(2, (1 << 20) + 1) == 0

    def verify(c=ch, V=1000, dt=0, p=P, pr=1000, q=P, qr=1000, ws=P, n=need, u=P):
        return L.hk_verify_draft(C.byref(c), V, dt, P, p, pr, q, qr, u, P, P, P, None, ws, n, None)
    assert verify(V=0) == 1 and verify(V=(1 << 20) + 1, pr=1 << 21, qr=1 << 21) == 3 and verify(dt=2) == 2
    assert verify(pr=999) == 1 and verify(qr=999) == 1 and verify(p=None) == 1 and verify(u=None) == 1
    assert verify(p=P + 2) == 4 and verify(q=P + 1) == 4 and verify(dt=1, p=P + 1) == 4
    assert verify(n=need - 1) == 5 and verify(ws=P + 8) == 4
    assert verify(c=hk.hk_chunks(None, 2, 16, 8)) == 1


def test_wrappers_refuse_short_and_strange_tensors(hk):
    """Tensors with fewer rows than the call would touch, other types or scattered heads."""
    T, Hq, Hkv, D = 8, 4, 2, 64
    bf, f32, i32 = torch.bfloat16, torch.float32, torch.int32
    kv = hk.PagedKV(torch.zeros(8, 16, D, dtype=bf), torch.zeros(8, 16, D, dtype=bf),
                    torch.zeros(4, 4, dtype=i32), torch.zeros(4, 4, dtype=torch.int16), torch.zeros(4, dtype=i32))
    d, ch = hk.dims(2, Hq, Hkv, D), hk.Chunks(torch.zeros(3, dtype=i32), T, T)
    al = hk.Allocator(torch.zeros(8, dtype=i32), torch.zeros(1, dtype=i32))
    ws = torch.zeros(1 << 16, dtype=torch.uint8)
    q, o = torch.zeros(T, Hq, D, dtype=bf), torch.zeros(T, Hq, D, dtype=bf)
    for bad in (q[:7], q.float(), torch.zeros(T, D, Hq, dtype=bf).transpose(1, 2), torch.zeros(T, Hq, 2 * D, dtype=bf)[:, :, :D]):
        with pytest.raises(hk.HardKVError):
            hk.hk_chunk_attn(d, kv, ch, bad, 0.1, o, ws)
    for bad_o, lse in ((o[:5], None), (o.float(), None), (o, torch.zeros(T * Hq - 1)), (o, torch.zeros(T, Hq, dtype=bf))):
        with pytest.raises(hk.HardKVError):
            hk.hk_chunk_attn(d, kv, ch, q, 0.1, bad_o, ws, lse=lse)
    k = torch.zeros(T, Hkv, D, dtype=bf)
    m = torch.zeros(T * Hkv, dtype=torch.int64)
    for a, b, c in ((k[:3], k, m), (k, k.float(), m), (k, k, m[:-1]), (k, k, m.int()), (k[None].expand(2, -1, -1, -1), k, m)):
        with pytest.raises(hk.HardKVError):
            hk.hk_write_kv(d, kv, T, c, a, b)
    with pytest.raises(hk.HardKVError):
        hk.hk_reserve_slots(hk.dims(4, Hq, Hkv, D), kv, ch, al, ws)              # more rows than the cache has
    with pytest.raises(hk.HardKVError):
        hk.hk_reserve_slots(d, kv, ch, al, ws, slot_map=m[:-1])
    with pytest.raises(hk.HardKVError):
        hk.hk_trim_slots(hk.dims(4, Hq, Hkv, D), kv, torch.zeros(2, dtype=i32), al, ws)
    with pytest.raises(hk.HardKVError):
        hk.hk_trim_slots(d, kv, torch.zeros(2, dtype=torch.int64), al, ws)
    tok, u, out = torch.zeros(T, dtype=i32), torch.zeros(T), torch.zeros(2, dtype=i32)
    p = torch.zeros(T, 100)
    for pp, qq, tt in ((p[:4], None, tok), (p.double(), None, tok), (p[:, :50], None, tok), (p, p.bfloat16(), tok),
                       (torch.zeros(100, T).t(), None, tok), (p, None, tok.long())):
        with pytest.raises(hk.HardKVError):
            hk.hk_verify_draft(ch, 100, tt, pp, u, out, out, out, ws, q=qq)
    with pytest.raises(hk.HardKVError):
        hk.Chunks(torch.zeros(3), T, T)


def test_pipeline_refuses_larger_chunks(hk):
    from paper_2606_28831_amd.pipeline import ChunkDecoder, Verifier
    i32, bf = torch.int32, torch.bfloat16
    kv = hk.PagedKV(torch.zeros(8, 16, 64, dtype=bf), torch.zeros(8, 16, 64, dtype=bf),
                    torch.zeros(2, 4, dtype=i32), torch.zeros(2, 4, dtype=torch.int16), torch.zeros(2, dtype=i32))
    al = hk.Allocator(torch.zeros(8, dtype=i32), torch.zeros(1, dtype=i32))
    dec = ChunkDecoder(2, 1, 1, 64, kv, al, 16, 8)
    start = torch.zeros(3, dtype=i32)
    sm = torch.zeros(32, dtype=torch.int64)
    for c in (hk.Chunks(start, 17, 8), hk.Chunks(start, 16, 9), hk.Chunks(start[:2], 16, 8)):
        with pytest.raises(hk.HardKVError):
            dec.reserve(c, sm)
    with pytest.raises(hk.HardKVError):
        dec.trim(torch.zeros(1, dtype=i32))
    with pytest.raises(hk.HardKVError):
        Verifier(1, 10, "cpu").verify(hk.Chunks(start, 4, 4), None, None, None, None, None, None)
