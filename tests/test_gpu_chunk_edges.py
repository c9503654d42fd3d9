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


# ------------------------------------------------------------------ more blocks, heads and values
@pytest.mark.parametrize("D,n,G", [(128, 40, 4), (64, 40, 4), (128, 131, 1), (64, 70, 2)])
def test_one_long_row_in_a_launch_of_many_sequences(D, n, G):
    """Whole tiles over more than 64 and more than 128 blocks of 32 keys: odd and even numbers of them,
    rows that end just past, at and just before a multiple of 2048 keys, among sequences without rows."""
    B, Hkv, at = 130, 8, 77
    rows = [9000, 4097, 6145, 2049, 8192, 4064, 6177, 2111]
    c = Cache([0] * (at * Hkv) + rows + [0] * ((B - at - 1) * Hkv), D, "bf16", holes=0.1, seed=n, keep_last=n)
    lens = [0] * B
    lens[at] = n
    _attend(c, lens, Hkv, G, D, "bf16", pad=1, heads=range(at * Hkv, at * Hkv + Hkv))


@pytest.mark.parametrize("layers,B,Hkv,lens,most", [
    (3, 86, 8, [200, 1, 150, 0, 33], 60),           # 2064 heads: cuts of more than eight pages
    (17, 121, 8, [17, 0, 1], 20)])                  # 16456 heads: sums of more than 256 blocks of 64
def test_slots_of_many_heads(layers, B, Hkv, lens, most):
    import paper_2606_28831_amd as hk
    H = layers * B * Hkv
    lens = [lens[s % len(lens)] for s in range(B)]
    ctx = [(7 * h) % most for h in range(H)]
    c = Cache(ctx, 64, "bf16", seed=5, width=(max(lens) + most) // 16 + 3, spare=H * (1 + max(lens) // 16) // 2 + 2 * H)
    ok, t, m, n, top, slots = CO.reserve(c.t, c.m, c.n, c.free, c.top, lens, Hkv)
    assert ok
    ch, sm, status = _reserve(c, lens, Hkv, layers, pad=1)
    c.t, c.m, c.n, c.top = t, m, n, top
    assert status == 0
    c.check("reserve")
    got, first = np_i(sm), np.concatenate([[0], np.cumsum(lens)])
    for h in range(0, H, 13):
        l, s, kv = h // (B * Hkv), h // Hkv % B, h % Hkv
        assert got[l, first[s]:first[s + 1], kv].tolist() == slots[h]
    assert (got[:, -1] == -1).all() and (got[:, :-1] >= 0).all()
    d = hk.dims(layers * B, Hkv, Hkv, 64)
    ws = hk.workspace(hk.OP_TRIM, d, c.width, DEV)
    for drops in ([x // 3 for x in lens], [x - x // 3 for x in lens], [most] * B):
        c.t, c.m, c.n, c.free, c.top = CO.trim(c.t, c.m, c.n, np_i(c.free_ids), c.top, drops, Hkv)
        hk.hk_trim_slots(d, c.kv, torch.tensor(drops, dtype=I32, device=DEV), c.alloc, ws)
        torch.cuda.synchronize()
        c.check(drops[:5])
    assert (c.n == 0).all()


@pytest.mark.parametrize("V", [262145, 1 << 20])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_verify_large_vocabularies(V, dtype):
    """More than 64 pieces of 4096 values: tokens drawn from the first, a middle and the last piece."""
    rng = np.random.default_rng(V)
    lens = [2, 1, 1]
    p, q = (rng.random((4, V)) ** 8 for _ in "pq")
    p, q = p / p.sum(1, keepdims=True), q / q.sum(1, keepdims=True)
    put = lambda x: torch.tensor(x, device=DEV).to({"f32": torch.float32, "bf16": torch.bfloat16}[dtype])  # noqa: E731
    p, q = put(p), put(q)
    tok = torch.tensor([3, int(q[1].float().argmax()), 9, 9], dtype=I32, device=DEV)
    pn, qn, tn = np64(p), np64(q), np_i(tok)
    for us, own in (([0.9999999, 0.99, 0.0, 0.5], q), ([0.3, 0.0, 0.9999999, 0.97], None)):
        u = torch.tensor(us, dtype=torch.float32, device=DEV)
        got, status = _verify(p, own, tok, u, lens, V)
        for s, n in enumerate(lens):
            a = sum(lens[:s])
            want = CO.verify(tn[a:a + n], pn[a:a + n], None if own is None else qn[a:a + n], np_i(u)[a:a + n])
            assert (got[0][s], got[1][s], got[2][s]) == want, (us, s)
        assert status == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_written_layer_by_layer(dtype):
    """K and V of one layer at a time: both pools hold what one call for all layers leaves."""
    import paper_2606_28831_amd as hk
    layers, Hkv, D, lens = 3, 2, 64, [4, 0, 21]
    c = Cache([(5 * i) % 40 for i in range(layers * 3 * Hkv)], D, dtype, seed=3, width=8)
    ch, sm, status = _reserve(c, lens, Hkv, layers, pad=2, lead=1)
    T = ch.n_tokens
    k, v = (torch.randn(layers, T, Hkv, D, device=DEV).to(c.k_pool.dtype) for _ in "kv")
    d, at = hk.dims(3, Hkv, Hkv, D), sm.view(-1)
    want = []
    for pool, x in ((c.k_pool, k), (c.v_pool, v)):
        want.append(pool.view(-1, D).clone())
        want[-1][at[at >= 0]] = x.reshape(-1, D)[at >= 0]
    for l in range(layers):
        hk.hk_write_kv(d, c.kv, T, sm[l], k[l], v[l])
    torch.cuda.synchronize()
    bits = torch.int16 if dtype == "bf16" else I32
    for pool, w in zip((c.k_pool, c.v_pool), want):
        assert torch.equal(pool.view(-1, D).view(bits), w.view(bits))


# ------------------------------------------------------------------ scores past 2^24
@pytest.mark.parametrize("L,n,width", [(310, 70, None), (300, 5, None), (6000, 70, 512), (6000, 3, 512)])
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
def test_scores_past_the_last_bit(dtype, D, L, n, width):
    """Scores up to 1e18, of either sign and beside ordinary ones: results are finite, the largest score's V
    where no other score is within the products' error of it, and the LSE is off by that error."""
    import paper_2606_28831_amd as hk
    G, scale = 2, 1 / math.sqrt(D)
    c = Cache([L, L - 9], D, dtype, seed=n, width=width, keep_last=n, holes=0.1)
    T, d = n, hk.dims(1, 2 * G, 2, D)
    ch = _chunks([n])
    g = torch.Generator(device=DEV).manual_seed(7)
    base = torch.randn(T, 2 * G, D, generator=g, device=DEV)
    ws = hk.chunk_attn_workspace(d, ch, c.width, DEV)
    for k_scale, q_scale, sign in ((1e3, 1e3, 0), (1e5, 1e5, 0), (1e9, 1e9, 0), (3e4, 1e6, -1), (1e5, 1e5, 1)):
        k = c.k_pool.float()
        k = k / k[~k.isnan()].abs().max() * 4.0 * k_scale
        q = base * q_scale
        if sign:
            k, q = k.abs(), q.abs() * sign
        q[1::3] = base[1::3] / (4.0 * k_scale)               # every third token's scores are ordinary
        c.k_pool.copy_(k)
        q = q.to(c.k_pool.dtype)
        o, lse = torch.zeros(T, 2 * G, D, dtype=q.dtype, device=DEV), torch.zeros(T, 2 * G, device=DEV)
        hk.hk_chunk_attn(d, c.kv, ch, q, scale, o, ws, lse=lse)
        torch.cuda.synchronize()
        assert torch.isfinite(o).all() and torch.isfinite(lse).all(), (k_scale, q_scale, sign)
        qn, on, ln = np64(q), np64(o), np64(lse)
        for h in range(2):
            keys, vals, valid, end = c.head(h)
            hs = slice(h * G, h * G + G)
            ro, rl, zabs, absv = CO.chunk_attn_head(qn[:, hs], keys, vals, valid, end, scale)
            bo, bl = _bound(dtype, len(valid), rl, zabs, absv, ro, D)
            assert (np.abs(ln[:, hs] - rl) <= bl).all(), (k_scale, q_scale, sign, h)
            dz = (D + 8) * 2.0 ** -23 * zabs
            sure = 0
            for i in range(n):
                see = np.nonzero(valid[:end - n + i + 1])[0]
                for x in range(G):
                    z = scale * (keys[see] @ qn[i, h * G + x])
                    first, second = np.argsort(z)[::-1][:2]
                    if dz[i, x] < 0.01:                      # the ordinary ones
                        assert (np.abs(on[i, h * G + x] - ro[i, x]) <= bo[i, x]).all()
                    elif z[first] - z[second] > 2 * dz[i, x] + 30:
                        v = vals[see[first]]
                        assert (np.abs(on[i, h * G + x] - v) <= 2.0 ** -7 * np.abs(v) + 2.0 ** -30).all(), (i, x, k_scale)
                        sure += 1
            assert sure >= n // 3


# ------------------------------------------------------------------ the bits of fp32 caches
def _two_keys(dtype, D, n, heads, width=None, ctx=2, seed=3):
    """A cache whose queries weigh two keys alone: z = q0 k0 within [-0.5, 0.5], products of one term; every
    other key's probability is below 2^-500.  V is 1 and -1 in the two, 0 elsewhere.  Returns (cache, q,
    z [heads, n, 2])."""
    c = Cache([ctx + n] * heads, D, dtype, seed=seed, width=width, keep_last=ctx + n)
    k, v = torch.zeros_like(c.k_pool), torch.zeros_like(c.v_pool)
    g = torch.Generator(device=DEV).manual_seed(seed)
    pair = (torch.rand(heads, 2, generator=g, device=DEV) - 0.5).to(k.dtype)
    k[..., 0] = -1000.0
    for h in range(heads):
        at = int(c.t[h, 0])
        k[at, :2, 0] = pair[h]
        v[at, 0], v[at, 1] = 1.0, -1.0
    c.k_pool.copy_(k)
    c.v_pool.copy_(v)
    q = torch.zeros(n, heads, D, device=DEV)
    q[..., 0] = 0.5 + 0.5 * torch.rand(n, heads, generator=g, device=DEV)
    q = q.to(k.dtype)
    return c, q, np64(q[..., 0]).T[:, :, None] * np64(pair)[:, None, :]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,ctx,width", [(20, 2, None), (64, 2, None), (20, 3000, 400), (64, 3000, 400)])
def test_fp32_probabilities_keep_their_bits(D, n, ctx, width):
    """o = tanh((z0 - z1) / 2) of two keys.  In base 2 an exponent lies within [-1.73, 0] below the reference:
    its rounding is 2^-24, c2's share 2^-25, the score's product 2^-25, so 0.7 (2^-24 + 2^-24) of a probability,
    and 2^-23 of the exponential itself; o takes p0 p1 |v0 - v1| = 2 p0 p1 <= 0.5 of both keys' errors.  Sums
    and products with V of a few steps, cut by the matrix cores: 2^-23 of a probability each (2 of V, 2 of the
    sum), the joins' factors are powers of two, 1 / l and its product 2^-23 of o."""
    import paper_2606_28831_amd as hk
    heads = 16
    c, q, z = _two_keys("f32", D, n, heads, width, ctx)
    d, ch = hk.dims(1, heads, heads, D), _chunks([n])
    o, lse = torch.zeros(n, heads, D, device=DEV), torch.zeros(n, heads, device=DEV)
    hk.hk_chunk_attn(d, c.kv, ch, q, 1.0, o, hk.chunk_attn_workspace(d, ch, c.width, DEV), lse=lse)
    torch.cuda.synchronize()
    want = np.tanh((z[..., 0] - z[..., 1]) / 2).T[:, :, None]
    p = 0.5 * (1 + np.abs(want))
    each = 0.7 * (2.0 ** -24 + 2.0 ** -24) + 2.0 ** -23
    bound = 2 * p * (1 - p) * 2 * each + 4 * 2.0 ** -23 * p + 2.0 ** -23 * np.abs(want)
    assert (np.abs(np64(o) - want) <= bound).all()


@pytest.mark.parametrize("dtype,D,n,ctx,width", [
    ("f32", 64, 20, 2, None), ("f32", 128, 64, 2, None), ("f32", 128, 20, 3000, 400), ("f32", 64, 64, 3000, 400),
    ("bf16", 128, 20, 2, None), ("bf16", 64, 20, 3000, 400), ("bf16", 128, 64, 2, None), ("bf16", 64, 64, 3000, 400)])
def test_small_lses(dtype, D, n, ctx, width):
    """LSEs of two keys, 0.2 to 1.2: off by what the probabilities are (above; in bf16 tiles an exponent of up to
    32, rounded to 2^-20), by two additions of the sum, cut, by the logarithm of a value in [0.5, 1), by the sum
    of it and a whole number up to 4 (2^-22), and by the product."""
    import paper_2606_28831_amd as hk
    heads = 16
    c, q, z = _two_keys(dtype, D, n, heads, width, ctx)
    d, ch = hk.dims(1, heads, heads, D), _chunks([n])
    o, lse = torch.zeros(n, heads, D, dtype=q.dtype, device=DEV), torch.zeros(n, heads, device=DEV)
    hk.hk_chunk_attn(d, c.kv, ch, q, 1.0, o, hk.chunk_attn_workspace(d, ch, c.width, DEV), lse=lse)
    torch.cuda.synchronize()
    want = np.logaddexp(z[..., 0], z[..., 1]).T
    tile = dtype == "bf16" and n > 32
    each = 0.7 * (2.0 ** -24 + (2.0 ** -20 if tile else 2.0 ** -24)) + 2.0 ** -23
    bound = each + 2 * 2.0 ** -23 + 0.7 * (2.0 ** -23 + 2.0 ** -23) + 2.0 ** -23 * np.abs(want)
    assert (np.abs(np64(lse) - want) <= bound).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,ctx,width", [(64, 2, None), (64, 3000, 400)])
def test_one_key_of_weight_has_its_v(D, n, ctx, width):
    """Longer chunks of a bf16 cache round P, but o stays a mean of V: of two keys V0 and V1 = -V0 it is off by
    p0 p1 |V0 - V1| of the two roundings' difference, 2 x 2^-8 at most, and by its own rounding; sums and
    products of a few steps beside.  A prompt's first token has the first V."""
    import paper_2606_28831_amd as hk
    heads = 16
    c, q, z = _two_keys("bf16", D, n, heads, width, ctx)
    for h in range(heads):
        c.k_pool[int(c.t[h, 0]), :2, 0] *= 16.0
    z = z * 16.0
    d, ch = hk.dims(1, heads, heads, D), _chunks([n])
    o = torch.zeros(n, heads, D, dtype=q.dtype, device=DEV)
    hk.hk_chunk_attn(d, c.kv, ch, q, 1.0, o, hk.chunk_attn_workspace(d, ch, c.width, DEV))
    torch.cuda.synchronize()
    want = np.tanh((z[..., 0] - z[..., 1]) / 2).T[:, :, None]
    p = 0.5 * (1 + np.abs(want))
    off = 2 * p * (1 - p) * (2 * 2.0 ** -8) * 1.02 + 2.0 ** -19
    assert (np.abs(np64(o) - want) <= off + 2.0 ** -8 * (np.abs(want) + off)).all()
    c = Cache([n] * 4, D, "bf16", seed=9)
    q, o, lse = _attend(c, [n], 4, 1, D, "bf16")
    for h in range(4):
        assert torch.equal(o[0, h], c.v_pool[int(c.t[h, 0]), 0])
