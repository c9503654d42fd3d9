"""The 8-bit cache on the GPU against the oracle: rows written and read back, attention of single
tokens and chunks, the rewrite, and all of them chained.  Wherever no token was written the pools hold
codes of NaN (e4m3; int8: -128) and scales of NaN, so that anything read from a masked slot, a page's
tail or a free page shows."""
import math

import numpy as np
import pytest
import torch

import oracle.chunk_oracle as CO
import oracle.kv8_oracle as O8
from hk_testlib import np64, np_i, rewrite_layout, unpack_bits

pytestmark = pytest.mark.gpu
DEV = "cuda"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
CODE = {"i8": torch.int8, "e4m3": torch.float8_e4m3fn}
GARBAGE = {"i8": 0x80, "e4m3": 0x7F}
I32 = torch.int32


def _bytes(t):
    return t.view(torch.uint8)


class Cache8:
    """An 8-bit cache of given row lengths with its tables on the host."""

    def __init__(self, lens, D, fmt, width=None, holes=0.0, seed=0, spare=100, keep_last=0, v_scale=1.0, k_scale=1.0):
        import paper_2606_28831_amd as hk
        rng = np.random.default_rng(seed)
        H, pages = len(lens), [-(-x // 16) for x in lens]
        self.width = max(pages + [2]) if width is None else width
        self.width += self.width % 2
        self.fmt, self.D = fmt, D
        pool = sum(pages) + spare
        perm = rng.permutation(pool)
        self.t = np.full((H, self.width), -1, np.int64)
        self.m = np.zeros((H, self.width), np.int64)
        self.n = np.array(pages, np.int64)
        at = 0
        for h, L in enumerate(lens):
            self.t[h, :pages[h]] = perm[at:at + pages[h]]
            at += pages[h]
            bits = rng.random(L) >= holes
            bits[max(0, L - max(keep_last, 1)):] = True       # the newest token stands
            for j in np.nonzero(bits)[0]:
                self.m[h, j // 16] |= 1 << (j % 16)
        self.free = np.zeros(pool, np.int64)
        self.top = pool - at
        self.free[:self.top] = perm[at:]
        rows = np.array([int(self.t[h, j // 16]) * 16 + j % 16 for h in range(H) for j in self.slots(h)], np.int64)
        for x, size in (("k", k_scale), ("v", v_scale)):
            codes = np.full((pool * 16, D), GARBAGE[fmt], np.uint8)
            scale = np.full(pool * 16, np.nan, np.float32)
            # codes of normal rows: the largest code's size somewhere, the rest below it
            y = rng.standard_normal((len(rows), D))
            if len(rows):
                y *= O8.MOST[fmt] / np.abs(y).max(1, keepdims=True)
                if fmt == "i8":
                    codes[rows] = np.rint(y).astype(np.int8).view(np.uint8)
                else:
                    codes[rows] = np_i(_bytes(torch.tensor(y).float().to(torch.float8_e4m3fn)))
                scale[rows] = (size * (0.5 + rng.random(len(rows))) * 3.0 / O8.MOST[fmt]).astype(np.float32)
            setattr(self, x + "_codes", codes)
            setattr(self, x + "_sc", scale)
            setattr(self, x + "_pool", torch.tensor(codes, device=DEV).view(CODE[fmt]).view(pool, 16, D))
            setattr(self, x + "_scale", torch.tensor(scale, device=DEV).view(pool, 16))
        put = lambda x, d: torch.tensor(x, device=DEV).to(d)  # noqa: E731
        self.page_table, self.n_pages = put(self.t, I32), put(self.n, I32)
        self.page_mask = put(self.m, I32).to(torch.int16)
        self.free_ids, self.free_top = put(self.free, I32), put(np.array([self.top]), I32)
        self.kv = hk.PagedKV8(self.k_pool, self.v_pool, self.k_scale, self.v_scale, self.page_table, self.page_mask,
                              self.n_pages)
        self.alloc = hk.Allocator(self.free_ids, self.free_top)

    def slots(self, h):
        return [j for j in range(16 * int(self.n[h])) if self.m[h, j // 16] >> (j % 16) & 1]

    def head(self, h):
        """keys, vals, valid, end of one head as numbers, from the host's codes."""
        n = int(self.n[h])
        if n == 0:
            return np.zeros((0, self.D)), np.zeros((0, self.D)), np.zeros(0, bool), 0
        at = (self.t[h, :n, None] * 16 + np.arange(16)).reshape(-1)
        valid = np.array([(self.m[h, j // 16] >> (j % 16)) & 1 for j in range(16 * n)], bool)
        out = []
        for c, s in ((self.k_codes, self.k_sc), (self.v_codes, self.v_sc)):
            x = np.zeros((16 * n, self.D))
            x[valid] = O8.values(c[at[valid]], self.fmt) * s[at[valid]].astype(np.float64)[:, None]
            out.append(x)
        return out[0], out[1], valid, CO.row_end(self.m[h], n)


def _bound(dtype, parts, n_keys, lse, zabs, absv, o, D):
    """Error bounds of (o, lse) against 64 bits, term by term:
      scores   D products summed in fp32, of one or (fp32 queries) three parts whose second and third
               are 2^-7 and 2^-15 of the first at most; each addition off by at most 2^-23, the matrix
               cores cut; then the scale's rounding, its product with the score, the reference taken off:
               dz = (1.01 D + 8) 2^-23 max sum |q k|;
      sums     probabilities off by 2 dz each and a few steps of the exponential, the running sum's n
               additions over 64 lanes at least, the states' joins: (n / 32 + 64) 2^-23;
      parts    P enters the product with V rounded: to fp16 once (1: 2^-11 of every term), in two bf16
               parts (2: 2^-16) or in three (3: 2^-23);
      dtype    of o: half a step, bf16 2^-8, fp32 2^-24;
      floor    p scale 2^-bias and its parts count as 0 below 2^-126: at most three such losses a term,
               each of 2^(bias - 126) times the code (448 at most), beside a largest p of at least a half,
               with bias at most 6 + log2 of the keys (the slack of 4 and two roundings up).  fp16 (1) has
               the step 2^-24 for small P: a term is off by 2^-25 at most, where the row's largest P is
               at least 2^8 (2^10, times a reference's rounding up, times a scale's fraction, a half each),
               which stands for no more than the largest p |v| of the row, and so of its sum p |v|:
               2^-33 of that a key."""
    dz = (1.01 * D + 8) * 2.0 ** -23 * zabs
    rest = (n_keys / 32 + 64) * 2.0 ** -23
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    p = {1: 2.0 ** -11, 2: 2.0 ** -16, 3: 2.0 ** -23}[parts]
    bo = half * np.abs(o) * 1.01 + (p + 2 * dz[..., None] + 2 * rest) * 1.05 * absv
    bo += 6 * n_keys * 448 * 2.0 ** (6 + math.log2(max(n_keys, 16)) - 126)
    if parts == 1:
        bo += n_keys * 2.0 ** -33 * absv.max(-1, keepdims=True)
    return bo, dz + rest + 2.0 ** -22 * np.maximum(1.0, np.abs(np.where(np.isfinite(lse), lse, 0.0)))


def _check_head(c, h, q, got_o, got_l, scale, dtype, parts):
    k, v, valid, end = c.head(h)
    ro, rl, zabs, absv = CO.chunk_attn_head(q, k, v, valid, end, scale)
    bo, bl = _bound(dtype, parts, len(valid), rl, zabs, absv, ro, c.D)
    assert (np.isneginf(got_l) == np.isneginf(rl)).all(), f"head {h}: empty rows"
    fin = np.isfinite(rl)
    assert np.isfinite(got_l[fin]).all() and np.isfinite(got_o).all(), f"head {h}: not finite"
    off = np.abs(got_o - ro)
    at = np.unravel_index(np.argmax(off / np.maximum(bo, 1e-300)), off.shape)
    if not (off <= bo).all():
        pytest.fail(f"head {h}: o{at} is {got_o[at]}, not {ro[at]}, bound {bo[at]:.3g}")
    worst = np.max(np.abs(got_l[fin] - rl[fin]) / bl[fin]) if fin.any() else 0
    assert (np.abs(got_l[fin] - rl[fin]) <= bl[fin]).all(), f"head {h}: lse is {worst:.2f} bounds off"
    assert (got_o[~fin] == 0).all()


def _decode(c, NS, Hkv, G, dtype, seed=5, q_scale=1.0, heads=None, check=True):
    import paper_2606_28831_amd as hk
    D, Hq = c.D, Hkv * G
    g = torch.Generator(device=DEV).manual_seed(seed)
    q = (torch.randn(NS, Hq, D, generator=g, device=DEV) * q_scale).to(DT[dtype])
    o = torch.full((NS, Hq, D), -7.0, device=DEV)
    lse = torch.full((NS, Hq), -7.0, device=DEV)
    d = hk.dims(NS, Hq, Hkv, D)
    ws = hk.workspace(hk.OP_DECODE8, d, c.width, DEV)
    ws.fill_(255)
    scale = 1 / math.sqrt(D)
    hk.hk_decode_attn8(d, q, c.kv, scale, o, lse, ws)
    torch.cuda.synchronize()
    if check:
        qn, on, ln = np64(q), np64(o), np64(lse)
        for h in range(NS * Hkv) if heads is None else heads:
            s, kv = divmod(h, Hkv)
            g = slice(kv * G, kv * G + G)
            _check_head(c, h, qn[s:s + 1, g], on[s:s + 1, g], ln[s:s + 1, g], scale, "f32", 3)
    return q, o, lse


def _chunks(lens, pad=0, max_len=None, lead=0):
    import paper_2606_28831_amd as hk
    start = np.concatenate([[0], np.cumsum(lens)]) + lead
    return hk.Chunks(torch.tensor(start, dtype=I32, device=DEV), int(start[-1]) + pad, max_len or max(max(lens), 1))


def _attend(c, lens, Hkv, G, dtype, seed=5, pad=0, lead=0, max_len=None, q_scale=1.0, heads=None, check=True):
    import paper_2606_28831_amd as hk
    ch = _chunks(lens, pad, max_len, lead)
    T, Hq, B, D = ch.n_tokens, Hkv * G, len(lens), c.D
    g = torch.Generator(device=DEV).manual_seed(seed)
    q = (torch.randn(T, Hq, D, generator=g, device=DEV) * q_scale).to(DT[dtype])
    o = torch.full((T, Hq, D), -7.0, dtype=DT[dtype], device=DEV)
    lse = torch.full((T, Hq), -7.0, device=DEV)
    d = hk.dims(B, Hq, Hkv, D)
    ws = hk.chunk_attn8_workspace(d, ch, c.width, DEV)
    ws.fill_(255)
    scale = 1 / math.sqrt(D)
    hk.hk_chunk_attn8(d, c.kv, ch, q, scale, o, ws, lse=lse)
    torch.cuda.synchronize()
    used = sum(lens)
    for t in (o, lse):
        assert (t[:lead] == -7.0).all() and (t[lead + used:] == -7.0).all(), "padding rows were written"
    if check:
        qn, on, ln = np64(q), np64(o), np64(lse)
        for h in range(B * Hkv) if heads is None else heads:
            s, kv = divmod(h, Hkv)
            a, n, g = lead + sum(lens[:s]), lens[s], slice(kv * G, kv * G + G)
            if n:
                _check_head(c, h, qn[a:a + n, g], on[a:a + n, g], ln[a:a + n, g], scale, dtype,
                            3 if dtype == "f32" else 2 if n * G <= 32 else 1)
    return q, o, lse


# ------------------------------------------------------------------ rows
def _odd_rows(n, D, seed):
    """Rows of every size, with ties, zeros, tiny, huge, infinite and NaN ones among them."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, D, generator=g) * torch.exp(torch.randn(n, 1, generator=g) * 6)
    x[0] = 0.0
    x[1] = -0.0
    x[2, :] = 2.0 ** -130
    x[3] = x[3] / x[3].abs().max() * 3.3e38
    x[4, 5], x[5, 0], x[6, D - 1] = float("nan"), float("inf"), float("-inf")
    x[7] = (torch.arange(D) - D // 2).float() + 0.5                 # halves: ties of int8 where the largest is 127
    x[7, 0] = 127.0
    x[8] = torch.where(torch.arange(D) % 2 == 0, 448.0, 18.0 * 2.0 ** -9)
    x[9] = 2.0 ** -99 * torch.rand(D, generator=g)
    x[10] = 1e-40
    return x


@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,Hkv,L,T", [(128, 3, 2, 13), (64, 1, 1, 12), (64, 5, 3, 7), (128, 8, 1, 65)])
def test_rows_written_and_read_back(fmt, dtype, D, Hkv, L, T):
    """Codes and scales to the bit, through maps with rows left out, from and into parts of larger tensors."""
    import paper_2606_28831_amd as hk
    pages = -(-L * T * Hkv // 16) + 3
    rng = np.random.default_rng(3)
    slots = rng.permutation(pages * 16)[:L * T * Hkv].reshape(L, T, Hkv)
    slots[:, T - 1] = -1                                              # padding
    slots[0, 1, 0] = pages * 16                                       # outside the pool
    wide = torch.zeros(L, T, 2 * Hkv + 1, D, dtype=DT[dtype], device=DEV)
    wide[:, :, :2 * Hkv] = _odd_rows(L * T * 2 * Hkv, D, 7).view(L, T, 2 * Hkv, D).to(DEV).to(DT[dtype])
    k, v = wide[:, :, :Hkv], wide[:, :, Hkv:2 * Hkv]
    pool = lambda: torch.full((pages, 16, D), GARBAGE[fmt], dtype=torch.uint8, device=DEV).view(CODE[fmt])  # noqa: E731
    kp, vp, ks, vs = pool(), pool(), torch.full((pages, 16), -3.0, device=DEV), torch.full((pages, 16), -3.0, device=DEV)
    some = torch.zeros(Hkv, 2, dtype=I32, device=DEV)
    kv = hk.PagedKV8(kp, vp, ks, vs, some, some.to(torch.int16), some[:, 0].contiguous())
    d, m = hk.dims(1, Hkv, Hkv, D), torch.tensor(slots, device=DEV)
    hk.hk_write_kv8(d, kv, T, m, k, v)
    out = torch.full((L, T, 3 * Hkv, D), -5.0, dtype=DT[dtype], device=DEV)
    hk.hk_read_kv8(d, kv, T, m, out[:, :, :Hkv], out[:, :, 2 * Hkv:])
    alone = torch.full((L, T, Hkv, D), -5.0, dtype=torch.float32, device=DEV)
    hk.hk_read_kv8(d, kv, T, m, alone)
    got, gots = {}, {}
    for name, p, s, x, y in (("k", kp, ks, k, out[:, :, :Hkv]), ("v", vp, vs, v, out[:, :, 2 * Hkv:])):
        codes = np.full((pages * 16, D), GARBAGE[fmt], np.uint8)
        scale = np.full(pages * 16, -3.0, np.float64)
        back = np.full((L, T, Hkv, D), -5.0)
        xn = np64(x)
        for at in np.ndindex(L, T, Hkv):
            j = slots[at]
            if 0 <= j < pages * 16:
                codes[j], scale[j] = O8.quantise(xn[at], fmt)
                back[at] = O8.values(codes[j], fmt) * scale[j]
        assert (np_i(_bytes(p)).reshape(-1, D) == codes).all(), name
        np.testing.assert_array_equal(np64(s).reshape(-1), scale)
        back32 = torch.tensor(back).float()                           # the product, rounded to fp32, then to the row type
        np.testing.assert_array_equal(np64(y), np64(back32.to(DT[dtype])))
        if name == "k":
            np.testing.assert_array_equal(np64(alone), np64(back32))
    assert (out[:, :, Hkv:2 * Hkv] == -5.0).all(), "rows beside the values were written"
    assert (out[:, T - 1] == -5.0).all()


@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
def test_a_row_is_off_by_half_a_step(fmt):
    import paper_2606_28831_amd as hk
    n, D = 4096, 128
    g = torch.Generator(device=DEV).manual_seed(1)
    x = torch.randn(1, n, 1, D, generator=g, device=DEV)
    kp = torch.zeros(n // 16, 16, D, dtype=torch.uint8, device=DEV).view(CODE[fmt])
    s = torch.zeros(n // 16, 16, device=DEV)
    some = torch.zeros(1, 2, dtype=I32, device=DEV)
    kv = hk.PagedKV8(kp, kp.clone(), s, s.clone(), some, some.to(torch.int16), some[:, 0].contiguous())
    m = torch.arange(n, device=DEV)
    d = hk.dims(1, 1, 1, D)
    hk.hk_write_kv8(d, kv, n, m, x, x)
    y = torch.empty_like(x)
    hk.hk_read_kv8(d, kv, n, m, y)
    a = x.abs().amax(-1, keepdim=True).double()
    # a few roundings of fp32 beside the code's own
    half = a / 254 if fmt == "i8" else torch.maximum(x.abs().double() * 2.0 ** -4, a / 448 / 1024)
    assert ((y.double() - x.double()).abs() <= half * (1 + 2.0 ** -20) + a * 2.0 ** -22).all()


def test_every_e4m3_code_reads_as_its_value():
    import paper_2606_28831_amd as hk
    codes = torch.arange(256, dtype=torch.uint8, device=DEV).view(1, 2, 128).repeat(1, 8, 1)
    one = torch.ones(1, 16, device=DEV)
    some = torch.zeros(1, 2, dtype=I32, device=DEV)
    m = torch.arange(16, device=DEV)
    for fmt in ("i8", "e4m3"):
        kv = hk.PagedKV8(codes.view(CODE[fmt]), codes.view(CODE[fmt]), one, one, some, some.to(torch.int16), some[:, 0].contiguous())
        for dtype in ("f32", "bf16"):
            k = torch.zeros(16, 1, 128, dtype=DT[dtype], device=DEV)
            hk.hk_read_kv8(hk.dims(1, 1, 1, 128), kv, 16, m, k)
            np.testing.assert_array_equal(np64(k).reshape(16, 128), O8.values(np_i(codes).reshape(16, 128), fmt))


# ------------------------------------------------------------------ one token
DECODE = [
    # D, Hkv, G, row lengths of the sequences
    (128, 2, 4, [37]),
    (128, 1, 1, [0, 1, 16, 17, 31, 32, 33, 700]),
    (64, 2, 3, [40, 0, 511, 130, 15]),
    (128, 1, 7, [1000, 129, 48]),
    (64, 1, 16, [300, 5]),
    (128, 1, 17, [300, 64, 0]),
    (64, 1, 33, [100, 257]),
    (128, 1, 64, [70, 5]),
    (64, 3, 1, [2000, 128, 127]),
    (128, 5, 8, [257, 96]),
]


@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("holes", [0.0, 0.35])
@pytest.mark.parametrize("D,Hkv,G,lens", DECODE)
def test_decode(fmt, dtype, holes, D, Hkv, G, lens):
    c = Cache8([max(x - 3 * kv, 0) for x in lens for kv in range(Hkv)], D, fmt, holes=holes, seed=G + len(lens))
    _decode(c, len(lens), Hkv, G, dtype)


@pytest.mark.parametrize("fmt,dtype,D,G,lens,width", [
    ("i8", "bf16", 128, 4, [9000], 4096), ("e4m3", "bf16", 64, 2, [5001, 3], 768), ("i8", "f32", 128, 1, [6000], 1024),
    ("e4m3", "f32", 64, 8, [4100, 900, 0], 300), ("i8", "bf16", 128, 33, [3000], 400), ("e4m3", "bf16", 128, 1, [17], 8192)])
def test_decode_over_ranges(fmt, dtype, D, G, lens, width):
    _decode(Cache8(lens, D, fmt, width=width, holes=0.1, seed=9), len(lens), 1, G, dtype)


@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
def test_decode_of_many_heads(fmt):
    """A launch that needs no ranges for its workgroups: long ones, rows of every length."""
    NS, Hkv = 300, 8
    c = Cache8([(37 * i) % 320 for i in range(NS * Hkv)], 64, fmt, width=200, seed=4)
    _decode(c, NS, Hkv, 2, "bf16", heads=range(0, NS * Hkv, 97))


def test_decode_in_a_wave_over_more_than_64_pages():
    """One range of 8192 / 64 = 128 pages and rows that fill it: every wave takes its ids twice at most."""
    c = Cache8([16 * 1024 - 5] * 64, 64, "i8", seed=4, spare=1)
    _decode(c, 64, 1, 1, "bf16", heads=[0, 63])


@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sharp_flat_and_far_scores(fmt, dtype):
    """Scores hundreds apart, where the running reference moves in almost every block, all alike, and
    past 2^24, where a whole number is less than a step."""
    c = Cache8([1500, 90], 128, fmt, seed=21, holes=0.1, keep_last=70)
    for q_scale in (40.0, 1e-3, 0.0):
        _decode(c, 2, 1, 4, dtype, q_scale=q_scale)
        _attend(c, [9, 70], 1, 2, dtype, q_scale=q_scale)
    _, o, lse = _decode(c, 2, 1, 4, dtype, q_scale=3e8, check=False)
    assert torch.isfinite(o).all() and torch.isfinite(lse).all()
    for s in range(2):
        _, v, valid, _ = c.head(s)
        far = np64(o[s])[:, None, :] - v[valid][None]
        assert (np.abs(far).max(2).min(1) <= 2.0 ** -22 * np.abs(v).max()).all(), "one key has all of the weight"


@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
@pytest.mark.parametrize("size", [1e30, 1e-20])
def test_values_near_the_ends_of_the_range(fmt, size):
    for lens in ([2000], [70]):
        c = Cache8(lens, 64, fmt, seed=2, v_scale=size)
        _decode(c, 1, 1, 4, "bf16")
        _attend(c, [3], 1, 4, "f32")
        _attend(c, [40], 1, 4, "bf16")


def test_values_at_the_top_stay_finite():
    c = Cache8([2000], 64, "i8", seed=2)
    c.v_scale.copy_(torch.where(torch.isnan(c.v_scale), c.v_scale, torch.tensor(3.4e38 / 127, device=DEV)))
    _, o, _ = _decode(c, 1, 1, 4, "bf16", check=False)
    assert torch.isfinite(o).all()
    _, o, _ = _attend(c, [70], 1, 4, "f32", check=False)
    assert torch.isfinite(o).all()


@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
def test_nan_rows_reach_who_sees_them_alone(fmt):
    """A row that was not finite has the scale NaN: queries that see it give NaN, the others nothing of it."""
    for which in ("k", "v"):
        for lens in ([6], [70]):
            c = Cache8([100], 128, fmt, seed=3)
            row = int(c.t[0, 97 // 16]) * 16 + 97 % 16               # the third newest token
            getattr(c, which + "_scale").view(-1)[row] = float("nan")
            _bytes(getattr(c, which + "_pool")).view(-1, 128)[row] = 0
            _, o, lse = _attend(c, lens, 1, 2, "bf16", check=False)
            n = lens[0]
            assert torch.isfinite(o[:n - 3]).all() and torch.isfinite(lse[:n - 3]).all()
            assert torch.isnan(o[n - 3:]).all()
            assert torch.isnan(lse[n - 3:]).all() == (which == "k")
            _, o, _ = _decode(c, 1, 1, 2, "bf16", check=False)
            assert torch.isnan(o).all()


@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_nan_row_that_is_alone_in_its_part(fmt, dtype):
    """A long row is cut into parts of eight pages; in one of them the only valid slot is a NaN row."""
    c = Cache8([700], 128, fmt, seed=3, width=64)
    row = int(c.t[0, 11]) * 16 + 5
    c.k_scale.view(-1)[row] = float("nan")
    _bytes(c.k_pool).view(-1, 128)[row] = 0
    c.page_mask[0, 8:16] = 0
    c.page_mask[0, 11] = 1 << 5
    for _, o, lse in (_decode(c, 1, 1, 2, dtype, check=False), _attend(c, [6], 1, 2, dtype, check=False),
                      _attend(c, [70], 1, 2, dtype, check=False)):
        assert torch.isnan(o).all() and torch.isnan(lse).all()


@pytest.mark.parametrize("D", [64, 128])
def test_masks_that_leave_nothing(D):
    """A head all of whose slots are masked, one with a single slot at the far end, one of plain rows."""
    c = Cache8([900, 900, 900], D, "i8", seed=3, width=64)
    c.m[0] = 0
    c.m[1] = 0
    c.m[1, 56] = 1 << 3
    c.page_mask.copy_(torch.tensor(c.m, device=DEV).to(torch.int16))
    _, o, lse = _decode(c, 1, 3, 4, "bf16")
    assert (o[0, :4] == 0).all() and torch.isneginf(lse[0, :4]).all()
    _attend(c, [1], 3, 4, "bf16")


def test_decode_of_more_heads_than_are_planned():
    NS, Hkv = 520, 8
    c = Cache8([(7 * i) % 45 for i in range(NS * Hkv)], 64, "e4m3", width=40, seed=4)
    _decode(c, NS, Hkv, 2, "f32", heads=list(range(0, NS * Hkv, 331)) + [NS * Hkv - 1])


@pytest.mark.parametrize("fmt,dtype,lens", [("i8", "bf16", [1100, 1040]), ("e4m3", "f32", [301, 260])])
def test_more_tiles_than_are_planned(fmt, dtype, lens):
    Hkv, G = 8, 8
    c = Cache8([n + 20 - k for n in lens for k in range(Hkv)], 64, fmt, seed=4, keep_last=2000)
    _attend(c, lens, Hkv, G, dtype, pad=2, heads=[0, 5, 15])


LONG = [("i8", 128, 4, [1030, 40, 3, 0], [700, 33, 900, 50]), ("e4m3", 128, 8, [515, 17], [1, 2000]),
        ("e4m3", 64, 4, [9, 1025, 31], [300, 0, 15]), ("i8", 64, 16, [257, 1, 2, 60], [16, 700, 0, 31])]


@pytest.mark.parametrize("holes", [0.0, 0.35])
@pytest.mark.parametrize("fmt,D,G,lens,ctx", LONG)
def test_long_chunks_beside_short_ones(fmt, D, G, lens, ctx, holes):
    """Chunks of 4096 query rows of a KV head and more, whose tiles are converted beforehand."""
    rows = [ctx[s] - min(ctx[s], 3 * kv) + lens[s] for s in range(len(lens)) for kv in range(2)]
    c = Cache8(rows, D, fmt, holes=holes, seed=G, keep_last=max(lens), width=256)
    _attend(c, lens, 2, G, "bf16", pad=3, lead=2)


@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
@pytest.mark.parametrize("D", [64, 128])
def test_chunks_that_may_be_long(fmt, D):
    """The same with a short chunk where a long one could be: sharp scores, scales near the range's ends, heads
    without pages, NaN rows."""
    most = dict(max_len=2048, pad=2048)
    for q_scale in (40.0, 0.0):
        _attend(Cache8([1500, 90, 0], D, fmt, seed=21, holes=0.1, keep_last=70), [40, 70, 0], 1, 2, "bf16", q_scale=q_scale, **most)
    for size in (1e30, 1e-20):
        _attend(Cache8([500], D, fmt, seed=2, v_scale=size), [40], 1, 4, "bf16", **most)
    for which in ("k", "v"):
        c = Cache8([100], D, fmt, seed=3)
        row = int(c.t[0, 97 // 16]) * 16 + 97 % 16
        getattr(c, which + "_scale").view(-1)[row] = float("nan")
        _bytes(getattr(c, which + "_pool")).view(-1, D)[row] = 0
        _, o, lse = _attend(c, [70], 1, 2, "bf16", check=False, **most)
        assert torch.isfinite(o[:67]).all() and torch.isfinite(lse[:67]).all()
        assert torch.isnan(o[67:70]).all() and torch.isnan(lse[67:70]).all() == (which == "k")
    # V scales far apart in a head, within 2^100 of one another
    c = Cache8([600], D, fmt, seed=3)
    far = torch.pow(2.0, -(torch.arange(c.v_scale.numel(), device=DEV) % 7) * 9.0).view_as(c.v_scale)
    c.v_scale.mul_(far)
    c.v_sc[:] = c.v_scale.view(-1).cpu().numpy()
    for long in (most, {}):
        _attend(c, [70], 1, 2, "bf16", **long)


# ------------------------------------------------------------------ chunks
ATTN = [
    ("bf16", 128, 2, 4, [5], [37]),
    ("bf16", 128, 1, 1, [1, 1, 1], [0, 1, 16]),
    ("bf16", 64, 2, 3, [0, 11, 0, 1, 10, 0], [40, 3, 0, 700, 15, 9]),
    ("bf16", 128, 2, 7, [64, 3, 37], [0, 511, 130]),
    ("bf16", 128, 1, 4, [257, 9, 8], [0, 100, 1000]),
    ("bf16", 64, 1, 8, [33, 4, 5, 100], [31, 32, 33, 300]),
    ("bf16", 128, 1, 1, [32, 33, 256, 257, 300], [17, 0, 0, 64, 999]),
    ("bf16", 64, 1, 1, [513, 31], [0, 2000]),
    ("bf16", 128, 1, 64, [3, 1, 0, 5], [70, 5, 8, 300]),
    ("bf16", 128, 1, 5, [13, 6, 7], [5, 48, 49]),
    ("f32", 128, 2, 4, [5, 0, 9], [37, 3, 600]),
    ("f32", 64, 2, 2, [130, 16, 17, 1], [0, 15, 16, 400]),
    ("f32", 128, 1, 7, [50, 4, 5], [0, 129, 1000]),
    ("f32", 64, 1, 6, [22, 1, 90], [64, 0, 33]),
]


@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
@pytest.mark.parametrize("holes", [0.0, 0.35])
@pytest.mark.parametrize("dtype,D,Hkv,G,lens,ctx", ATTN)
def test_chunk_attention(fmt, dtype, D, Hkv, G, lens, ctx, holes):
    rows = [ctx[s] - min(ctx[s], 3 * kv) + lens[s] for s in range(len(lens)) for kv in range(Hkv)]
    c = Cache8(rows, D, fmt, holes=holes, seed=len(lens) + G, keep_last=max(lens))
    _attend(c, lens, Hkv, G, dtype, pad=3, lead=2 if holes else 0)


@pytest.mark.parametrize("fmt,dtype,D,G,lens,ctx,width", [
    ("i8", "bf16", 128, 4, [3], [9000], 4096), ("e4m3", "bf16", 64, 2, [100], [5001], 768),
    ("i8", "bf16", 128, 7, [20, 2], [4000, 300], 300), ("e4m3", "bf16", 128, 1, [700], [2000], 400),
    ("i8", "f32", 64, 4, [2, 60], [4100, 900], 300), ("e4m3", "f32", 128, 1, [1], [6000], 1024)])
def test_chunk_attention_over_ranges(fmt, dtype, D, G, lens, ctx, width):
    c = Cache8([a + b for a, b in zip(ctx, lens)], D, fmt, width=width, holes=0.1, seed=9, keep_last=max(lens))
    _attend(c, lens, 1, G, dtype, pad=1)


@pytest.mark.parametrize("fmt,dtype,D,B,G", [("i8", "bf16", 128, 70, 8), ("e4m3", "bf16", 64, 40, 8), ("i8", "f32", 64, 70, 4)])
def test_many_chunks(fmt, dtype, D, B, G):
    """Launches of many workgroups; rows without pages and chunks that are short among them."""
    lens = [20 - s % 3 - 17 * (s % 9 == 4) for s in range(B)]
    ctx = [(97 * s) % 300 for s in range(B)]
    rows = [lens[s] + max(ctx[s] - 5 * kv, 0) for s in range(B) for kv in range(8)]
    rows[8 * 7 + 3] = 0
    c = Cache8(rows, D, fmt, width=200, seed=3, keep_last=20)
    _attend(c, lens, 8, G, dtype, pad=2, heads=list(range(0, 8 * B, 7)) + [59])


def test_chunks_longer_than_promised_are_cut():
    """max_len bounds the launch: a longer chunk's further tokens are not computed, nothing beside is touched."""
    c = Cache8([200, 60], 128, "i8", seed=5)
    _, o, lse = _attend(c, [50, 20], 1, 2, "bf16", max_len=30, check=False)
    assert (lse[30:50] == -7.0).all() and (o[30:50] == -7.0).all() and torch.isfinite(lse[50:]).all()


def test_strided_queries():
    import paper_2606_28831_amd as hk
    c = Cache8([300], 128, "e4m3", seed=5)
    q, o, lse = _attend(c, [37], 1, 4, "bf16")
    wide = torch.full((37, 9, 128), float("nan"), dtype=torch.bfloat16, device=DEV)
    wide[:, 2:6] = q
    ch, d = _chunks([37]), hk.dims(1, 4, 1, 128)
    ws = hk.chunk_attn8_workspace(d, ch, c.width, DEV)
    o2, lse2 = torch.empty_like(o), torch.empty_like(lse)
    hk.hk_chunk_attn8(d, c.kv, ch, wide[:, 2:6], 1 / math.sqrt(128), o2, ws, lse=lse2)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    hk.hk_chunk_attn8(d, c.kv, ch, wide[:, 2:6], 1 / math.sqrt(128), o2.zero_(), ws)
    assert torch.equal(o, o2)


def test_the_same_call_gives_the_same_bits():
    c = Cache8([4000, 900], 128, "i8", width=400, seed=5, holes=0.1, keep_last=90)
    for run in (lambda: _decode(c, 2, 1, 4, "bf16", check=False), lambda: _attend(c, [7, 90], 1, 4, "bf16", check=False)):
        a, b = run(), run()
        assert torch.equal(a[1], b[1]) and torch.equal(a[2], b[2])


# ------------------------------------------------------------------ the rewrite
@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
@pytest.mark.parametrize("D,L_dense,L_sparse,modes", [
    (128, 0, 0, None), (64, 40, 70, None), (128, 16, 10 ** 6, None), (64, 33, 0, [0, 1, 2]), (128, 0, 0, [2, 2, 0])])
def test_rewrite(fmt, D, L_dense, L_sparse, modes):
    import paper_2606_28831_amd as hk
    lens = [0, 5, 16, 333, 700, 64, 17, 250, 129]
    c = Cache8(lens, D, fmt, holes=0.2, seed=8, spare=150)
    H, S = len(lens), c.width * 16
    rng = np.random.default_rng(2)
    words = rng.integers(0, 2 ** 32, (H, S // 32), dtype=np.uint64).astype(np.uint32)
    words[4] = 0
    words[5] = 0xFFFFFFFF
    sel = torch.tensor(words.view(np.int32), device=DEV)
    mode = None if modes is None else torch.tensor([modes[h % 3] for h in range(H)], dtype=I32, device=DEV)
    d = hk.dims(3, 3, 3, D)
    ws = hk.workspace(hk.OP_COMPACT, d, c.width, DEV)
    status = torch.zeros(1, dtype=I32, device=DEV)
    hk.hk_compact8(d, c.kv, sel, L_dense, L_sparse, c.alloc, status, ws, head_mode=mode)
    assert int(status) == 0
    table, mask, n = np_i(c.page_table), np_i(c.page_mask).astype(np.int64) & 0xFFFF, np_i(c.n_pages)
    codes = {x: np_i(_bytes(getattr(c, x + "_pool"))).reshape(-1, D) for x in "kv"}
    scale = {x: np64(getattr(c, x + "_scale")).reshape(-1) for x in "kv"}
    live = []
    for h in range(H):
        want = rewrite_layout(c.t[h], c.m[h], c.n[h], unpack_bits(words[h], S), L_dense,
                              2 if modes is None else modes[h % 3], L_sparse).pages
        assert int(n[h]) == len(want), h
        assert (table[h, len(want):] == -1).all() and (mask[h, len(want):] == 0).all()
        for p, page in enumerate(want):
            assert mask[h, p] == page.mask
            live.append(int(table[h, p]))
            if page.kind != "new":
                assert table[h, p] == page.phys
                rows = [(page.phys * 16 + t, page.phys * 16 + t) for t in range(16)]
            else:
                rows = [(int(table[h, p]) * 16 + i, src * 16 + t) for i, (src, t) in enumerate(page.src)]
            for to, at in rows:
                for x in "kv":
                    old_c, old_s = getattr(c, x + "_codes"), getattr(c, x + "_sc")
                    assert (codes[x][to] == old_c[at]).all()
                    np.testing.assert_array_equal(scale[x][to], old_s[at])
    top = int(c.free_top)
    free = np_i(c.free_ids)[:top]
    assert len(set(live)) == len(live) and sorted(live + free.tolist()) == list(range(len(c.free)))


def test_rewrite_without_room_changes_nothing():
    import paper_2606_28831_amd as hk
    c = Cache8([400, 300], 128, "i8", seed=1, spare=3)
    before = [x.clone() for x in (c.page_table, c.page_mask, c.n_pages, c.free_ids, c.free_top, _bytes(c.k_pool), c.k_scale)]
    d = hk.dims(2, 1, 1, 128)
    status = torch.zeros(1, dtype=I32, device=DEV)
    sel = torch.full((2, c.width // 2), -1, dtype=I32, device=DEV)
    hk.hk_compact8(d, c.kv, sel, 0, 0, c.alloc, status, hk.workspace(hk.OP_COMPACT, d, c.width, DEV))
    assert int(status) == hk.FLAG_NOSPACE
    for a, b in zip(before, (c.page_table, c.page_mask, c.n_pages, c.free_ids, c.free_top, _bytes(c.k_pool), c.k_scale)):
        assert torch.equal(a.nan_to_num(), b.nan_to_num())


# ------------------------------------------------------------------ chained
def _empty(H, D, fmt, width, pool):
    import paper_2606_28831_amd as hk
    z = lambda *s, dt=torch.uint8: torch.zeros(*s, dtype=dt, device=DEV)  # noqa: E731
    kv = hk.PagedKV8(z(pool, 16, D).fill_(GARBAGE[fmt]).view(CODE[fmt]), z(pool, 16, D).fill_(GARBAGE[fmt]).view(CODE[fmt]),
                     z(pool, 16, dt=torch.float32).fill_(float("nan")), z(pool, 16, dt=torch.float32).fill_(float("nan")),
                     z(H, width, dt=I32) - 1, z(H, width, dt=torch.int16), z(H, dt=I32))
    al = hk.Allocator(z(pool, dt=I32), z(1, dt=I32))
    hk.hk_alloc_init(al, 0, pool)
    return kv, al


@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
def test_a_loop_over_an_8_bit_cache(fmt):
    """Prompts in chunks, single tokens, drafts taken back, compression and more tokens through
    DecodeLoop: every attention call against 64 bits over the rows as they read back."""
    import paper_2606_28831_amd as hk
    from paper_2606_28831_amd.pipeline import DecodeLoop
    L, B, Hq, Hkv, D, W = 2, 2, 8, 2, 128, 4
    G, H = Hq // Hkv, L * B * Hkv
    kv, al = _empty(H, D, fmt, 40, 700)
    loop = DecodeLoop(L, B, Hq, Hkv, D, W, kv, al, 0.9, 64, max_tokens=150)
    g = torch.Generator(device=DEV).manual_seed(3)
    rnd = lambda *s: torch.randn(*s, generator=g, device=DEV).to(torch.bfloat16)  # noqa: E731
    rows = [[] for _ in range(H)]                                     # (k, v) of every head's slots, as written

    def wrote(k, v, lens):                                            # [L, T, Hkv, D]
        at = 0
        for s, n in enumerate(lens):
            for l in range(L):
                for h in range(Hkv):
                    for t in range(at, at + n):
                        pair = []
                        for x in (k, v):
                            c, sc = O8.quantise(np64(x[l, t, h]), fmt)
                            pair.append(O8.values(c, fmt) * sc)
                        rows[(l * B + s) * Hkv + h].append(pair)
            at += n

    def check(h, q, o, lse, dtype, parts):                            # q [n, G, D]
        k, v = (np.array([r[i] for r in rows[h]]) for i in range(2))
        ro, rl, zabs, absv = CO.chunk_attn_head(q, k, v, np.ones(len(k), bool), len(k), 1 / math.sqrt(D))
        bo, bl = _bound(dtype, parts, len(k), rl, zabs, absv, ro, D)
        assert (np.abs(o - ro) <= bo).all() and (np.abs(lse - rl) <= bl).all(), h

    def extend(lens):
        T = sum(lens)
        q, k, v = rnd(L, T, Hq, D), rnd(L, T, Hkv, D), rnd(L, T, Hkv, D)
        o, lse = torch.empty_like(q), torch.empty(L, T, Hq, device=DEV)
        loop.extend(_chunks(lens), q, k, v, o, lse)
        wrote(k, v, lens)
        qn, on, ln = np64(q), np64(o), np64(lse)
        for h in range(H):
            ls, hh = divmod(h, Hkv)
            l, s = divmod(ls, B)
            a, gs = sum(lens[:s]), slice(hh * G, hh * G + G)
            n = lens[s]
            check(h, qn[l, a:a + n, gs], on[l, a:a + n, gs], ln[l, a:a + n, gs], "bf16", 2 if n * G <= 32 else 1)

    lse_win = torch.empty(W, L * B, Hq, device=DEV)
    q_win = rnd(W, L * B, Hq, D)

    def steps():
        for t in range(W):
            k, v = rnd(L * B, Hkv, D), rnd(L * B, Hkv, D)
            loop.step(q_win[t], k, v, lse_win[t])
            wrote(k.view(L, B, Hkv, D), v.view(L, B, Hkv, D), [1] * B)
            qn, on, ln = np64(q_win[t]), np64(loop.o), np64(lse_win[t])
            for h in range(H):
                s, hh = divmod(h, Hkv)
                gs = slice(hh * G, hh * G + G)
                check(h, qn[s:s + 1, gs], on[s:s + 1, gs], ln[s:s + 1, gs], "f32", 3)

    extend([100, 50])
    extend([90, 1])
    steps()
    # drafts, two and one of which are taken back
    extend([5, 3])
    loop.chunked.trim(torch.tensor([2, 1], dtype=I32, device=DEV))
    for h in range(H):
        drop = [2, 1][(h // Hkv) % B]
        rows[h] = rows[h][:-drop]
    steps()
    # compression: the rows that stay are those of the selection, and the dense tier
    n_before = np_i(kv.n_pages)
    loop.compress(q_win, lse_win)
    sel = np.stack([unpack_bits(w.view(np.uint32), 640) for w in np_i(loop.comp.buf.sel_bits)])
    cand = np_i(loop.comp.buf.cand_len)
    for h in range(H):
        c = int(cand[h])
        assert c == 16 * max(0, int(n_before[h]) - 4)
        rows[h] = [r for j, r in enumerate(rows[h]) if j >= c or sel[h, j]]
    assert int(loop.status) == 0 and int(loop.comp.buf.status) == 0
    extend([7, 40])
    steps()
    assert int(loop.status) == 0


@pytest.mark.parametrize("budget", [False, True])
def test_compressors_score_8_bit_rows_as_they_read_back(budget):
    """Scores and selection of an 8-bit cache, in groups of sequences, are those of a bf16 cache that
    holds what its rows read back as."""
    import paper_2606_28831_amd as hk
    from paper_2606_28831_amd.pipeline import BudgetCompressor, Compressor, ScoringCopy
    NS, Hkv, G, D, W = 5, 2, 2, 64, 4
    c = Cache8([100 + 37 * i for i in range(NS * Hkv)], D, "i8", holes=0.1, seed=6, spare=400)
    pools = []
    for codes, s in ((c.k_codes, c.k_sc), (c.v_codes, c.v_sc)):
        x = torch.tensor(O8.values(codes, "i8") * s.astype(np.float64)[:, None]).float().to(torch.bfloat16)
        pools.append(x.to(DEV).view(-1, 16, D))
    kv16 = hk.PagedKV(pools[0], pools[1], c.page_table.clone(), c.page_mask.clone(), c.n_pages.clone())
    al16 = hk.Allocator(c.free_ids.clone(), c.free_top.clone())
    g = torch.Generator(device=DEV).manual_seed(1)
    q = torch.randn(W, NS, Hkv * G, D, generator=g, device=DEV).to(torch.bfloat16)
    made = []
    for kv, al in ((c.kv, c.alloc), (kv16, al16)):
        if budget:
            x = BudgetCompressor(NS, Hkv * G, Hkv, D, W, kv, al, 0.8, 100, 200, L_dense=32, n_sink=4, rank_by_c=True)
        else:
            x = Compressor(NS, Hkv * G, Hkv, D, W, kv, al, 0.8, L_dense=32)
        if kv is c.kv:
            small = ScoringCopy(NS, Hkv * G, Hkv, D, W, kv, max_bytes=2 * Hkv * c.width * 16 * D * 2)
            assert small.n == 2                                        # groups of 2, 2 and 1 sequences
            x.copy = small
            if budget:
                x.buf["ws_score"] = small.ws
            else:
                x.buf.ws_score = small.ws
        x.step(q)
        made.append(x)
    torch.cuda.synchronize()
    a, b = (m.buf if budget else vars(m.buf) for m in made)
    assert int(a["status"]) == 0 and int(b["status"]) == 0
    for name in ("cand_len", "row_lse", "s_attn", "sel_bits", "k") + (("votes", "head_mode") if budget else ()):
        assert torch.equal(a[name], b[name]), name
    assert torch.equal(c.page_mask, kv16.page_mask) and torch.equal(c.n_pages, kv16.n_pages)
    assert torch.equal(c.page_table, kv16.page_table) and torch.equal(c.free_ids, al16.free_ids)


def test_captured_and_replayed_on_another_stream():
    """Append, chunk attention, single tokens, trimming and the rewrite in one graph, replayed with new
    rows between eager calls: the same as eager calls."""
    import paper_2606_28831_amd as hk
    from paper_2606_28831_amd.pipeline import ChunkDecoder, Decoder
    B, Hq, Hkv, D = 2, 4, 2, 64
    kv, al = _empty(B * Hkv, D, "i8", 20, 100)
    chd, dec = ChunkDecoder(B, Hq, Hkv, D, kv, al, 40, 30), Decoder(B, Hq, Hkv, D, kv, al)
    start = torch.tensor([0, 9, 26], dtype=I32, device=DEV)
    ch = hk.Chunks(start, 40, 30)
    g = torch.Generator(device=DEV).manual_seed(2)
    draw = lambda *s: torch.randn(*s, generator=g, device=DEV).to(torch.bfloat16)  # noqa: E731
    k, v, q = draw(40, Hkv, D), draw(40, Hkv, D), draw(40, Hq, D)
    k1, v1, q1 = draw(B, Hkv, D), draw(B, Hkv, D), draw(B, Hq, D)
    sm = torch.empty(40 * Hkv, dtype=torch.int64, device=DEV)
    o, lse = torch.zeros_like(q), torch.zeros(40, Hq, device=DEV)
    o1, lse1 = torch.zeros(B, Hq, D, device=DEV), torch.zeros(B, Hq, device=DEV)
    drop = torch.tensor([1, 0], dtype=I32, device=DEV)
    sel = torch.full((B * Hkv, 10), 0x5F5F5F5F, dtype=I32, device=DEV)
    d, status = hk.dims(B, Hq, Hkv, D), torch.zeros(1, dtype=I32, device=DEV)
    ws = hk.workspace(hk.OP_COMPACT, d, 20, DEV)

    def work():
        chd.append(ch, k, v, sm)
        chd.attend(ch, q, o, lse)
        dec.append(k1, v1)
        dec.attend(q1, o1, lse1)
        chd.trim(drop)
        hk.hk_compact8(d, kv, sel, 16, 0, al, status, ws)

    tensors = (kv.page_table, kv.page_mask, kv.n_pages, al.free_ids, al.free_top, _bytes(kv.k_pool), _bytes(kv.v_pool),
               kv.k_scale, kv.v_scale)
    clean = [t.clone() for t in tensors]
    outs = (o, lse, o1, lse1, kv.page_table, kv.page_mask, kv.n_pages, al.free_top, kv.k_scale)

    def reset(i):
        for t, x in zip(tensors, clean):
            t.copy_(x)
        for t in (o, lse, o1, lse1):                                  # (rows behind the last chunk stay as they are)
            t.zero_()
        gi = torch.Generator(device=DEV).manual_seed(100 + i)
        for t in (k, v, q, k1, v1, q1):
            t.copy_(torch.randn(t.shape, generator=gi, device=DEV))
        start.copy_(torch.tensor([0, 9 + i, 26 - i], dtype=I32))

    want = []
    for i in range(4):
        reset(i)
        work()
        work()
        torch.cuda.synchronize()
        want.append([t.clone() for t in outs])
    reset(0)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        work()
    for i in (0, 3, 1, 2, 0):
        reset(i)
        torch.cuda.synchronize()
        graph.replay()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, want[i]):
            assert torch.equal(a.nan_to_num(9.0), b.nan_to_num(9.0))
    assert int(status) == 0 and int(chd.status) == 0 and int(dec.status) == 0


@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
def test_a_captured_segment_of_a_loop(fmt):
    """Steps and their compression through DecodeLoop in one graph, replayed between eager work: the same as eager."""
    from paper_2606_28831_amd.pipeline import DecodeLoop
    L, B, Hq, Hkv, D, W = 2, 2, 4, 2, 64, 6
    H, loops = L * B * Hkv, []
    for _ in range(2):
        kv, al = _empty(H, D, fmt, 40, 400)
        loops.append(DecodeLoop(L, B, Hq, Hkv, D, W, kv, al, 0.9, 32))
    q, k, v = (torch.empty(W, L * B, h, D, dtype=torch.bfloat16, device=DEV) for h in (Hq, Hkv, Hkv))
    lse = torch.empty(W, L * B, Hq, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(8)

    def fill():
        for t in (q, k, v):
            t.copy_(torch.randn(t.shape, generator=g, device=DEV))

    fill()
    loops[0].segment(q, k, v, lse)
    loops[1].segment(q, k, v, lse)
    graph = loops[1].capture_segment(q, k, v, lse)
    for _ in range(12):
        fill()
        loops[0].segment(q, k, v, lse)
        torch.cuda.synchronize()
        want = lse.clone(), loops[0].o.clone()
        lse.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(lse, want[0]) and torch.equal(loops[1].o, want[1])
        for name in ("page_table", "page_mask", "n_pages"):
            assert torch.equal(getattr(loops[0].kv, name), getattr(loops[1].kv, name)), name
    assert all(int(x.status) == 0 and int(x.comp.buf.status) == 0 for x in loops)
    assert int(loops[0].kv.n_pages.max()) > 2


def test_calls_on_a_stream_of_their_own():
    import paper_2606_28831_amd as hk
    c = Cache8([500, 60], 128, "e4m3", seed=5)
    q, o, lse = _decode(c, 2, 1, 4, "bf16")
    d = hk.dims(2, 4, 1, 128)
    ws, o2, l2 = hk.workspace(hk.OP_DECODE8, d, c.width, DEV), torch.zeros_like(o), torch.zeros_like(lse)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    hk.hk_decode_attn8(d, q, c.kv, 1 / math.sqrt(128), o2, l2, ws, stream=s)
    s.synchronize()
    assert torch.equal(o, o2) and torch.equal(lse, l2)


def test_offsets_past_32_bits():
    """Pages past 2^31 bytes of a pool: rows written, read back, attended to and rewritten there."""
    import paper_2606_28831_amd as hk
    D, pool = 128, (1 << 21) + 4096                                   # 4 GiB and a little per pool
    first = pool - 40
    kp, vp = (torch.empty(pool, 16, D, dtype=torch.int8, device=DEV) for _ in range(2))
    ks, vs = (torch.empty(pool, 16, device=DEV) for _ in range(2))
    t = torch.full((1, 20), -1, dtype=I32, device=DEV)
    t[0, :10] = torch.arange(first, first + 10, dtype=I32)
    m = torch.zeros(1, 20, dtype=torch.int16, device=DEV)
    m[0, :10] = -1
    n = torch.tensor([10], dtype=I32, device=DEV)
    kv = hk.PagedKV8(kp, vp, ks, vs, t, m, n)
    free = torch.zeros(pool, dtype=I32, device=DEV)
    free[:20] = torch.arange(first + 10, first + 30, dtype=I32)
    al = hk.Allocator(free, torch.tensor([20], dtype=I32, device=DEV))
    g = torch.Generator(device=DEV).manual_seed(1)
    k, v = (torch.randn(160, 1, D, generator=g, device=DEV) for _ in range(2))
    sm = first * 16 + torch.arange(160, device=DEV)
    d = hk.dims(1, 2, 1, D)
    hk.hk_write_kv8(d, kv, 160, sm, k, v)
    rk, rv = torch.zeros_like(k), torch.zeros_like(v)
    hk.hk_read_kv8(d, kv, 160, sm, rk, rv)
    assert ((rk - k).abs() <= k.abs().amax(-1, keepdim=True) / 250).all()
    q = torch.randn(1, 2, D, generator=g, device=DEV)
    o, lse = torch.zeros(1, 2, D, device=DEV), torch.zeros(1, 2, device=DEV)
    ws = hk.workspace(hk.OP_DECODE8, d, 20, DEV)

    def check(keep):
        hk.hk_decode_attn8(d, q, kv, 0.1, o, lse, ws)
        kk, vv = np64(rk)[keep, 0], np64(rv)[keep, 0]
        ro, rl, zabs, absv = CO.chunk_attn_head(np64(q), kk, vv, np.ones(len(kk), bool), len(kk), 0.1)
        bo, bl = _bound("f32", 3, len(kk), rl, zabs, absv, ro, D)
        assert (np.abs(np64(o) - ro) <= bo).all() and (np.abs(np64(lse) - rl) <= bl).all()

    check(np.arange(160))
    sel = torch.full((1, 10), 0x0F0F0F0F, dtype=I32, device=DEV)
    status = torch.zeros(1, dtype=I32, device=DEV)
    hk.hk_compact8(d, kv, sel, 0, 0, al, status, hk.workspace(hk.OP_COMPACT, d, 20, DEV))
    assert int(status) == 0 and int(n) == 5 and int(t[0, 0]) >= first + 10
    check(np.array([j for j in range(160) if j % 8 < 4]))
