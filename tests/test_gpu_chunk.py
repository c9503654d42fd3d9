"""Calls with several new tokens per sequence on the GPU against the oracle: slots, rows, attention,
drafts, and all of them chained.  Pools are filled with NaN wherever no token was written, so that
anything read from a masked slot, a page's tail or a free page shows."""
import math

import numpy as np
import pytest
import torch

import oracle.chunk_oracle as CO
from hk_testlib import np64, np_i

pytestmark = pytest.mark.gpu
DEV = "cuda"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
I32 = torch.int32


class Cache:
    """A paged cache of given row lengths with its tables on the host; every slot of the pool that
    holds no valid token is NaN."""

    def __init__(self, lens, D, dtype, width=None, holes=0.0, seed=0, spare=200, keep_last=0, v_scale=1.0,
                 first_page=0, k_scale=1.0):
        import paper_2606_28831_amd as hk
        rng = np.random.default_rng(seed)
        H, pages = len(lens), [-(-x // 16) for x in lens]
        self.width = max(pages + [2]) if width is None else width
        self.width += self.width % 2
        pool = sum(pages) + spare + first_page
        perm = first_page + rng.permutation(sum(pages) + spare)
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
        self.top = len(perm) - at
        self.free[:self.top] = perm[at:]
        dt = DT[dtype]
        k = torch.full((pool * 16, D), float("nan"), dtype=dt, device=DEV)
        v = k.clone()
        rows = torch.tensor(self.rows_of_all(), dtype=torch.long, device=DEV)
        g = torch.Generator(device=DEV).manual_seed(seed + 1)
        if len(rows):
            k[rows] = (torch.randn(len(rows), D, generator=g, device=DEV) * k_scale).to(dt)
            v[rows] = (torch.randn(len(rows), D, generator=g, device=DEV) * v_scale).to(dt)
        self.k_pool, self.v_pool = k.view(pool, 16, D), v.view(pool, 16, D)
        put = lambda x, d: torch.tensor(x, device=DEV).to(d)  # noqa: E731
        self.page_table, self.n_pages = put(self.t, I32), put(self.n, I32)
        self.page_mask = put(self.m, I32).to(torch.int16)
        self.free_ids, self.free_top = put(self.free, I32), put(np.array([self.top]), I32)
        self.kv = hk.PagedKV(self.k_pool, self.v_pool, self.page_table, self.page_mask, self.n_pages)
        self.alloc = hk.Allocator(self.free_ids, self.free_top)

    def slots(self, h):
        return [j for j in range(16 * int(self.n[h])) if self.m[h, j // 16] >> (j % 16) & 1]

    def rows_of_all(self):
        return [int(self.t[h, j // 16]) * 16 + j % 16 for h in range(len(self.n)) for j in self.slots(h)]

    def head(self, h):
        """keys, vals, valid, end of one head from the device pools and the host tables."""
        n, D = int(self.n[h]), self.k_pool.shape[2]
        if n == 0:
            return np.zeros((0, D)), np.zeros((0, D)), np.zeros(0, bool), 0
        ids = torch.tensor(self.t[h, :n], device=DEV)
        valid = np.array([(self.m[h, j // 16] >> (j % 16)) & 1 for j in range(16 * n)], bool)
        k, v = (np64(x[ids].reshape(-1, D)) for x in (self.k_pool, self.v_pool))
        k[~valid], v[~valid] = 0.0, 0.0
        return k, v, valid, CO.row_end(self.m[h], n)

    def check(self, what=""):
        """The device tables against the host's."""
        top = int(self.free_top.item())
        assert top == self.top, what
        assert (np_i(self.n_pages) == self.n).all(), what
        assert (np_i(self.page_table) == self.t).all(), what
        assert ((np_i(self.page_mask).astype(np.int64) & 0xFFFF) == self.m).all(), what
        assert (np_i(self.free_ids)[:top] == self.free[:top]).all(), what


def _chunks(lens, pad=0, max_len=None, lead=0):
    import paper_2606_28831_amd as hk
    start = np.concatenate([[0], np.cumsum(lens)]) + lead
    return hk.Chunks(torch.tensor(start, dtype=I32, device=DEV), int(start[-1]) + pad, max_len or max(max(lens), 1))


def _bound(dtype, n_keys, lse, zabs, absv, o, D):
    """Error bounds of (o, lse) against 64 bits, term by term:
      scores   D products summed in fp32 (each addition off by at most 2^-23, the matrix cores cut), and
               the scaling: dz = (D + 8) 2^-23 max sum |q k|;
      sums     probabilities off by 2 dz each and a few steps of the exponential, the running sum's n
               additions over 64 lanes at least, the states' joins: (n / 32 + 64) 2^-23;
      bf16     P rounded before the product with V, 2^-8 of every term, and the output, 2^-8."""
    dz = (D + 8) * 2.0 ** -23 * zabs
    rest = (n_keys / 32 + 64) * 2.0 ** -23
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    p = half if dtype == "bf16" else 0.0
    bo = half * np.abs(o) * 1.01 + (p + 2 * dz[..., None] + 2 * rest) * 1.05 * absv
    return bo, dz + rest + 2.0 ** -22 * np.maximum(1.0, np.abs(np.where(np.isfinite(lse), lse, 0.0)))


def _check_attn(c, ch_lens, first, q, o, lse, Hkv, G, scale, dtype, D, heads=None):
    qn, on, ln = np64(q), np64(o), np64(lse)
    for h in range(len(ch_lens) * Hkv) if heads is None else heads:
        s, kv = divmod(h, Hkv)
        n, a = ch_lens[s], first[s]
        if n == 0:
            continue
        k, v, valid, end = c.head(h)
        g = slice(kv * G, kv * G + G)
        ro, rl, zabs, absv = CO.chunk_attn_head(qn[a:a + n, g], k, v, valid, end, scale)
        bo, bl = _bound(dtype, len(valid), rl, zabs, absv, ro, D)
        got_o, got_l = on[a:a + n, g], ln[a:a + n, g]
        assert (np.isneginf(got_l) == np.isneginf(rl)).all(), f"head {h}: empty rows"
        fin = np.isfinite(rl)
        assert np.isfinite(got_l[fin]).all() and np.isfinite(got_o).all(), f"head {h}: not finite"
        worst = np.max(np.abs(got_o - ro) / np.maximum(bo, 1e-300)) if bo.size else 0
        assert (np.abs(got_o - ro) <= bo).all(), f"head {h}: o is {worst:.2f} bounds off"
        assert (np.abs(got_l[fin] - rl[fin]) <= bl[fin]).all(), f"head {h}: lse"
        assert (got_o[~fin] == 0).all()


def _attend(c, lens, Hkv, G, D, dtype, seed=5, pad=0, lead=0, max_len=None, q_scale=1.0, check=True, heads=None, ws_fill=255):
    import paper_2606_28831_amd as hk
    ch = _chunks(lens, pad, max_len, lead)
    T, Hq, B = ch.n_tokens, Hkv * G, len(lens)
    g = torch.Generator(device=DEV).manual_seed(seed)
    q = (torch.randn(T, Hq, D, generator=g, device=DEV) * q_scale).to(DT[dtype])
    o = torch.full((T, Hq, D), -7.0, dtype=DT[dtype], device=DEV)
    lse = torch.full((T, Hq), -7.0, device=DEV)
    d = hk.dims(B, Hq, Hkv, D)
    ws = hk.chunk_attn_workspace(d, ch, c.width, DEV)
    ws.fill_(ws_fill)
    scale = 1 / math.sqrt(D)
    hk.hk_chunk_attn(d, c.kv, ch, q, scale, o, ws, lse=lse)
    torch.cuda.synchronize()
    used = sum(lens)
    for t in (o, lse):
        assert (t[:lead] == -7.0).all() and (t[lead + used:] == -7.0).all(), "padding rows were written"
    if check:
        first = [lead + sum(lens[:s]) for s in range(B)]
        _check_attn(c, lens, first, q, o, lse, Hkv, G, scale, dtype, D, heads)
    return q, o, lse


# ------------------------------------------------------------------ attention
# chunk lengths from nothing to several tiles, contexts from nothing on, at every edge of a page, a
# key block and a row tile; masked slots; groups that divide a tile and that do not
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


@pytest.mark.parametrize("holes", [0.0, 0.35])
@pytest.mark.parametrize("dtype,D,Hkv,G,lens,ctx", ATTN)
def test_chunk_attention(dtype, D, Hkv, G, lens, ctx, holes):
    rows = [ctx[s] - min(ctx[s], 3 * kv) + lens[s] for s in range(len(lens)) for kv in range(Hkv)]
    c = Cache(rows, D, dtype, holes=holes, seed=len(lens) + G, keep_last=max(lens))
    _attend(c, lens, Hkv, G, D, dtype, pad=3, lead=2 if holes else 0)


@pytest.mark.parametrize("dtype,D,G,lens,ctx,width", [
    ("bf16", 128, 4, [3], [9000], 4096),             # one row over many splits
    ("bf16", 64, 2, [100], [5001], 768),             # one tile over many splits
    ("bf16", 128, 7, [20, 2], [4000, 300], 300),     # a split tile and rows with fewer splits
    ("bf16", 128, 1, [700], [2000], 400),
    ("f32", 64, 4, [2, 60], [4100, 900], 300),
    ("f32", 128, 1, [1], [6000], 1024)])
def test_chunk_attention_over_splits(dtype, D, G, lens, ctx, width):
    c = Cache([a + b for a, b in zip(ctx, lens)], D, dtype, width=width, holes=0.1, seed=9, keep_last=max(lens))
    _attend(c, lens, 1, G, D, dtype, pad=1)


@pytest.mark.parametrize("dtype,D,B,G", [("bf16", 128, 40, 8), ("bf16", 64, 70, 8), ("f32", 64, 40, 8), ("f32", 128, 70, 8)])
def test_more_tiles_than_workgroups(dtype, D, B, G):
    """Tables wide enough for tiles in pieces: workgroups with several pieces (B 40), a launch of too many
    tiles for that (B 70); rows without pages and chunks that are short among them."""
    lens = [20 - s % 3 - 17 * (s % 9 == 4) for s in range(B)]
    ctx = [(97 * s) % 300 for s in range(B)]
    rows = [lens[s] + max(ctx[s] - 5 * kv, 0) for s in range(B) for kv in range(8)]
    rows[8 * 7 + 3] = 0
    c = Cache(rows, D, dtype, width=200, seed=3, keep_last=20)
    _attend(c, lens, 8, G, D, dtype, pad=2)


def test_sharp_and_flat_scores():
    """Scores hundreds apart: the running reference moves in almost every block."""
    for dtype in ("bf16", "f32"):
        c = Cache([1500, 90], 128, dtype, seed=21, holes=0.1, keep_last=70)
        _attend(c, [70, 2], 1, 4, 128, dtype, q_scale=30.0)
        _attend(c, [70, 2], 1, 4, 128, dtype, q_scale=1e-3)


def test_queries_that_see_nothing():
    """Chunks longer than their row, rows without a valid slot, rows without a page: o = 0, lse = -inf."""
    for dtype in ("bf16", "f32"):
        c = Cache([4, 40, 0, 20, 700], 64, dtype, seed=2, keep_last=40)
        c.m[1, :], c.m[3, 1] = 0, 0                  # nothing valid; an empty newest page
        c.page_mask.copy_(torch.tensor(c.m, device=DEV).to(torch.int16))
        q, o, lse = _attend(c, [9, 3, 2, 3, 60], 1, 3, 64, dtype)
        assert torch.isneginf(lse[:5]).all() and torch.isfinite(lse[5:9]).all()
        assert torch.isneginf(lse[9:14]).all() and (o[9:14] == 0).all()


def test_values_near_the_end_of_the_range():
    for dtype in ("bf16", "f32"):
        c = Cache([2000, 3000], 128, dtype, seed=4, keep_last=60)
        c.v_pool.copy_(torch.where(torch.isnan(c.v_pool), c.v_pool, torch.full_like(c.v_pool, 3e38)))
        q, o, lse = _attend(c, [2, 60], 1, 4, 128, dtype, check=False)
        assert torch.isfinite(o).all() and ((o.float() / 3e38 - 1).abs() < 0.01).all()


@pytest.mark.parametrize("dtype,D,G,n", [("bf16", 128, 2, 40), ("bf16", 64, 3, 9), ("f32", 128, 1, 40), ("f32", 64, 4, 3)])
def test_infinite_rows_of_unseen_tokens_do_not_matter(dtype, D, G, n):
    """Later tokens' infinite K and V change nothing for the tokens before them; those that see them
    have what the formula gives."""
    L = 310
    c = Cache([L], D, dtype, seed=6, keep_last=n)
    q, o, lse = _attend(c, [n], 1, G, D, dtype)
    j = L - n + n // 2                               # the token in the middle of the chunk, and the last
    for x in (j, L - 1):
        page, slot = int(c.t[0, x // 16]), x % 16
        c.v_pool[page, slot, 3], c.v_pool[page, slot, D - 1] = float("inf"), float("nan")
    c.k_pool[int(c.t[0, (L - 1) // 16]), (L - 1) % 16] = float("inf")
    q2, o2, lse2 = _attend(c, [n], 1, G, D, dtype, check=False)
    m = n // 2
    assert torch.equal(o[:m], o2[:m]) and torch.equal(lse[:n - 1], lse2[:n - 1])
    odd = torch.tensor([3, D - 1], device=DEV)
    assert torch.isposinf(o2[m:n - 1, :, 3]).all() and torch.isnan(o2[m:n - 1, :, D - 1]).all()
    rest = torch.ones(D, dtype=torch.bool, device=DEV)
    rest[odd] = False
    torch.testing.assert_close(o2[m:n - 1][..., rest], o[m:n - 1][..., rest], rtol=2 ** -6 if dtype == "bf16" else 1e-5,
                               atol=2 ** -8 if dtype == "bf16" else 1e-6)
    assert torch.isnan(lse2[n - 1]).all()


def test_single_tokens_agree_with_decode():
    import paper_2606_28831_amd as hk
    from paper_2606_28831_amd.pipeline import Decoder
    for dtype, D, G in (("bf16", 128, 4), ("f32", 64, 2), ("bf16", 64, 8)):
        Hkv, B = 2, 3
        c = Cache([100, 33, 1, 900, 16, 2500], D, dtype, seed=8, holes=0.2)
        q, o, lse = _attend(c, [1] * B, Hkv, G, D, dtype)
        for pool in (c.k_pool, c.v_pool):                # decode multiplies what masked slots hold by 0
            pool.nan_to_num_(nan=0.0)
        dec = Decoder(B, Hkv * G, Hkv, D, c.kv, c.alloc)
        od, ld = torch.empty(B, Hkv * G, D, device=DEV), torch.empty(B, Hkv * G, device=DEV)
        dec.attend(q, od, ld)
        torch.testing.assert_close(lse, ld, rtol=0, atol=2e-5)
        torch.testing.assert_close(o.float(), od, rtol=0, atol=0.02 if dtype == "bf16" else 1e-5)


def test_query_views_streams_and_no_lse():
    """Q as a slice of a projection of Q, K and V; another stream; no LSE: the same bits."""
    import paper_2606_28831_amd as hk
    Hkv, G, D, lens = 2, 4, 128, [70, 3, 1]
    c = Cache([200, 190, 50, 40, 3, 9], D, "bf16", seed=12, keep_last=70)
    q, o, lse = _attend(c, lens, Hkv, G, D, "bf16")
    T = q.shape[0]
    packed = torch.full((T, Hkv * G + 2 * Hkv, D), float("nan"), dtype=torch.bfloat16, device=DEV)
    packed[:, :Hkv * G] = q
    ch, d = _chunks(lens), hk.dims(3, Hkv * G, Hkv, D)
    o2 = torch.empty_like(o)
    ws = hk.chunk_attn_workspace(d, ch, c.width, DEV)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    hk.hk_chunk_attn(d, c.kv, ch, packed[:, :Hkv * G], 1 / math.sqrt(D), o2, ws, stream=st)
    st.synchronize()
    assert torch.equal(o, o2)


def test_tensors_on_other_devices_are_refused():
    """Any one of a call's tensors in host memory: an error before the launch."""
    import paper_2606_28831_amd as hk
    c = Cache([20, 30], 64, "bf16", seed=1)
    d, ch = hk.dims(1, 4, 2, 64), _chunks([3])
    q = torch.zeros(3, 4, 64, dtype=torch.bfloat16, device=DEV)
    k, sm = torch.zeros(3, 2, 64, dtype=torch.bfloat16, device=DEV), torch.full((6,), -1, dtype=torch.int64, device=DEV)
    ws, n = torch.empty(1 << 22, dtype=torch.uint8, device=DEV), torch.zeros(1, dtype=I32, device=DEV)
    away = hk.Chunks(ch.start.cpu(), 3, 3)
    p, u, tok = torch.ones(3, 8, device=DEV), torch.zeros(3, device=DEV), torch.zeros(3, dtype=I32, device=DEV)
    for f, args in ((lambda q, o, ws: hk.hk_chunk_attn(d, c.kv, ch, q, 0.1, o, ws), (q, q.clone(), ws)),
                    (lambda a, b, s: hk.hk_write_kv(d, c.kv, 3, s, a, b), (k, k, sm)),
                    (lambda s, w: hk.hk_reserve_slots(d, c.kv, ch, c.alloc, w, slot_map=s), (sm, ws)),
                    (lambda x, w: hk.hk_trim_slots(d, c.kv, x, c.alloc, w), (n, ws)),
                    (lambda t, q, u, x, w: hk.hk_verify_draft(ch, 8, t, p, u, x, x.clone(), x.clone(), w, q=q), (tok, p, u, n, ws))):
        for i in range(len(args)):
            with pytest.raises(hk.HardKVError):
                f(*(x.cpu() if i == j else x for j, x in enumerate(args)))
    with pytest.raises(hk.HardKVError):
        hk.hk_chunk_attn(d, c.kv, away, q, 0.1, q.clone(), ws)
    c.check()


def test_infinite_rows_in_pieces():
    """The same over rows in several pieces: unseen infinite rows of the newest pages change nothing."""
    for dtype, D, G, n in (("bf16", 128, 4, 70), ("bf16", 64, 3, 60), ("f32", 64, 4, 70)):
        L = 6000
        c = Cache([L], D, dtype, seed=36, keep_last=n, width=512)
        q, o, lse = _attend(c, [n], 1, G, D, dtype)
        for x in range(L - n // 2, L):
            c.v_pool[int(c.t[0, x // 16]), x % 16] = float("inf") if x % 2 else float("nan")
        q2, o2, lse2 = _attend(c, [n], 1, G, D, dtype, check=False)
        m = n - n // 2
        assert torch.equal(o[:m], o2[:m]) and torch.equal(lse, lse2)
        assert not torch.isfinite(o2[m:]).any()


def test_graphs_of_one_workspace():
    """Two captured calls of different sizes on one workspace, replayed in turn over other lengths: tiles in
    pieces, whole tiles and short rows, each replay equal to the eager call."""
    import paper_2606_28831_amd as hk
    Hkv, G, D, width = 2, 4, 128, 300
    c = Cache([4000, 3000, 700, 690, 2500, 2600], D, "bf16", seed=31, width=width, keep_last=300, holes=0.1)
    d, scale = hk.dims(3, Hkv * G, Hkv, D), 1 / math.sqrt(D)
    calls, ws = [], None
    for T, most in ((400, 300), (24, 8)):
        start = torch.zeros(4, dtype=I32, device=DEV)
        ch = hk.Chunks(start, T, most)
        q = torch.zeros(T, Hkv * G, D, dtype=torch.bfloat16, device=DEV)
        o = [torch.zeros_like(q) for _ in range(2)]
        lse = [torch.zeros(T, Hkv * G, device=DEV) for _ in range(2)]
        ws = hk.chunk_attn_workspace(d, ch, width, DEV) if ws is None else ws     # the larger call's
        own = hk.chunk_attn_workspace(d, ch, width, DEV)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            hk.hk_chunk_attn(d, c.kv, ch, q, scale, o[1], ws, lse=lse[1])
        calls.append((ch, start, q, o, lse, own, graph))
    for lens in (([300, 1, 99], [8, 8, 8]), ([1, 2, 3], [1, 0, 8]), ([0, 0, 300], [0, 0, 0]), ([130, 140, 130], [5, 6, 7])):
        for (ch, start, q, o, lse, own, graph), n in zip(calls, lens):
            start.copy_(torch.tensor(np.concatenate([[0], np.cumsum(n)]), device=DEV).to(I32))
            q.copy_(torch.randn(q.shape, device=DEV).bfloat16())
            hk.hk_chunk_attn(d, c.kv, ch, q, scale, o[0], own, lse=lse[0])
        for _ in range(2):
            for call in calls:
                call[6].replay()
        torch.cuda.synchronize()
        for ch, start, q, o, lse, own, graph in calls:
            assert torch.equal(o[0], o[1]) and torch.equal(lse[0], lse[1]), lens


def test_chunks_out_of_bounds_stay_in_bounds():
    """Starts outside the rows or descending, chunks over max_len: every access stays within the rows,
    and the sequences that are as promised have their results."""
    import paper_2606_28831_amd as hk
    c = Cache([50, 60, 70], 64, "bf16", seed=14, keep_last=20)
    T, d = 24, hk.dims(3, 2, 1, 64)
    q = torch.randn(T + 8, 2, 64, device=DEV).bfloat16()
    for start, good in (([0, 6, 40, 50], [0]), ([-5, 3, 3, 9], [2]), ([0, 20, 10, 24], []), ([0, 4, 24, 24], [0])):
        ch = hk.Chunks(torch.tensor(start, dtype=I32, device=DEV), T, 12)
        o = torch.full((T + 8, 2, 64), -7.0, dtype=torch.bfloat16, device=DEV)
        lse = torch.full((T + 8, 2), -7.0, device=DEV)
        hk.hk_chunk_attn(d, c.kv, ch, q, 0.125, o, hk.chunk_attn_workspace(d, ch, c.width, DEV), lse=lse)
        torch.cuda.synchronize()
        assert (o[T:] == -7.0).all() and (lse[T:] == -7.0).all()
        for s in good:
            n, a = start[s + 1] - start[s], start[s]
            k, v, valid, end = c.head(s)
            ro, rl, zabs, absv = CO.chunk_attn_head(np64(q[a:a + n]), k, v, valid, end, 0.125)
            bo, _ = _bound("bf16", len(valid), rl, zabs, absv, ro, 64)
            assert (np.abs(np64(o[a:a + n]) - ro) <= bo).all()


def test_pages_past_32_bit_offsets():
    """Pages whose byte and element offsets pass 2^32 and 2^31."""
    D, first = 128, (1 << 20) + 5000                  # 16 x 128 elements a page
    c = Cache([700, 20], D, "bf16", seed=15, keep_last=64, first_page=first)
    assert c.t[0, 0] * 16 * D > 1 << 31 and c.t[0, 0] * 16 * D * 2 > 1 << 32
    _attend(c, [64, 3], 1, 4, D, "bf16")


def test_graph_serves_every_mixture():
    """One captured step (slots, rows, attention, trim) replayed over other lengths, contents and
    random sizes equals the eager step, bit for bit."""
    import paper_2606_28831_amd as hk
    from paper_2606_28831_amd.pipeline import ChunkDecoder
    B, Hkv, G, D, T, most = 4, 2, 4, 128, 120, 60
    ctx = [100, 80, 7, 0, 33, 200, 16, 15]
    made = [Cache(ctx, D, "bf16", seed=16, width=24) for _ in range(2)]
    decs = [ChunkDecoder(B, Hkv * G, Hkv, D, c.kv, c.alloc, T, most) for c in made]
    start = torch.zeros(B + 1, dtype=I32, device=DEV)
    ch = hk.Chunks(start, T, most)
    q = torch.zeros(T, Hkv * G, D, dtype=torch.bfloat16, device=DEV)
    k, v = (torch.zeros(T, Hkv, D, dtype=torch.bfloat16, device=DEV) for _ in "kv")
    drop = torch.zeros(B, dtype=I32, device=DEV)
    outs = [(torch.zeros(T, Hkv * G, D, dtype=torch.bfloat16, device=DEV), torch.zeros(T, Hkv * G, device=DEV),
             torch.zeros(1, T, Hkv, dtype=torch.int64, device=DEV)) for _ in range(2)]

    def step(i):
        o, lse, sm = outs[i]
        decs[i].append(ch, k, v, sm)
        decs[i].attend(ch, q, o, lse)
        decs[i].trim(drop)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(1)
    rng = np.random.default_rng(3)
    for rep, lens in enumerate([[60, 1, 0, 50], [1, 1, 1, 1], [0, 0, 0, 0], [3, 40, 9, 60], [8, 8, 8, 8]]):
        start.copy_(torch.tensor(np.concatenate([[0], np.cumsum(lens)]), device=DEV).to(I32))
        drop.copy_(torch.tensor([int(rng.integers(0, x + 1)) for x in lens], device=DEV).to(I32))
        for t in (q, k, v):
            t.copy_(torch.randn(t.shape, device=DEV).bfloat16())
        step(0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(*outs):
            assert torch.equal(a, b), rep
        for name in ("page_table", "page_mask", "n_pages", "free_top", "free_ids"):
            assert torch.equal(getattr(made[0], name), getattr(made[1], name)), (rep, name)
        for name in ("k_pool", "v_pool"):
            assert torch.equal(getattr(made[0], name).view(torch.int16), getattr(made[1], name).view(torch.int16)), rep
    assert int(decs[0].status.item()) == int(decs[1].status.item()) == 0


# ------------------------------------------------------------------ slots
def _reserve(c, lens, Hkv, layers, pad=0, lead=0, max_len=None, ch=None, slot_map=True):
    import paper_2606_28831_amd as hk
    ch = ch or _chunks(lens, pad, max_len, lead)
    d = hk.dims(layers * len(lens), Hkv, Hkv, c.k_pool.shape[2])
    sm = torch.full((layers, ch.n_tokens, Hkv), -9, dtype=torch.int64, device=DEV) if slot_map else None
    status = torch.zeros(1, dtype=I32, device=DEV)
    ws = hk.workspace(hk.OP_RESERVE, d, c.width, DEV)
    ws.fill_(0x5a)
    hk.hk_reserve_slots(d, c.kv, ch, c.alloc, ws, slot_map=sm, status=status)
    torch.cuda.synchronize()
    return ch, sm, int(status.item())


SLOTS = [  # layers, Hkv, lens, contexts per (layer, sequence, head), holes
    (1, 1, [1], [0], 0.0),
    (1, 2, [5, 0, 17], [0, 15, 16, 17, 31, 32], 0.3),
    (3, 2, [4, 40], [3, 12, 64, 0, 1, 47, 48, 49, 160, 161, 15, 14], 0.0),
    (2, 1, [300, 0, 1, 16, 15], [0, 9, 31, 100, 1, 16, 0, 2, 3, 250], 0.2),
    (1, 3, [33] * 50, [(7 * i) % 90 for i in range(150)], 0.1),      # several count blocks of 64 heads
    (16, 8, [1, 2, 3, 4, 5, 0, 17, 1], [(11 * i) % 40 for i in range(16 * 64)], 0.0),
]


@pytest.mark.parametrize("layers,Hkv,lens,ctx,holes", SLOTS)
def test_reserve_write_and_trim(layers, Hkv, lens, ctx, holes):
    """Tables, masks, pops, slot map and rows against the oracle; then part of it, then everything
    taken back."""
    import paper_2606_28831_amd as hk
    D = 64
    c = Cache(ctx, D, "bf16", holes=holes, seed=len(ctx), width=max(ctx) // 16 + max(lens) // 16 + 3, spare=3 * len(ctx) * (2 + max(lens) // 16))
    ok, t, m, n, top, slots = CO.reserve(c.t, c.m, c.n, c.free, c.top, lens, Hkv)
    assert ok
    lead, pad = 1, 4
    ch, sm, status = _reserve(c, lens, Hkv, layers, pad=pad, lead=lead)
    before = (c.t, c.m, c.n, c.top)
    c.t, c.m, c.n, c.top = t, m, n, top
    assert status == 0
    c.check("reserve")
    got, B, T = np_i(sm), len(lens), ch.n_tokens
    first = [lead + sum(lens[:s]) for s in range(B)]
    used = np.zeros(T, bool)
    for s in range(B):
        used[first[s]:first[s] + lens[s]] = True
        for l in range(layers):
            for kv in range(Hkv):
                assert got[l, first[s]:first[s] + lens[s], kv].tolist() == slots[((l * B) + s) * Hkv + kv]
    assert (got[:, ~used] == -1).all()
    # rows of a projection's output; what lies beside them is not touched
    packed = torch.randn(layers, T, 2 * Hkv + 1, D, device=DEV).bfloat16()
    k_before, v_before = c.k_pool.clone(), c.v_pool.clone()
    d = hk.dims(B, Hkv, Hkv, D)
    hk.hk_write_kv(d, c.kv, T, sm, packed[:, :, 1:Hkv + 1], packed[:, :, Hkv + 1:])
    torch.cuda.synchronize()
    at = torch.tensor(got[:, used].reshape(-1), device=DEV)
    for pool, old, x in ((c.k_pool, k_before, packed[:, :, 1:Hkv + 1]), (c.v_pool, v_before, packed[:, :, Hkv + 1:])):
        want = old.view(-1, D).clone()
        if at.numel():
            want[at] = x[:, torch.tensor(used, device=DEV)].reshape(-1, D)
        assert torch.equal(pool.view(-1, D).view(torch.int16), want.view(torch.int16))
    # one layer's rows alone
    c.k_pool.copy_(k_before)
    c.v_pool.copy_(v_before)
    for l in range(layers):
        hk.hk_write_kv(d, c.kv, T, sm[l], packed[l, :, 1:Hkv + 1], packed[l, :, Hkv + 1:])
    torch.cuda.synchronize()
    assert torch.equal(pool.view(-1, D).view(torch.int16), want.view(torch.int16))
    # some of the new tokens back, then the rest, then more than the rows hold
    D_all = hk.dims(layers * B, Hkv, Hkv, D)
    ws = hk.workspace(hk.OP_TRIM, D_all, c.width, DEV)
    some = [x // 2 for x in lens]
    for i, drops in enumerate((some, [x - y for x, y in zip(lens, some)], [-3] * B, [3] * B, [10 ** 6] * B)):
        c.t, c.m, c.n, c.free, c.top = CO.trim(c.t, c.m, c.n, np_i(c.free_ids), c.top, drops, Hkv)
        hk.hk_trim_slots(D_all, c.kv, torch.tensor(drops, dtype=I32, device=DEV), c.alloc, ws)
        torch.cuda.synchronize()
        c.check(f"trim {drops}")
        if i == 1 and not holes:
            assert (c.n == before[2]).all() and (c.t == before[0]).all() and (c.m == before[1]).all() and c.top == before[3]
    assert (c.n == 0).all()


def test_reserve_refuses_whole():
    """A pool or a row too small, chunks that are not as promised: flags, nothing moved, no slot given."""
    import paper_2606_28831_amd as hk
    for spare, width, start, T, most, flag in (
            (3, 20, [0, 40, 41], 41, 40, hk.FLAG_NOSPACE), (40, 4, [0, 40, 41], 41, 40, hk.FLAG_NOSPACE),
            (40, 20, [0, 9, 5], 41, 40, hk.FLAG_CHUNK), (40, 20, [0, 9, 42], 41, 40, hk.FLAG_CHUNK),
            (40, 20, [-1, 9, 12], 41, 40, hk.FLAG_CHUNK), (40, 20, [0, 9, 29], 41, 19, hk.FLAG_CHUNK),
            (4, 20, [0, 9, 29], 41, 19, hk.FLAG_CHUNK)):
        c = Cache([20, 30, 40, 50], 64, "bf16", seed=1, width=width, spare=spare)
        ch = hk.Chunks(torch.tensor(start, dtype=I32, device=DEV), T, most)
        _, sm, status = _reserve(c, [0, 0], 2, 1, ch=ch)
        assert status & flag and (flag == hk.FLAG_CHUNK or status == flag), (spare, width, start, status)
        c.check("refused")
        assert (np_i(sm) == -1).all()
        k = torch.ones(T, 2, 64, dtype=torch.bfloat16, device=DEV)
        before = c.k_pool.clone()
        hk.hk_write_kv(hk.dims(2, 2, 2, 64), c.kv, T, sm, k, k)
        torch.cuda.synchronize()
        assert torch.equal(before.view(torch.int16), c.k_pool.view(torch.int16))


def test_reserve_to_the_last_page_and_without_a_map():
    c = Cache([20, 30], 64, "f32", seed=1, width=6, spare=8)
    ok, c.t, c.m, c.n, c.top, _ = CO.reserve(c.t, c.m, c.n, c.free, c.top, [66], 2)
    assert ok and c.top == 0 and c.n.tolist() == [6, 6]
    _, _, status = _reserve(c, [66], 2, 1, slot_map=False)
    assert status == 0
    c.check()


def test_write_skips_slots_outside_the_pool():
    import paper_2606_28831_amd as hk
    c = Cache([16], 64, "f32", seed=1, spare=3)
    sm = torch.tensor([[-1], [4 * 16], [1 << 40], [17], [-(1 << 50)]], dtype=torch.int64, device=DEV)
    k = torch.randn(5, 1, 64, device=DEV)
    want = c.k_pool.view(-1, 64).clone()
    want[17] = k[3, 0]
    hk.hk_write_kv(hk.dims(1, 1, 1, 64), c.kv, 5, sm, k, k)
    torch.cuda.synchronize()
    assert torch.equal(c.k_pool.view(-1, 64).view(I32), want.view(I32))


def test_layers_that_begin_anywhere():
    """Layers of three heads: their tables begin between 16-byte boundaries."""
    import paper_2606_28831_amd as hk
    from paper_2606_28831_amd.pipeline import ChunkDecoder
    L, B, D, lens = 3, 3, 64, [9, 2, 30]
    c = Cache([20, 5, 40, 0, 33, 16, 7, 8, 9], D, "bf16", seed=3, width=6)
    ch = _chunks(lens)
    T = ch.n_tokens
    dec = ChunkDecoder(B, 2, 1, D, c.kv, c.alloc, T, 30, layers=L)
    k, v = (torch.randn(L, T, 1, D, device=DEV).bfloat16() for _ in "kv")
    q = torch.randn(L, T, 2, D, device=DEV).bfloat16()
    sm = torch.zeros(L, T, 1, dtype=torch.int64, device=DEV)
    o, lse = torch.zeros(L, T, 2, D, device=DEV).bfloat16(), torch.zeros(L, T, 2, device=DEV)
    dec.append(ch, k, v, sm)
    for l in range(L):
        dec.attend(ch, q[l], o[l], lse[l], layer=l)
    ok, c.t, c.m, c.n, c.top, _ = CO.reserve(c.t, c.m, c.n, c.free, c.top, lens, 1)
    c.check()
    first = [0, 9, 11]
    whole = (c.t, c.m, c.n)
    for l in range(L):
        c.t, c.m, c.n = (x[l * B:(l + 1) * B] for x in whole)
        _check_attn(c, lens, first, q[l], o[l], lse[l], 1, 2, 0.125, "bf16", D)


# ------------------------------------------------------------------ drafts
def _verify(p, q, tokens, u, lens, V, lead=0, pad=0):
    import paper_2606_28831_amd as hk
    from paper_2606_28831_amd.pipeline import Verifier
    ch, B = _chunks(lens, pad, None, lead), len(lens)
    out = [torch.full((B + 1,), -77, dtype=I32, device=DEV) for _ in range(3)]
    ver = Verifier(B, V, DEV)
    ver.ws.fill_(0x7b)
    ver.verify(ch, tokens, p, u, out[0][:B], out[1][:B], out[2][:B], q=q)
    torch.cuda.synchronize()
    assert all(int(x[B]) == -77 for x in out)
    return [np_i(x[:B]).tolist() for x in out], int(ver.status.item())


def _drafts(rng, T, V, dtype, near=0.6):
    z = rng.normal(size=(T, V)) * 2
    p = np.exp(z - z.max(1, keepdims=True))
    p /= p.sum(1, keepdims=True)
    z = np.roll(z, 1, 0) + rng.normal(size=(T, V)) * near
    q = np.exp(z - z.max(1, keepdims=True))
    q /= q.sum(1, keepdims=True)
    tok = np.array([rng.choice(V, p=x) for x in q])
    put = lambda x: torch.tensor(x, device=DEV).to(DT[dtype])  # noqa: E731
    return put(p), put(q), torch.tensor(tok, dtype=I32, device=DEV), torch.tensor(rng.random(T), dtype=torch.float32, device=DEV)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1, 2, 63, 1000, 4095, 4096, 4097, 20011])
@pytest.mark.parametrize("own_q", [True, False])
def test_verify(V, dtype, own_q):
    rng = np.random.default_rng(V)
    lens = [5, 1, 0, 9, 2, 3] if V < 10000 else [4, 2]
    T = sum(lens) + 3
    p, q, tok, u = _drafts(rng, T, V, dtype)
    if not own_q:
        q, tok = None, torch.where(torch.rand(T, device=DEV) < 0.6, torch.roll(p.float().argmax(1), 1).to(I32), tok)
    got, status = _verify(p, q, tok, u, lens, V, lead=1, pad=2)
    pn, qn, tn, un = np64(p), None if q is None else np64(q), np_i(tok), np_i(u)
    for s, n in enumerate(lens):
        a = 1 + sum(lens[:s])
        want = CO.verify(tn[a:a + n], pn[a:a + n], None if q is None else qn[a:a + n], un[a:a + n])
        assert (got[0][s], got[1][s], got[2][s]) == want, s
    # rows of a wider tensor, no alignment: the same tokens
    wide = torch.full((T, V + 3), float("nan"), dtype=p.dtype, device=DEV)
    wide[:, 1:V + 1] = p
    wq = None
    if q is not None:
        wq = torch.full((T, V + 5), float("nan"), dtype=p.dtype, device=DEV)
        wq[:, 3:V + 3] = q
        wq = wq[:, 3:V + 3]
    assert _verify(wide[:, 1:V + 1], wq, tok, u, lens, V, lead=1, pad=2) == (got, status)
    # a sequence alone: the same token as in the batch
    a, n = 1, lens[0]
    alone, _ = _verify(p[a:a + n], None if q is None else q[a:a + n], tok[a:a + n], u[a:a + n], [n], V)
    assert [x[0] for x in alone] == [x[0] for x in got]


def test_verify_strange_values():
    """Zero rows, NaN, values outside [0, 1], tokens outside the vocabulary, u at and past its ends,
    long drafts."""
    import paper_2606_28831_amd as hk
    V, nan = 5000, float("nan")
    p = torch.zeros(80, V, device=DEV)
    tok = torch.zeros(80, dtype=I32, device=DEV)
    u = torch.full((80,), 0.5, device=DEV)
    assert _verify(p, None, tok, u, [1, 2, 3], V) == ([[0, 0, 0], [-1, -1, -1], [0, 1, 2]], 0)
    p[:, 4999] = 1.0
    tok.fill_(4999)
    got, status = _verify(p, None, tok, u, [80], V)                  # every one of 79 drafts kept
    assert got == [[79], [4999], [0]] and status == 0
    tok[70] = 4998
    assert _verify(p, None, tok, u, [80], V)[0] == [[69], [4999], [10]]
    for bad in (-1, V, 2 ** 31 - 1, -2 ** 31):
        tok[3] = bad
        assert _verify(p, None, tok, u, [6], V)[0] == [[2], [4999], [3]]
    p.zero_()
    p[0, 7], p[0, 8], p[0, 9] = nan, 3.0, -2.0                       # 8 counts 1, the others 0
    got, status = _verify(p, None, tok, u, [1], V)
    assert got == [[0], [8], [0]] and status == hk.FLAG_NAN | hk.FLAG_RANGE
    p.zero_()
    p[0, 10], p[0, 4200] = 0.25, 0.75
    for x, want in ((0.0, 10), (0.2499, 10), (0.25, 4200), (1.0, 4200), (7.0, 4200), (-1.0, 10), (nan, 10), (1 - 2.0 ** -24, 4200)):
        u[0] = x
        assert _verify(p, None, tok, u, [1], V)[0][1] == [want], x


# ------------------------------------------------------------------ all of them together
def test_prompts_drafts_and_compression_chained():
    """DecodeLoop over two layers: prompts in chunks, drafts kept and taken back, single decode steps
    and a compression, against a host model of every row; the draft steps also from a graph."""
    import paper_2606_28831_amd as hk
    from paper_2606_28831_amd.pipeline import DecodeLoop, Verifier
    L, B, Hkv, G, D, W, V, T = 2, 4, 2, 4, 128, 8, 97, 90
    Hq, H, scale = Hkv * G, L * B * Hkv, 1 / math.sqrt(D)
    c = Cache([0] * H, D, "bf16", seed=30, width=20, spare=400)
    loop = DecodeLoop(L, B, Hq, Hkv, D, W, c.kv, c.alloc, 0.9, 32, max_tokens=T, max_len=80)
    ver = Verifier(B, V, DEV)
    bf = torch.bfloat16
    start = torch.zeros(B + 1, dtype=I32, device=DEV)
    ch = hk.Chunks(start, T, 80)
    proj = torch.zeros(L, T, Hq + 2 * Hkv, D, dtype=bf, device=DEV)
    q, k, v = proj[:, :, :Hq], proj[:, :, Hq:Hq + Hkv], proj[:, :, Hq + Hkv:]
    o, lse = torch.zeros(L, T, Hq, D, dtype=bf, device=DEV), torch.zeros(L, T, Hq, device=DEV)
    p, qd = torch.zeros(T, V, device=DEV), torch.zeros(T, V, device=DEV)
    tok, u = torch.zeros(T, dtype=I32, device=DEV), torch.zeros(T, device=DEV)
    acc = [torch.zeros(B, dtype=I32, device=DEV) for _ in range(3)]
    model = [[] for _ in range(H)]                                   # rows (k, v) of every head
    rng = np.random.default_rng(31)

    def fill(lens):
        start.copy_(torch.tensor(np.concatenate([[0], np.cumsum(lens)]), device=DEV).to(I32))
        proj.copy_(torch.randn(proj.shape, device=DEV).to(bf))

    def check(lens, what):
        """o and lse of the chunk against the model, which then holds the chunk's rows."""
        kn, vn, first = np64(k), np64(v), [sum(lens[:s]) for s in range(B)]
        for l in range(L):
            qn, on, ln = np64(q[l]), np64(o[l]), np64(lse[l])
            for s in range(B):
                for x in range(Hkv):
                    rows = model[(l * B + s) * Hkv + x]
                    rows += [(kn[l, t, x], vn[l, t, x]) for t in range(first[s], first[s] + lens[s])]
                    if lens[s] == 0:
                        continue
                    K, Vv = np.array([r[0] for r in rows]), np.array([r[1] for r in rows])
                    a, g = slice(first[s], first[s] + lens[s]), slice(x * G, x * G + G)
                    ro, rl, zabs, absv = CO.chunk_attn_head(qn[a, g], K, Vv, np.ones(len(K), bool), len(K), scale)
                    bo, bl = _bound("bf16", len(K), rl, zabs, absv, ro, D)
                    assert (np.abs(on[a, g] - ro) <= bo).all() and (np.abs(ln[a, g] - rl) <= bl).all(), what

    def rows_are(what):
        t, m, n = np_i(c.page_table), np_i(c.page_mask).astype(np.int64) & 0xFFFF, np_i(c.n_pages)
        kp, vp = np64(c.k_pool), np64(c.v_pool)
        for h in range(H):
            at = [(int(t[h, j // 16]), j % 16) for j in range(16 * int(n[h])) if m[h, j // 16] >> (j % 16) & 1]
            assert len(at) == len(model[h]), (what, h)
            for (pg, sl), (kr, vr) in zip(at, model[h]):
                assert (kp[pg, sl] == kr).all() and (vp[pg, sl] == vr).all(), (what, h)

    for lens in ([40, 0, 17, 9], [35, 33, 1, 2], [1, 80, 5, 0]):    # prompts come in pieces
        fill(lens)
        loop.extend(ch, q, k, v, o, lse)
        torch.cuda.synchronize()
        check(lens, f"prompt {lens}")
    rows_are("prompts")

    def draft():
        loop.extend(ch, q, k, v, o, lse)
        loop.accept(ver, ch, tok, p, u, *acc, q=qd)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        draft()
    for rep, lens in enumerate(([5, 4, 1, 2], [3, 6, 7, 1], [8, 1, 2, 5], [2, 2, 2, 2])):
        fill(lens)
        pn, qn_, tn, un = _drafts(rng, T, V, "f32", near=0.8)
        for a, b in ((p, pn), (qd, qn_), (tok, tn), (u, un)):
            a.copy_(b)
        torch.cuda.synchronize()
        draft() if rep == 0 else graph.replay()
        torch.cuda.synchronize()
        check(lens, f"draft {lens}")
        kept, nxt, drop = (np_i(x).tolist() for x in acc)
        for s in range(B):
            a = slice(sum(lens[:s]), sum(lens[:s + 1]))
            assert (kept[s], nxt[s], drop[s]) == CO.verify(np_i(tok)[a], np64(p)[a], np64(qd)[a], np_i(u)[a])
            for l in range(L):
                for x in range(Hkv):
                    rows = model[(l * B + s) * Hkv + x]
                    del rows[len(rows) - drop[s]:]
        rows_are(f"draft {lens}")
    # single steps of the loop's own decode, and a compression of what the chunks have filled
    for t in range(W):
        fill([0] * B)
        qs, ks, vs = (torch.randn(L * B, n, D, device=DEV).to(bf) for n in (Hq, Hkv, Hkv))
        ls = torch.zeros(L * B, Hq, device=DEV)
        loop.step(qs, ks, vs, ls)
        torch.cuda.synchronize()
        for h in range(H):
            model[h].append((np64(ks)[h // Hkv, h % Hkv], np64(vs)[h // Hkv, h % Hkv]))
            s, x = divmod(h, Hkv)
            K, Vv = np.array([r[0] for r in model[h]]), np.array([r[1] for r in model[h]])
            ro, rl, zabs, _ = CO.chunk_attn_head(np64(qs)[s:s + 1, x * G:x * G + G], K, Vv, np.ones(len(K), bool), len(K), scale)
            assert np.abs(np64(ls)[s, x * G:x * G + G] - rl[0]).max() < 1e-4
    rows_are("steps")
    loop.comp.step(torch.randn(W, L * B, Hq, D, device=DEV).to(bf))
    torch.cuda.synchronize()
    assert int(loop.comp.buf.status.item()) == 0
    t, m, n = np_i(c.page_table), np_i(c.page_mask).astype(np.int64) & 0xFFFF, np_i(c.n_pages)
    kp, vp = np64(c.k_pool), np64(c.v_pool)
    for h in range(H):                                               # what is left, in its order
        at = [(int(t[h, j // 16]), j % 16) for j in range(16 * int(n[h])) if m[h, j // 16] >> (j % 16) & 1]
        left = [(kp[a], vp[a]) for a in at]
        it = iter(model[h])
        assert all(any((kr == a).all() and (vr == b).all() for a, b in it) for kr, vr in left)
        # (rows within the dense tier of 32 tokens, a whole number of pages, stay as they are)
        assert len(left) < len(model[h]) or len(model[h]) <= 32
        model[h] = left
    fill([6, 20, 1, 3])                                              # and drafts over the compressed rows
    loop.extend(ch, q, k, v, o, lse)
    torch.cuda.synchronize()
    check([6, 20, 1, 3], "after the compression")
    assert int(loop.status.item()) == int(ver.status.item()) == 0
