"""Scores and selections of an 8-bit cache, in groups of sequences, against those of a cache that holds what its
rows read back as: the same kernels over the same numbers, so the same bits."""
import numpy as np
import pytest
import torch

import oracle.kv8_oracle as O8
from hk_testlib import np64
from test_gpu_kv8 import DEV, DT, I32, Cache8

pytestmark = pytest.mark.gpu
NS, HKV, G, D, W = 5, 2, 2, 64, 4


def _caches(dtype, fmt="i8"):
    """An 8-bit cache and one of its rows in `dtype`, with their allocators."""
    import paper_2606_28831_amd as hk
    c = Cache8([100 + 37 * i for i in range(NS * HKV)], D, fmt, holes=0.1, seed=6, spare=400)
    pools = []
    for codes, s in ((c.k_codes, c.k_sc), (c.v_codes, c.v_sc)):
        x = torch.tensor(O8.values(codes, fmt) * s.astype(np.float64)[:, None]).float().to(DT[dtype])
        pools.append(x.to(DEV).view(-1, 16, D))
    plain = hk.PagedKV(pools[0], pools[1], c.page_table.clone(), c.page_mask.clone(), c.n_pages.clone())
    return c, plain, hk.Allocator(c.free_ids.clone(), c.free_top.clone())


def _queries(dtype, seed=1):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randn(W, NS, HKV * G, D, generator=g, device=DEV).to(DT[dtype])


def _in_groups(x, c, dtype):
    """The compressor's copies made small: groups of 2, 2 and 1 sequences."""
    from paper_2606_28831_amd.pipeline import ScoringCopy
    small = ScoringCopy(NS, HKV * G, HKV, D, W, c.kv, DT[dtype], max_bytes=2 * HKV * c.width * 16 * D * DT[dtype].itemsize)
    assert small.n == 2
    x.copy = small
    if isinstance(x.buf, dict):
        x.buf["ws_score"] = small.ws
    else:
        x.buf.ws_score = small.ws
    return x


def _same(a, b, names):
    torch.cuda.synchronize()
    kvs, als = (a.kv, b.kv), (a.alloc, b.alloc)
    a, b = (m if isinstance(m, dict) else vars(m) for m in (a.buf, b.buf))
    assert int(a["status"]) == 0 and int(b["status"]) == 0
    for name in names:
        assert torch.equal(a[name], b[name]), name
    for what in ("page_mask", "n_pages", "page_table"):
        assert torch.equal(getattr(kvs[0], what), getattr(kvs[1], what)), what
    for what in ("free_ids", "free_top"):
        assert torch.equal(getattr(als[0], what), getattr(als[1], what)), what


@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
@pytest.mark.parametrize("budget", [False, True])
@pytest.mark.parametrize("q_dtype", ["f32", "bf16"])
def test_scores_in_fp32(q_dtype, budget, fmt):
    """K read back in fp32, with fp32 queries or bf16 ones widened."""
    from paper_2606_28831_amd.pipeline import BudgetCompressor, Compressor
    c, plain, al = _caches("f32", fmt)
    q = _queries(q_dtype)
    made = []
    for kv, alloc, more in ((c.kv, c.alloc, dict(score_dtype=torch.float32)), (plain, al, {})):
        if budget:
            x = BudgetCompressor(NS, HKV * G, HKV, D, W, kv, alloc, 0.8, 100, 200, L_dense=32, n_sink=4, rank_by_c=True, **more)
        else:
            x = Compressor(NS, HKV * G, HKV, D, W, kv, alloc, 0.8, L_dense=32, **more)
        made.append(x)
    _in_groups(made[0], c, "f32").step(q)
    made[1].step(q.float())
    _same(made[0], made[1], ("cand_len", "row_lse", "s_attn", "sel_bits", "k") + (("votes", "head_mode") if budget else ()))


@pytest.mark.parametrize("flat", [False, True])
@pytest.mark.parametrize("red", [False, True])
@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_references_and_given_lses_in_groups(dtype, given, red, flat):
    """Redundancy and row LSEs of the caller's, cut for groups of sequences; in another shape too."""
    from paper_2606_28831_amd.pipeline import Compressor
    c, plain, al = _caches(dtype)
    q, H = _queries(dtype), NS * HKV
    more = dict(metric="attn+red", n_ref=6) if red else {}
    x = Compressor(NS, HKV * G, HKV, D, W, c.kv, c.alloc, 0.8, L_dense=32, score_dtype=DT[dtype], **more)
    y = Compressor(NS, HKV * G, HKV, D, W, plain, al, 0.8, L_dense=32, **more)
    rng = np.random.default_rng(5)
    ref = torch.tensor(np.array([rng.choice(c.slots(h), 6, replace=False) for h in range(H)]), dtype=I32, device=DEV) if red else None
    lse = torch.randn(W, NS, HKV * G, device=DEV, generator=torch.Generator(device=DEV).manual_seed(3)) + 4.0 if given else None
    shaped = lambda t, *s: t if t is None or not flat else t.view(*s)  # noqa: E731
    _in_groups(x, c, dtype).step(shaped(q, W, NS, HKV, G, D), ref_slots=shaped(ref, NS, HKV, 6),
                                 row_lse_in=shaped(lse, W * NS, HKV * G))
    y.step(q, ref_slots=ref, row_lse_in=lse)
    _same(x, y, ("cand_len", "s_attn", "sel_bits", "k") + (() if given else ("row_lse",)) +
          (("x_red", "T_red") if red else ()))


def _read_back(loop_kv, dtype):
    """A cache of the rows' values in `dtype`, every valid slot read back (the others 0), with the same tables."""
    import paper_2606_28831_amd as hk
    pages, _, d = loop_kv.k_pool.shape
    pools = []
    for codes, s in ((loop_kv.k_pool, loop_kv.k_scale), (loop_kv.v_pool, loop_kv.v_scale)):
        x = (codes.float() * s[..., None]).nan_to_num(0.0)
        pools.append(x.to(DT[dtype]).contiguous())
    return hk.PagedKV(pools[0], pools[1], loop_kv.page_table.clone(), loop_kv.page_mask.clone(), loop_kv.n_pages.clone())


@pytest.mark.parametrize("score", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
def test_a_loop_selects_by_its_rows_as_they_read_back(fmt, score):
    """The selection of DecodeLoop.compress, from the steps' own LSEs over the codes, is that of a compressor over
    the rows read back, given the same LSEs."""
    import paper_2606_28831_amd as hk
    from paper_2606_28831_amd.pipeline import Compressor, DecodeLoop
    from test_gpu_kv8 import _empty
    L, B = 2, 3
    kv, al = _empty(L * B * HKV, D, fmt, 20, 400)
    loop = DecodeLoop(L, B, HKV * G, HKV, D, W, kv, al, 0.7, 16, score_dtype=DT[score])
    g = torch.Generator(device=DEV).manual_seed(8)
    rnd = lambda *s: torch.randn(*s, generator=g, device=DEV).to(torch.bfloat16)  # noqa: E731
    for i in range(3):
        n = 40 if i == 0 else W
        q, k, v = rnd(n, L * B, HKV * G, D), rnd(n, L * B, HKV, D), rnd(n, L * B, HKV, D)
        lse = torch.empty(n, L * B, HKV * G, device=DEV)
        for t in range(n):
            loop.step(q[t], k[t], v[t], lse[t])
        plain = _read_back(kv, score)
        comp = Compressor(L * B, HKV * G, HKV, D, W, plain, hk.Allocator(al.free_ids.clone(), al.free_top.clone()), 0.7, L_dense=16)
        loop.compress(q[n - W:], lse[n - W:])
        comp.step(q[n - W:].to(DT[score]), row_lse_in=lse[n - W:].contiguous())
        _same(loop.comp, comp, ("cand_len", "s_attn", "sel_bits", "k"))
        assert int(loop.status) == 0 and 0 < int(loop.comp.buf.k.sum()) < int(loop.comp.buf.cand_len.sum())


@pytest.mark.parametrize("score", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
def test_how_far_given_lses_are_from_the_scores(fmt, score):
    """A row's probabilities under hk_decode_attn8's own LSE: with K rounded to bf16 for the scores every score is
    off by 2^-9 sum |q k| / sqrt(D) at most, and so the sum over the row by that factor; with fp32 copies they sum
    to 1 within the score pass's own tolerance (1e-5; bf16 2e-3) and the LSE's."""
    from paper_2606_28831_amd.pipeline import Compressor, Decoder
    c, _, _ = _caches("f32", fmt)
    q = _queries("bf16")[:1]
    o, lse = torch.empty(NS, HKV * G, D, device=DEV), torch.empty(1, NS, HKV * G, device=DEV)
    Decoder(NS, HKV * G, HKV, D, c.kv, c.alloc).attend(q[0], o, lse[0])
    comp = Compressor(NS, HKV * G, HKV, D, 1, c.kv, c.alloc, 0.8, score_dtype=DT[score])
    comp.score(q, row_lse_in=lse)
    total = np.exp(np64(comp.buf.s_attn)).sum(1)                      # mean over the G rows of a head
    for h in range(NS * HKV):
        s, kv = divmod(h, HKV)
        k, _, valid, _ = c.head(h)
        zabs = (np.abs(np64(q[0, s, kv * G:kv * G + G])) @ np.abs(k[valid]).T).max() / np.sqrt(D)
        bound = 3e-5 if score == "f32" else np.expm1(1.01 * 2.0 ** -9 * zabs) + 2e-3
        assert abs(total[h] - 1) <= bound, (h, total[h], bound)
