"""What the compressors refuse of the window queries of an 8-bit cache, without a GPU."""
import pytest
import torch

BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32
NS, HKV, G, D, W = 5, 2, 2, 64, 4


@pytest.fixture(scope="module")
def hk():
    import paper_2606_28831_amd as m
    m.lib()
    return m


def _cache(hk, heads=NS * HKV, pages=20, width=4):
    z = lambda *s, dt=torch.uint8: torch.zeros(*s, dtype=dt)  # noqa: E731
    kv = hk.PagedKV8(z(pages, 16, D).view(torch.int8), z(pages, 16, D).view(torch.int8), z(pages, 16, dt=F32),
                     z(pages, 16, dt=F32), z(heads, width, dt=I32), z(heads, width, dt=torch.int16), z(heads, dt=I32))
    return kv, hk.Allocator(z(pages, dt=I32), z(1, dt=I32))


def _compressor(hk, **more):
    from paper_2606_28831_amd.pipeline import Compressor
    kv, al = _cache(hk)
    return Compressor(NS, HKV * G, HKV, D, W, kv, al, 0.8, **more)


def _q(dtype, *shape):
    return torch.zeros(*(shape or (W, NS, HKV * G, D)), dtype=dtype)


def test_queries_are_not_rounded_without_a_word(hk):
    from paper_2606_28831_amd.pipeline import BudgetCompressor, DecodeLoop
    comp = _compressor(hk)
    for dtype in (F32, torch.float16, torch.float64):
        for call in (comp.score, comp.step):
            with pytest.raises(hk.HardKVError, match="score_dtype"):
                call(_q(dtype))
    kv, al = _cache(hk)
    budget = BudgetCompressor(NS, HKV * G, HKV, D, W, kv, al, 0.8, 100, 200)
    for call in (budget.select, budget.step):
        with pytest.raises(hk.HardKVError, match="score_dtype"):
            call(_q(F32))
    loop = DecodeLoop(1, NS, HKV * G, HKV, D, W, kv, al, 0.8, 16)
    with pytest.raises(hk.HardKVError, match="score_dtype"):
        loop.compress(_q(F32), torch.zeros(W, NS, HKV * G))
    with pytest.raises(hk.HardKVError, match="score_dtype"):     # (before a step of the segment is taken)
        loop.segment(_q(F32), _q(F32, W, NS, HKV, D), _q(F32, W, NS, HKV, D), torch.zeros(W, NS, HKV * G))
    with pytest.raises(hk.HardKVError, match="score_dtype"):
        _compressor(hk, score_dtype=F32).score(_q(torch.float64))


def test_queries_of_the_type_or_widened_go_on(hk):
    """(to the call that wants a GPU)"""
    for dtype, to in ((BF, BF), (F32, F32), (BF, F32)):
        with pytest.raises(hk.HardKVError, match="outside the GPU"):
            _compressor(hk, score_dtype=to).score(_q(dtype))


def test_arguments_are_cut_by_sequence_only_where_they_fit(hk):
    """References, LSEs and queries go to the score pass a few sequences at a time: what does not hold one entry for
    each head or row would be read past its end, or spread over rows it is not of."""
    comp, q = _compressor(hk, metric="attn+red", n_ref=3), _q(BF)
    H, Hq = NS * HKV, HKV * G
    ref = torch.zeros(H, 3, dtype=I32)
    for bad in (ref[:7], ref[:, :2].contiguous(), ref.long(), torch.zeros(H, 4, dtype=I32), torch.zeros(H * 3 - 1, dtype=I32)):
        with pytest.raises(hk.HardKVError, match="ref_slots"):
            comp.score(q, ref_slots=bad)
    for bad in (torch.zeros(W, 1, Hq), torch.zeros(1, NS, Hq), torch.zeros(W, NS), torch.zeros(W, NS, Hq, dtype=BF),
                torch.zeros(W, Hq, NS).transpose(1, 2)[:, :, :1], torch.zeros(NS, W, Hq).transpose(0, 1)[:2]):
        with pytest.raises(hk.HardKVError, match="row_lse_in"):
            comp.score(q, row_lse_in=bad)
    for bad in (_q(BF, 1, NS, Hq, D), _q(BF, W, 1, Hq, D), _q(BF, W, NS, Hq, 1), _q(BF, W, NS, Hq), _q(BF, W, NS, Hq, D + 64)):
        with pytest.raises(hk.HardKVError, match="window queries"):
            comp.score(bad)


def test_arguments_of_another_shape_with_as_many_entries_go_on(hk):
    """(to the call that wants a GPU: contiguous ones are one buffer in any shape)"""
    comp, Hq = _compressor(hk, metric="attn+red", n_ref=3), HKV * G
    for q, ref, lse in ((_q(BF, W, NS, HKV, G, D), torch.zeros(NS, HKV, 3, dtype=I32), torch.zeros(W, NS * Hq)),
                        (_q(BF, W * NS * Hq * D), torch.zeros(NS * HKV * 3, dtype=I32), torch.zeros(W * NS * Hq)),
                        (_q(BF, NS, W, Hq, D).transpose(0, 1), None, torch.zeros(NS, W, Hq).transpose(0, 1))):
        with pytest.raises(hk.HardKVError, match="outside the GPU"):
            comp.score(q, ref_slots=ref, row_lse_in=lse)


def test_caches_of_fewer_rows_than_heads_are_refused(hk):
    """(a row of tables alone would be spread over all heads)"""
    from paper_2606_28831_amd.pipeline import BudgetCompressor, Compressor
    for heads in (1, NS * HKV - 1):
        kv, al = _cache(hk, heads=heads)
        with pytest.raises(hk.HardKVError, match="fewer rows"):
            Compressor(NS, HKV * G, HKV, D, W, kv, al, 0.8).score(_q(BF))
        with pytest.raises(hk.HardKVError, match="fewer rows"):
            BudgetCompressor(NS, HKV * G, HKV, D, W, kv, al, 0.8, 100, 200).select(_q(BF))
    kv, al = _cache(hk)
    with pytest.raises(hk.HardKVError, match="head size"):
        Compressor(NS, HKV * G, HKV, 128, W, kv, al, 0.8).score(_q(BF, W, NS, HKV * G, 128))
