"""The 8-bit cache without a GPU: the oracle's rows by hand, and every refusal of its calls."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import oracle.kv8_oracle as O8

BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32


@pytest.fixture(scope="module")
def hk():
    import paper_2606_28831_amd as m
    m.lib()
    return m


# ------------------------------------------------------------------ the oracle
def test_int8_rows_by_hand():
    codes, s = O8.quantise([127.0, -127.0, 0.5, 1.5, -2.5, 0.0, 63.49, 1e-9], "i8")
    assert s == 1.0 and codes.view(np.int8).tolist() == [127, -127, 0, 2, -2, 0, 63, 0]
    codes, s = O8.quantise([0.0, -0.0], "i8")
    assert codes.tolist() == [0, 0] and s == float(np.float32(2.0 ** -100 / 127))
    codes, s = O8.quantise([1.0, math.inf], "i8")
    assert math.isnan(s) and codes.tolist() == [0, 0]
    assert math.isnan(O8.quantise([math.nan, 1.0], "e4m3")[1])


def test_e4m3_codes_by_hand_and_against_torch():
    for x, b in ((0.0, 0x00), (448.0, 0x7E), (-448.0, 0xFE), (2.0 ** -9, 0x01), (2.0 ** -10, 0x00), (3 * 2.0 ** -10, 0x02),
                 (2.0 ** -6, 0x08), (1.0, 0x38), (1.0625, 0x38), (1.1875, 0x3A), (460.0, 0x7E)):
        assert O8.e4m3_code(x) == b, x
    every = np.arange(256, dtype=np.uint8)
    want = torch.tensor(every).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(O8.values(every, "e4m3"), want)
    x = torch.randn(5000, generator=torch.Generator().manual_seed(1)) * 60
    x = x.clamp(-448, 448)
    got = np.array([O8.e4m3_code(float(v)) for v in x], np.uint8)
    assert (got == x.to(torch.float8_e4m3fn).view(torch.uint8).numpy()).all()


# ------------------------------------------------------------------ the C entry points
P = 1 << 20


def _kv8(hk, dtype=2, max_pages=4, ks=P, vs=P, **more):
    kv = hk.hk_paged_kv(P, P, P, P, P, 64, max_pages, dtype)
    for k, v in more.items():
        setattr(kv, k, v)
    return hk.hk_paged_kv8(kv, ks, vs)


BAD_CACHES = [(dict(dtype=0), 2), (dict(dtype=1), 2), (dict(dtype=4), 2), (dict(ks=None), 1), (dict(vs=None), 1),
              (dict(ks=P + 4), 4), (dict(vs=P + 8), 4), (dict(max_pages=3), 3), (dict(max_pages=0), 1), (dict(k_pool=None), 1),
              (dict(v_pool=None), 1), (dict(v_pool=P + 8), 4), (dict(page_table=P + 2), 4), (dict(page_mask=P + 1), 4),
              (dict(n_pages=None), 1), (dict(num_pages=0), 1)]


@pytest.mark.parametrize("bad,want", BAD_CACHES)
def test_caches_that_are_refused(hk, bad, want):
    L, d, al = hk.lib(), hk.dims(2, 8, 2, 128), hk.hk_allocator(P, P, 64)
    kv, r, c = _kv8(hk, **bad), C.byref, hk.hk_chunks(P, 2, 16, 8)
    big = 1 << 30
    assert L.hk_write_kv8(r(d), r(kv), 1, 8, P, 1, P, 0, 256, P, 0, 256, None) == want
    assert L.hk_read_kv8(r(d), r(kv), 1, 8, P, 1, P, 0, 256, None, 0, 0, None) == want
    assert L.hk_decode_attn8(r(d), 1, P, r(kv), 0.1, P, P, P, big, None) == want
    assert L.hk_chunk_attn8(r(d), r(kv), r(c), 1, P, 1024, 0.1, P, None, P, big, None) == want
    assert L.hk_compact8(r(d), r(kv), P, 0, 0, None, r(al), None, P, big, None) == want


def test_8_bit_caches_are_refused_where_rows_are_read(hk):
    """Entry points that read or write rows of fp32 or bf16."""
    L, d, al, r = hk.lib(), hk.dims(2, 8, 2, 128, 4), hk.hk_allocator(P, P, 64), C.byref
    for dtype in (2, 3):
        kv = hk.hk_paged_kv(P, P, P, P, P, 64, 4, dtype)
        assert L.hk_score(r(d), P, r(kv), 0, 0.1, None, None, P, P, None, 0, None, P, 1 << 30, None) == 2
        assert L.hk_compact(r(d), r(kv), P, 0, 0, r(al), None, P, 1 << 30, None) == 2
        assert L.hk_decode_attn(r(d), P, r(kv), 0.1, P, P, P, 1 << 30, None) == 2
        assert L.hk_append_kv(r(d), r(kv), P, P, r(al), None, P, 1 << 30, None) == 2
        assert L.hk_write_kv(r(d), r(kv), 1, 8, P, P, 0, 256, P, 0, 256, None) == 2
        assert L.hk_chunk_attn(r(d), r(kv), r(hk.hk_chunks(P, 2, 16, 8)), P, 1024, 0.1, P, None, P, 1 << 30, None) == 2
        assert L.hk_score_rows(r(d), P, r(kv), 0, 0.1, P, P, None) == 2
        assert L.hk_compress(r(d), P, r(kv), 0, 0, 0.1, None, 0.9, 1, 0, r(al), None, P, None, P, 1 << 40, None) == 2


def test_row_refusals(hk):
    L, d, kv, r = hk.lib(), hk.dims(1, 8, 2, 128), _kv8(hk), C.byref

    def write(layers=1, T=8, m=P, dt=1, k=P, kr=256, v=P, vr=256, ls=0, d=d):
        return L.hk_write_kv8(r(d), r(kv), layers, T, m, dt, k, ls, kr, v, ls, vr, None)

    def read(layers=1, T=8, m=P, dt=1, k=P, kr=256, v=P, vr=256, ls=0, d=d):
        return L.hk_read_kv8(r(d), r(kv), layers, T, m, dt, k, ls, kr, v, ls, vr, None)
    for f in (write, read):
        assert f(layers=0) == 1 and f(T=0) == 1 and f(m=None) == 1 and f(k=None) == 1
        assert f(kr=255) == 1 and f(vr=128) == 1              # rows shorter than the heads
        assert f(k=P + 8) == 4 and f(kr=260) == 4 and f(layers=2, ls=100) == 4 and f(m=P + 4) == 4
        assert f(dt=2) == 2 and f(dt=7) == 2
        assert f(layers=1 << 20, T=1 << 20, ls=1 << 24) == 3 and f(T=(1 << 24) + 1) == 3
        assert f(d=hk.dims(1, 8, 2, 96)) == 3 and f(d=hk.dims(1, 7, 2, 128)) == 3
    assert write(v=None) == 1
    assert L.hk_write_kv8(r(d), None, 1, 8, P, 1, P, 0, 256, P, 0, 256, None) == 1


def test_attention_refusals(hk):
    L, r = hk.lib(), C.byref
    d, kv, ch = hk.dims(2, 8, 2, 128), _kv8(hk), hk.hk_chunks(P, 2, 16, 8)
    need = L.hk_workspace_size(hk.OP_DECODE8, r(d), 4)
    assert need > 0 and L.hk_workspace_size(hk.OP_DECODE8, r(hk.dims(2, 130, 2, 128)), 4) == 0

    def decode(d=d, dt=1, q=P, scale=0.1, o=P, lse=P, ws=P, n=need):
        return L.hk_decode_attn8(r(d), dt, q, r(kv), scale, o, lse, ws, n, None)
    assert decode(d=hk.dims(2, 8, 2, 96)) == 3 and decode(d=hk.dims(2, 9, 2, 128)) == 3
    assert decode(d=hk.dims(2, 130, 2, 128), n=1 << 30) == 3
    assert decode(dt=2) == 2 and decode(q=None) == 1 and decode(o=None) == 1
    for bad in (0.0, -1.0, math.inf, math.nan):
        assert decode(scale=bad) == 1
    assert decode(q=P + 8) == 4 and decode(o=P + 4) == 4 and decode(lse=P + 2) == 4
    assert decode(n=need - 1) == 5 and decode(ws=None) == 5 and decode(ws=P + 16) == 4

    cneed = L.hk_chunk_attn8_workspace_size(r(d), r(ch), 4)
    assert cneed > 0

    def attn(d=d, c=ch, dt=1, q=P, row=1024, scale=0.1, o=P, lse=None, ws=P, n=cneed):
        return L.hk_chunk_attn8(r(d), r(kv), r(c), dt, q, row, scale, o, lse, ws, n, None)
    assert attn(d=hk.dims(2, 8, 2, 96)) == 3 and attn(d=hk.dims(2, 130, 2, 128), row=130 * 128) == 3
    assert attn(c=hk.hk_chunks(P, 1, 16, 8)) == 3 and attn(c=hk.hk_chunks(None, 2, 16, 8)) == 1
    assert attn(c=hk.hk_chunks(P, 2, 0, 8)) == 1 and attn(c=hk.hk_chunks(P, 2, 16, 0)) == 1
    assert attn(dt=3) == 2 and attn(q=None) == 1 and attn(o=None) == 1 and attn(row=1023) == 1
    assert attn(q=P + 2) == 4 and attn(row=1028) == 4 and attn(o=P + 8) == 4 and attn(lse=P + 1) == 4
    assert attn(c=hk.hk_chunks(P + 2, 2, 16, 8)) == 4
    assert attn(scale=0.0) == 1 and attn(scale=math.nan) == 1
    assert attn(n=cneed - 1) == 5 and attn(ws=None) == 5 and attn(ws=P + 16) == 4
    # more workgroups than a launch takes
    big = hk.dims(1, 64 * 1000, 1000, 128)
    for tokens, want in ((1 << 24, 3), (1 << 19, 3), (1 << 12, 5)):
        c = hk.hk_chunks(P, 1, tokens, 8)
        assert L.hk_chunk_attn8(r(big), r(kv), r(c), 1, P, 64 * 1000 * 128, 0.1, P, None, None if want == 5 else P,
                                0 if want == 5 else 1 << 62, None) == want


@pytest.mark.parametrize("D", [64, 128])
def test_a_workspace_for_more_tokens_serves_fewer(hk, D):
    L, d = hk.lib(), hk.dims(2, 8, 2, D)
    size = lambda t, m, p=2048: L.hk_chunk_attn8_workspace_size(C.byref(d), C.byref(hk.hk_chunks(P, 2, t, m)), p)  # noqa: E731
    sizes = [size(t, t) for t in (1, 2, 4, 5, 7, 8, 9, 31, 64, 300, 1000, 5000, 40000, 1 << 20)]
    assert sizes == sorted(sizes) and sizes[0] > 0 and size(5000, 1) <= size(5000, 5000)
    assert [size(100, 100, p) for p in (2, 8, 10, 100, 60000)] == sorted(size(100, 100, p) for p in (2, 8, 10, 100, 60000))
    assert L.hk_chunk_attn8_workspace_size(C.byref(d), None, 4) == 0 and size(0, 1) == 0 and size(1, 1, 0) == 0


def test_rewrite_refusals(hk):
    L, d, r = hk.lib(), hk.dims(2, 8, 2, 128), C.byref
    need = L.hk_workspace_size(hk.OP_COMPACT, r(d), 4)

    def compact(kv=_kv8(hk), sel=P, ld=0, ls=0, al=hk.hk_allocator(P, P, 64), ws=P, n=need):
        return L.hk_compact8(r(d), r(kv), sel, ld, ls, None, r(al), None, ws, n, None)
    assert compact(sel=None) == 1 and compact(ld=-1) == 1 and compact(ls=-1) == 1
    assert compact(al=hk.hk_allocator(P, P, 63)) == 1 and compact(al=hk.hk_allocator(None, P, 64)) == 1
    assert compact(n=need - 1) == 5 and compact(ws=None) == 5 and compact(ws=P + 8) == 4
    assert compact(kv=_kv8(hk, max_pages=30000), n=1 << 30) == 3
    assert compact(kv=_kv8(hk, page_mask=P + 2)) == 4         # tables are read 16 bytes at a time here


# ------------------------------------------------------------------ the wrappers
def _cache(hk, fmt=torch.int8, heads=4, pages=8, D=64, **more):
    z = lambda *s, dt=torch.uint8: torch.zeros(*s, dtype=dt)  # noqa: E731
    t = dict(k=z(pages, 16, D).view(fmt), v=z(pages, 16, D).view(fmt), ks=z(pages, 16, dt=F32), vs=z(pages, 16, dt=F32),
             table=z(heads, 4, dt=I32), mask=z(heads, 4, dt=torch.int16), n=z(heads, dt=I32))
    t.update(more)
    return hk.PagedKV8(t["k"], t["v"], t["ks"], t["vs"], t["table"], t["mask"], t["n"])


@pytest.mark.parametrize("bad,words", [
    (dict(ks=torch.zeros(7, 16)), "scales must"), (dict(vs=torch.zeros(8, 16, dtype=BF)), "scales must"),
    (dict(ks=torch.zeros(16, 8).t()), "scales must"), (dict(v=torch.zeros(8, 16, 64, dtype=torch.uint8).view(torch.float8_e4m3fn)), "one type"),
    (dict(table=torch.zeros(3, 4, dtype=I32)), "fewer rows"), (dict(mask=torch.zeros(4, 2, dtype=torch.int16)), "tables must"),
    (dict(n=torch.zeros(4, dtype=torch.int64)), "tables must")])
def test_wrappers_refuse_tensors_that_do_not_fit(hk, bad, words):
    d, ch = hk.dims(2, 4, 2, 64), hk.Chunks(torch.zeros(3, dtype=I32), 8, 8)
    ws = torch.zeros(1 << 16, dtype=torch.uint8)
    kv, al = _cache(hk, **bad), hk.Allocator(torch.zeros(8, dtype=I32), torch.zeros(1, dtype=I32))
    q = torch.zeros(8, 4, 64, dtype=BF)
    for call in (lambda: hk.hk_decode_attn8(d, q[:2], kv, 0.1, torch.zeros(2, 4, 64), None, ws),
                 lambda: hk.hk_chunk_attn8(d, kv, ch, q, 0.1, q.clone(), ws),
                 lambda: hk.hk_compact8(d, kv, torch.zeros(4, 2, dtype=I32), 0, 0, al, None, ws)):
        with pytest.raises(hk.HardKVError, match=words):
            call()


def test_wrappers_refuse_short_and_strange_arguments(hk):
    T, Hq, Hkv, D = 8, 4, 2, 64
    d, ch = hk.dims(2, Hq, Hkv, D), hk.Chunks(torch.zeros(3, dtype=I32), T, T)
    kv, ws = _cache(hk), torch.zeros(1 << 16, dtype=torch.uint8)
    al = hk.Allocator(torch.zeros(8, dtype=I32), torch.zeros(1, dtype=I32))
    err = hk.HardKVError
    with pytest.raises(err):
        hk.PagedKV8(torch.zeros(8, 16, D), torch.zeros(8, 16, D), torch.zeros(8, 16), torch.zeros(8, 16),
                    torch.zeros(4, 4, dtype=I32), torch.zeros(4, 4, dtype=torch.int16), torch.zeros(4, dtype=I32))
    bf16 = hk.PagedKV(torch.zeros(8, 16, D, dtype=BF), torch.zeros(8, 16, D, dtype=BF), torch.zeros(4, 4, dtype=I32),
                      torch.zeros(4, 4, dtype=torch.int16), torch.zeros(4, dtype=I32))
    q, o = torch.zeros(T, Hq, D, dtype=BF), torch.zeros(T, Hq, D, dtype=BF)
    with pytest.raises(err, match="8-bit cache"):
        hk.hk_chunk_attn8(d, bf16, ch, q, 0.1, o, ws)
    with pytest.raises(err, match="8-bit cache"):
        hk.hk_write_kv8(d, bf16, T, torch.zeros(T * Hkv, dtype=torch.int64), q[:, :2], q[:, :2])
    for bad in (q[:7], q.half(), torch.zeros(T, D, Hq, dtype=BF).transpose(1, 2), torch.zeros(T, Hq, 2 * D, dtype=BF)[:, :, :D]):
        with pytest.raises(err):
            hk.hk_chunk_attn8(d, kv, ch, bad, 0.1, o, ws)
    for bad_o, lse in ((o[:5], None), (o.float(), None), (o, torch.zeros(T * Hq - 1)), (o, torch.zeros(T, Hq, dtype=BF))):
        with pytest.raises(err):
            hk.hk_chunk_attn8(d, kv, ch, q, 0.1, bad_o, ws, lse=lse)
    q1, o1 = torch.zeros(2, Hq, D, dtype=BF), torch.zeros(2, Hq, D)
    for a in (dict(q=q1[:1]), dict(q=q1.half()), dict(o=o1.to(BF)), dict(o=o1[:1]), dict(lse=torch.zeros(7))):
        a = dict(dict(q=q1, o=o1, lse=None), **a)
        with pytest.raises(err):
            hk.hk_decode_attn8(d, a["q"], kv, 0.1, a["o"], a["lse"], ws)
    k, m = torch.zeros(T, Hkv, D, dtype=BF), torch.zeros(T * Hkv, dtype=torch.int64)
    for a in (dict(k=k[:7]), dict(k=k.float()), dict(v=k[:, :1]), dict(m=m[1:]), dict(m=m.int()), dict(k=k.half(), v=k.half()),
              dict(k=k[None].expand(2, -1, -1, -1), v=k)):
        a = dict(dict(k=k, v=k, m=m), **a)
        for f in (hk.hk_write_kv8, hk.hk_read_kv8):
            with pytest.raises(err):
                f(d, kv, T, a["m"], a["k"], a["v"])
    with pytest.raises(err):
        hk.hk_write_kv8(d, kv, T, m, k, None)
    for sel, mode in ((torch.zeros(4, 1, dtype=I32), None), (torch.zeros(4, 2, dtype=torch.int64), None),
                      (torch.zeros(4, 2, dtype=I32), torch.zeros(3, dtype=I32))):
        with pytest.raises(err):
            hk.hk_compact8(d, kv, sel, 0, 0, al, None, ws, head_mode=mode)
    with pytest.raises(err, match="outside the GPU"):
        hk.hk_chunk_attn8(d, kv, ch, q, 0.1, o, ws)


def test_views_of_an_8_bit_cache_keep_its_kind(hk):
    kv = _cache(hk, heads=6)
    v = kv.rows(2, 3)
    assert isinstance(v, hk.PagedKV8) and v.sizes() == (3, 64, -1) and v.desc8.k_scale == kv.k_scale.data_ptr()
    assert v.desc.page_table == kv.page_table.data_ptr() + 2 * 16 and v.desc.dtype == 2
    assert _cache(hk, fmt=torch.float8_e4m3fn).desc.dtype == 3
