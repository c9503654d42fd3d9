"""What keeps the calls with several new tokens per sequence from touching what is not theirs, on
the CPU: everything here ends before a launch."""
import ctypes as C

import pytest
import torch


@pytest.fixture(scope="module")
def hk():
    import paper_2606_28831_amd as hk
    return hk


I32 = torch.int32


def test_the_word_of_granted_chunks(hk):
    """Chunks carry their decoder's word to later calls; anything but an int32 word of the starts'
    device is refused."""
    start, word = torch.zeros(3, dtype=I32), torch.ones(1, dtype=I32)
    ch = hk.Chunks(start, 4, 4)
    assert ch.granted is None and ch.desc.granted is None
    ch = hk.Chunks(start, 4, 4, granted=word)
    assert ch.desc.granted == word.data_ptr() and C.sizeof(ch.desc) == 32
    ch.granted_by(None)
    assert ch.desc.granted is None
    for bad in (torch.ones(1), torch.ones(1, dtype=torch.int64), torch.zeros(0, dtype=I32), torch.empty(1, dtype=I32, device="meta")):
        with pytest.raises(hk.HardKVError):
            ch.granted_by(bad)
    assert ch.granted is None


def _set(hk, D=64, heads=4, **other):
    """A cache of 4 heads, an allocator and the tensors of every call, with some of them replaced."""
    bf = torch.bfloat16
    t = dict(k=torch.zeros(8, 16, D, dtype=bf), v=torch.zeros(8, 16, D, dtype=bf), table=torch.zeros(heads, 4, dtype=I32),
             mask=torch.zeros(heads, 4, dtype=torch.int16), n=torch.zeros(heads, dtype=I32),
             ids=torch.zeros(8, dtype=I32), top=torch.zeros(1, dtype=I32))
    t.update(other)
    return hk.PagedKV(t["k"], t["v"], t["table"], t["mask"], t["n"]), hk.Allocator(t["ids"], t["top"])


def _calls(hk, D):
    """Every call that works on a cache, for 2 sequences of 2 KV heads of size D."""
    T, bf = 8, torch.bfloat16
    d, ch = hk.dims(2, 4, 2, D), hk.Chunks(torch.zeros(3, dtype=I32), T, T)
    ws, sm = torch.zeros(1 << 16, dtype=torch.uint8), torch.zeros(T * 2, dtype=torch.int64)
    q, k = torch.zeros(T, 4, D, dtype=bf), torch.zeros(T, 2, D, dtype=bf)
    return dict(attn=lambda kv, al: hk.hk_chunk_attn(d, kv, ch, q, 0.1, q.clone(), ws),
                write=lambda kv, al: hk.hk_write_kv(d, kv, T, sm, k, k),
                reserve=lambda kv, al: hk.hk_reserve_slots(d, kv, ch, al, ws, slot_map=sm),
                trim=lambda kv, al: hk.hk_trim_slots(d, kv, torch.zeros(2, dtype=I32), al, ws))


def test_caches_of_another_head_size_are_refused(hk):
    """Rows of 128 over a pool of 64 would be read and written past the pool's end."""
    for have, D in ((64, 128), (128, 64)):
        for name, call in _calls(hk, D).items():
            with pytest.raises(hk.HardKVError, match="head size"):
                call(*_set(hk, D=have))


@pytest.mark.parametrize("other,what", [
    (dict(mask=torch.zeros(3, 4, dtype=torch.int16)), "fewer rows"),
    (dict(n=torch.zeros(3, dtype=I32)), "fewer rows"),
    (dict(table=torch.zeros(3, 4, dtype=I32)), "fewer rows"),
    (dict(mask=torch.zeros(4, 2, dtype=torch.int16)), "tables must be"),
    (dict(mask=torch.zeros(4, 4, dtype=I32)), "tables must be"),
    (dict(table=torch.zeros(4, 4, dtype=torch.int64)), "tables must be"),
    (dict(n=torch.zeros(4, dtype=torch.int64)), "tables must be"),
    (dict(table=torch.zeros(4, 8, dtype=I32)[:, ::2]), "contiguous"),
    (dict(v=torch.zeros(7, 16, 64, dtype=torch.bfloat16)), "pools must be"),
    (dict(v=torch.zeros(8, 16, 64)), "pools must be"),
    (dict(k=torch.zeros(8, 64, 16, dtype=torch.bfloat16).transpose(1, 2)), "contiguous")])
def test_caches_whose_tensors_do_not_agree_are_refused(hk, other, what):
    for name, call in _calls(hk, 64).items():
        if name == "write" and what == "fewer rows":
            continue                                     # (only the pools are used)
        with pytest.raises(hk.HardKVError, match=what):
            call(*_set(hk, **other))


@pytest.mark.parametrize("other", [dict(ids=torch.zeros(8, dtype=torch.int64)), dict(top=torch.zeros(1, dtype=torch.int64)),
                                   dict(top=torch.zeros(0, dtype=I32)), dict(ids=torch.zeros(16, dtype=I32)[::2])])
def test_allocators_that_are_not_what_they_say_are_refused(hk, other):
    calls = _calls(hk, 64)
    for name in ("reserve", "trim"):
        with pytest.raises(hk.HardKVError, match="allocator"):
            calls[name](*_set(hk, **other))


def test_status_words_and_tensors_outside_the_gpu_are_refused(hk):
    kv, al = _set(hk)
    d, ch = hk.dims(2, 4, 2, 64), hk.Chunks(torch.zeros(3, dtype=I32), 8, 8)
    ws, out = torch.zeros(1 << 16, dtype=torch.uint8), torch.zeros(2, dtype=I32)
    p, u, tok = torch.zeros(8, 10), torch.zeros(8), torch.zeros(8, dtype=I32)
    for bad in (torch.zeros(1, dtype=torch.uint8), torch.zeros(0, dtype=I32), torch.zeros(1)):
        with pytest.raises(hk.HardKVError, match="status"):
            hk.hk_reserve_slots(d, kv, ch, al, ws, status=bad)
        with pytest.raises(hk.HardKVError, match="status"):
            hk.hk_verify_draft(ch, 10, tok, p, u, out, out, out, ws, status=bad)
    for call in _calls(hk, 64).values():
        with pytest.raises(hk.HardKVError, match="outside the GPU"):
            call(kv, al)
    with pytest.raises(hk.HardKVError, match="outside the GPU"):
        hk.hk_verify_draft(ch, 10, tok, p, u, out, out, out, ws)


def test_chunk_attn_refuses_launches_that_the_hardware_does_not_take(hk):
    """Tiles of 128 queries x KV heads x 256 threads pass 2^32 from 33554 tokens of 64000 query heads on,
    also with a workspace and with fewer than 2^34 queries."""
    L = hk.lib()
    P = 1 << 20
    d, kv = hk.dims(1, 64 * 1000, 1000, 128), hk.hk_paged_kv(P, P, P, P, P, 64, 4, 1)
    for tokens in (33554, 1 << 17, 1 << 18):
        c = hk.hk_chunks(P, 1, tokens, 8)
        need = L.hk_chunk_attn_workspace_size(C.byref(d), C.byref(c), 4)
        args = (C.byref(d), C.byref(kv), C.byref(c), P, 64 * 1000 * 128, 0.1, P, None)
        assert L.hk_chunk_attn(*args, P, need, None) == 3
        assert L.hk_chunk_attn(*args, P, need - 1, None) == 5
