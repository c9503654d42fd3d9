"""Attention over an 8-bit cache where workgroups have much to do: runs of many steps and of several units, ids
and masks fetched again, rows cut into many parts.  Long rows share physical pages, some of whose slots hold codes
and scales of NaN and are masked in every row."""
import numpy as np
import pytest
import torch

import oracle.kv8_oracle as O8
from hk_testlib import np_i
from test_gpu_kv8 import CODE, DEV, GARBAGE, I32, Cache8, _attend, _bytes, _decode

pytestmark = pytest.mark.gpu
GROUPS = {128: 512, 64: 768}                      # workgroups that share a launch's steps
STEP = 128                                        # keys of a step


class Shared8(Cache8):
    """Rows of given lengths over `phys` pages that they share, in an order of each row's own."""

    def __init__(self, lens, D, fmt, width=None, holes=0.1, seed=0, phys=96):
        import paper_2606_28831_amd as hk
        rng = np.random.default_rng(seed)
        H = len(lens)
        self.n = np.array([-(-x // 16) for x in lens], np.int64)
        self.width = int(max(self.n.max(), 2)) if width is None else width
        self.width += self.width % 2
        self.fmt, self.D = fmt, D
        live = np.arange(self.width)[None, :] < self.n[:, None]
        self.t = np.where(live, rng.integers(0, phys, (H, self.width)), -1)
        never = rng.random((phys, 16)) < 0.1
        at = np.arange(self.width * 16).reshape(1, self.width, 16)
        bits = (at < np.array(lens).reshape(-1, 1, 1)) & (rng.random((H, self.width, 16)) >= holes) & ~never[self.t]
        self.m = (bits << np.arange(16)).sum(-1) * live
        for x in ("k", "v"):
            y = rng.standard_normal((phys * 16, D))
            y *= O8.MOST[fmt] / np.abs(y).max(1, keepdims=True)
            if fmt == "i8":
                codes = np.rint(y).astype(np.int8).view(np.uint8)
            else:
                codes = np_i(_bytes(torch.tensor(y).float().to(torch.float8_e4m3fn))).astype(np.uint8)
            scale = ((0.5 + rng.random(phys * 16)) * 3.0 / O8.MOST[fmt]).astype(np.float32)
            codes[never.reshape(-1)] = GARBAGE[fmt]
            scale[never.reshape(-1)] = np.nan
            setattr(self, x + "_codes", codes)
            setattr(self, x + "_sc", scale)
            setattr(self, x + "_pool", torch.tensor(codes, device=DEV).view(CODE[fmt]).view(phys, 16, D))
            setattr(self, x + "_scale", torch.tensor(scale, device=DEV).view(phys, 16))
        self.page_table, self.n_pages = (torch.tensor(x, device=DEV).to(I32) for x in (self.t, self.n))
        self.page_mask = torch.tensor(self.m, device=DEV).to(I32).to(torch.int16)
        self.kv = hk.PagedKV8(self.k_pool, self.v_pool, self.k_scale, self.v_scale, self.page_table, self.page_mask,
                              self.n_pages)

    def steps(self):
        return int(sum(max(1, -(-int(n) // 8)) for n in self.n))


# ------------------------------------------------------------------ single tokens and drafts
@pytest.mark.parametrize("chunk", [False, True])
@pytest.mark.parametrize("fmt,dtype,D", [("i8", "bf16", 128), ("e4m3", "f32", 128), ("e4m3", "bf16", 64), ("i8", "f32", 64)])
def test_a_wave_of_more_than_32_blocks(fmt, dtype, D, chunk):
    """Runs of more than 33 steps of one row: every wave fetches ids and masks a second time."""
    NS, each = 24, 34 * GROUPS[D] // 24 + 8
    c = Shared8([STEP * each - 37 * s for s in range(NS)], D, fmt, seed=D)
    assert c.steps() > 33.5 * GROUPS[D]
    if chunk:
        _attend(c, [1 + s % 4 for s in range(NS)], 1, 2, dtype, heads=[0, 13])
    else:
        _decode(c, NS, 1, 2, dtype, heads=[0, 13])


@pytest.mark.parametrize("fmt,dtype", [("i8", "bf16"), ("e4m3", "f32")])
@pytest.mark.parametrize("D", [128, 64])
def test_long_rows_of_a_launch_that_is_not_planned(fmt, dtype, D):
    """More units than a launch plans: a workgroup takes a whole row of 34 steps and more."""
    H = 4100
    lens = [5 + h % 90 for h in range(H)]
    lens[0], lens[2049], lens[H - 1] = 34 * STEP - 3, 40 * STEP, 33 * STEP + 1
    c = Shared8(lens, D, fmt, seed=2)
    _decode(c, H, 1, 2, dtype, heads=[0, 1, 1000, 2049, H - 1])


@pytest.mark.parametrize("chunk", [False, True])
@pytest.mark.parametrize("holes", [0.0, 0.35])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
@pytest.mark.parametrize("D", [128, 64])
def test_runs_of_several_steps_and_units(D, fmt, dtype, holes, chunk):
    """Rows of every length, two steps a workgroup and more; sharp scores move the reference in most blocks."""
    NS, Hkv = 40, 4
    lens = [(1711 * i) % 3700 for i in range(NS * Hkv)]
    c = Shared8(lens, D, fmt, holes=holes, seed=7)
    assert c.steps() > 2 * GROUPS[D]
    heads = [0, 3, 38, 77, 121, 159]
    for q_scale, G in ((1.0, 4), (40.0, 5)):
        if chunk:
            _attend(c, [1 + s % 6 for s in range(NS)], Hkv, G, dtype, q_scale=q_scale, heads=heads)
        else:
            _decode(c, NS, Hkv, G, dtype, q_scale=q_scale, heads=heads)


@pytest.mark.parametrize("fmt,dtype", [("i8", "f32"), ("e4m3", "bf16")])
def test_runs_of_many_short_units(fmt, dtype):
    """Heads of 128: a workgroup ends and begins several units, of none to three steps."""
    NS, Hkv = 300, 8
    c = Shared8([(37 * i) % 320 for i in range(NS * Hkv)], 128, fmt, width=40, seed=4)
    assert c.steps() > 4 * GROUPS[128]
    _decode(c, NS, Hkv, 2, dtype, heads=list(range(0, NS * Hkv, 397)) + [NS * Hkv - 1])


@pytest.mark.parametrize("fmt,dtype,D,G,lens,rows", [
    # few units: four waves share a row's parts, each more than 64 of them
    ("i8", "bf16", 128, 4, None, [131072]), ("e4m3", "f32", 64, 2, None, [131072, 100]),
    # a wave a row
    ("i8", "f32", 128, 4, None, [50000] + [40] * 16), ("e4m3", "bf16", 64, 3, None, [90000] + [40] * 24),
    # four rows a wave
    ("i8", "bf16", 128, 8, [4] + [1] * 16, [50000] + [40] * 16), ("e4m3", "f32", 128, 5, [6] + [1] * 16, [40000] + [40] * 16),
    # a long chunk's rows
    ("i8", "bf16", 128, 4, [40] + [1] * 16, [50000] + [40] * 16), ("e4m3", "bf16", 64, 4, [45], [131072])])
def test_rows_cut_into_more_than_64_parts_a_wave(fmt, dtype, D, G, lens, rows):
    c = Shared8(rows, D, fmt, seed=6)
    assert c.steps() > 300
    if lens is None:
        _decode(c, len(rows), 1, G, dtype, heads=[0, len(rows) - 1])
    else:
        _attend(c, lens, 1, G, dtype, heads=[0, len(rows) - 1])


# ------------------------------------------------------------------ long bf16 chunks
@pytest.mark.parametrize("long", [{}, dict(max_len=1100, pad=900)], ids=["converting", "converted"])
@pytest.mark.parametrize("holes", [0.0, 0.35])
@pytest.mark.parametrize("fmt,D,keys", [("i8", 128, 9300), ("e4m3", 128, 9300), ("i8", 64, 13600), ("e4m3", 64, 13600)])
def test_a_run_of_more_than_32_tiles(fmt, D, keys, holes, long):
    """Runs of more than eight steps of one unit of a long chunk: ids and masks are fetched a second time."""
    B, Hkv, G, n = 8, 2, 4, 100
    c = Shared8([keys - 11 * i for i in range(B * Hkv)], D, fmt, holes=holes, seed=8)
    assert 4 * c.steps() > 8.5 * GROUPS[D]
    for q_scale in (1.0, 40.0):
        _attend(c, [n] * B, Hkv, G, "bf16", q_scale=q_scale, heads=[1, 14], **long)


@pytest.mark.parametrize("fmt,D", [("i8", 128), ("e4m3", 64)])
def test_long_chunks_that_convert_and_are_not_planned(fmt, D):
    """More units of tiles than are planned, below the rows from which tiles are converted beforehand."""
    B, Hkv, G, n = 4, 8, 8, 500
    c = Shared8([n + 700 + 13 * i for i in range(B * Hkv)], D, fmt, seed=9)
    assert (B * n * G // 128 + B) * Hkv > 1024 and n * G < 4096
    _attend(c, [n] * B, Hkv, G, "bf16", heads=[0, 13, 31])
