"""Long bf16 chunks over an 8-bit cache whose rows of V differ in size by more than any fixed exponent of a
softmax's sum could span, against 64 bits."""
import math

import numpy as np
import pytest
import torch

import oracle.chunk_oracle as CO
from hk_testlib import np64
from test_gpu_kv8 import Cache8, DEV, _attend, _bound

pytestmark = pytest.mark.gpu
READY = dict(max_len=2048, pad=2048)              # tiles converted before the attention


def _sized(c, powers, heads=None):
    """V's scales times powers of two, by slot of every row."""
    mul = np.ones(len(c.v_sc))
    for h in range(len(c.n)) if heads is None else heads:
        for j in c.slots(h):
            mul[int(c.t[h, j // 16]) * 16 + j % 16] = 2.0 ** powers(j)
    c.v_sc[:] = (c.v_sc.astype(np.float64) * mul).astype(np.float32)
    c.v_scale.copy_(torch.tensor(c.v_sc, device=DEV).view_as(c.v_scale))
    return c


def _lost(q, k, v, valid, end, lse, D):
    """What keys of a probability below 2^-125 add to o.  The parts of a row that is cut are joined with fp32 weights
    2^(m - the largest m), 0 below 2^-126, where 2^m is more than a part's sum of exponentials and at most twice it:
    the probabilities in a part of weight 0 add up to less than 2^-125."""
    z = np.einsum("igd,jd->igj", q, k) / math.sqrt(D)
    see = valid[None, :] & (np.arange(len(valid))[None, :] < end - len(q) + 1 + np.arange(len(q))[:, None])
    p = np.where(see[:, None], np.exp(np.minimum(z - lse[..., None], 0.0)), 0.0)
    return np.where(p < 2.0 ** -125, p, 0.0) @ np.abs(v)


def _check(c, n, G, q_scale, most={}, dtype="bf16", parts=1):
    q, o, lse = _attend(c, [n], 1, G, dtype, q_scale=q_scale, check=False, **most)
    _check_rows(c, 0, np64(q)[:n], np64(o)[:n], np64(lse)[:n], dtype, parts)


def _check_rows(c, h, q, o, lse, dtype="bf16", parts=1):
    k, v, valid, end = c.head(h)
    ro, rl, zabs, absv = CO.chunk_attn_head(q, k, v, valid, end, 1 / math.sqrt(c.D))
    # a score and its row's exponent are one fp32 number y, |y| <= 1.4427 |z| + 212 in powers of two: off by 2^-24
    # of it, which is 2^-24 (|z| + 147) in the units of _bound, whose (1.01 D + 8) 2^-23 zabs it adds to
    more = 2.0 ** -24 * (zabs + 147)
    bo, bl = _bound(dtype, parts, len(valid), rl, zabs, absv, ro, c.D)
    bo, bl = bo + 2.1 * more[..., None] * absv + _lost(q, k, v, valid, end, rl, c.D), bl + more
    assert np.isfinite(o).all() and np.isfinite(lse).all()
    assert (np.abs(lse - rl) <= bl).all(), f"lse off by {np.max(np.abs(lse - rl) / bl):.3g} bounds"
    off = np.abs(o - ro) / bo
    at = np.unravel_index(np.argmax(off), off.shape)
    assert off[at] <= 1, f"o{at} is {o[at]}, not {ro[at]}, bound {bo[at]:.3g}"


SIZES = {"up": lambda j: -76 + 88 * (j // 80), "down": lambda j: 100 - 88 * (j // 80), "mixed": lambda j: (0, 104, -76)[j % 3],
         "one": lambda j: 104 * (j == 150)}


@pytest.mark.parametrize("most", [{}, READY], ids=["converting", "converted"])
@pytest.mark.parametrize("fmt,D", [("i8", 128), ("e4m3", 128), ("i8", 64), ("e4m3", 64)])
@pytest.mark.parametrize("sizes", sorted(SIZES))
def test_rows_of_any_size_in_one_head(sizes, fmt, D, most):
    """Prompts whose first tokens see small rows alone, or large ones, or both, with flat and sharp scores."""
    c = _sized(Cache8([240], D, fmt, seed=3, width=32), SIZES[sizes])
    for q_scale in (0.0, 1.0, 40.0):
        _check(c, 240, 2, q_scale, most)


@pytest.mark.parametrize("most", [{}, READY], ids=["converting", "converted"])
@pytest.mark.parametrize("D", [128, 64])
def test_rows_of_any_size_in_a_row_that_is_cut(D, most):
    """The parts of a long row each count exponents from their own first keys."""
    c = _sized(Cache8([3000], D, "i8", seed=4, holes=0.2, keep_last=40), lambda j: (100, -76)[(j // 200) % 2] + (j % 5))
    for q_scale in (0.0, 40.0):
        _check(c, 40, 4, q_scale, most)


@pytest.mark.parametrize("most", [{}, READY], ids=["converting", "converted"])
@pytest.mark.parametrize("sizes", sorted(SIZES))
def test_rows_of_any_size_under_scores_past_2_24(sizes, most):
    """One key has all of the weight, and a step of a score is more than a row's exponent moves it."""
    c = _sized(Cache8([240], 128, "i8", seed=3, width=32), SIZES[sizes])
    _, o, lse = _attend(c, [240], 1, 2, "bf16", q_scale=3e8, check=False, **most)
    assert torch.isfinite(lse[:240]).all()
    _, v, _, _ = c.head(0)
    on = np64(o)[:240].reshape(-1, 1, 128)
    # o is rounded to bf16 (2^-8), the key's weight to fp16 (2^-11) where the sum is not
    far = np.abs(on - v[None, :240]).max(2) / np.abs(v[None, :240]).max(2)
    assert (far.min(1) <= 2.0 ** -8 + 2.0 ** -11 + 2.0 ** -18).all()


@pytest.mark.parametrize("dtype,n,parts", [("bf16", 12, 2), ("f32", 12, 3), ("f32", 240, 3)])
@pytest.mark.parametrize("fmt,D", [("i8", 128), ("e4m3", 64)])
@pytest.mark.parametrize("sizes", sorted(SIZES))
def test_rows_of_any_size_in_the_other_forms(sizes, fmt, D, dtype, n, parts):
    """Short chunks and fp32 rows, whose probabilities take V's scales in fp32."""
    c = _sized(Cache8([240], D, fmt, seed=3, width=32), SIZES[sizes])
    for q_scale in (0.0, 1.0, 40.0):
        _check(c, n, 2, q_scale, dtype=dtype, parts=parts)


@pytest.mark.parametrize("most", [{}, dict(max_len=1100)], ids=["converting", "converted"])
@pytest.mark.parametrize("fmt,D", [("i8", 128), ("e4m3", 64)])
def test_rows_of_any_size_in_some_units_of_a_run(fmt, D, most):
    """Workgroups that end one unit and begin another, of heads whose rows differ in size beside others', and beside
    heads with a row of NaN: a second pass over one unit, and none over the next."""
    B, Hkv, G, n = 60, 8, 4, 30
    c = Cache8([n + 105 + 7 * (h % 40) for h in range(B * Hkv)], D, fmt, seed=5)
    _sized(c, lambda j: (100, -76, 12)[j // 50 % 3], heads=range(0, B * Hkv, 3))
    for h in range(1, B * Hkv, 9):                                    # the fourth newest token
        j = n + 105 + 7 * (h % 40) - 4
        c.v_scale.view(-1)[int(c.t[h, j // 16]) * 16 + j % 16] = float("nan")
    for q_scale in (0.0, 8.0):
        q, o, lse = (np64(x) for x in _attend(c, [n] * B, Hkv, G, "bf16", q_scale=q_scale, check=False, **most))
        for h in (0, 3, 4, 5, 240, 243, 245, 477, 479):
            a, g = h // Hkv * n, slice(h % Hkv * G, h % Hkv * G + G)
            _check_rows(c, h, q[a:a + n, g], o[a:a + n, g], lse[a:a + n, g])
        for h in (1, 10, 244):
            a, g = h // Hkv * n, slice(h % Hkv * G, h % Hkv * G + G)
            assert np.isnan(o[a + n - 4:a + n, g]).all() and np.isfinite(o[a:a + n - 4, g]).all()
            assert np.isfinite(lse[a:a + n, g]).all()
