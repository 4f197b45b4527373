"""Prompts over a cache in which values are not finite that only some of a tile's rows see: these rows are taken again, right and
soon."""
import math

import numpy as np
import pytest
import torch

from paged_util import Problem, attention_tolerance
from paper_2504_08378_b200 import afx
from test_gpu_paged_attn import attend
from test_gpu_paged_poison import median_us
from test_gpu_paged_prompts import busy

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cache,dim,heads,kv,page", [("bf16", 128, 8, 2, 16), ("f16", 64, 4, 4, 24), ("f16", 128, 6, 2, 64), ("bf16", 64, 16, 2, 1)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (70, 0), (70, 5), (300, 40)])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_rows_that_see_them_and_rows_that_do_not(cache, dim, heads, kv, page, window, sinks, value):
    n, new = 420, 260
    p = Problem(*busy([n, 33], [new, 33]), heads, kv, dim, page, cache, seed=window)
    b = p.lens.index(n)
    hurt = [1, 3, 20, 150, 171, 300, 415, 419]
    rows = p.rows_of(p.both, b, 1).clone()
    for x, j in enumerate(hurt):
        rows[j, :, (7 * x) % dim] = value
    rows[419, :, 9] = math.nan
    rows[300, 0, :] = value
    p.cells(b, 1)[:] = rows
    q = p.randn(p.rows, heads, dim, dtype=cache)
    out, lse = attend(p, q, p.upload(afx), cache, cache, window, sinks)
    with np.errstate(all="ignore"):
        want, want_lse, mass, norm = p.attend(q, window, sinks)
    o, fin = out.double().numpy(), np.isfinite(want)
    assert fin.any() and not fin.all()
    tol = attention_tolerance(np.where(fin, want, 0), np.where(fin, mass, 0), norm, dim, cache, cache)
    with np.errstate(invalid="ignore"):
        assert (np.abs(o - want)[fin] <= tol[fin]).all()
    assert not np.isfinite(o[~fin]).any()
    some = np.isfinite(want_lse)
    ltol = 2 * ((dim + 4) * 2.0 ** -23 * norm + 2.0 ** -20) + 2.0 ** -22 * np.abs(want_lse)
    assert (np.abs(lse.double().numpy() - want_lse)[some] <= ltol[some]).all()


def test_bad_pages_behind_rows_that_are_taken_again():
    p = Problem(*busy([400], [200]), 4, 2, 64, 16, "f16", seed=1)
    b = p.lens.index(400)
    rows = p.rows_of(p.both, b, 1).clone()
    rows[399, :, 3] = math.inf
    p.cells(b, 1)[:] = rows
    q = p.randn(p.rows, 4, 64, dtype="f16")
    kvd = p.upload(afx)
    p.d_table[b, 2], p.d_table[b, 20] = -1, p.n_pages
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, _ = attend(p, q, kvd, "f16", "f16", status=status)
    assert status.item() == 1
    K, V = (p.rows_of(p.both, b, c).double() for c in (0, 1))
    for i in (0, 100, 150, 198):
        keep = torch.tensor([j for j in range(200 + i + 1) if j // 16 not in (2, 20)])
        for h in range(4):
            w = torch.softmax(K[keep, h // 2] @ q[i, h].double() / 8, 0)
            want, mass = w @ V[keep, h // 2], w @ V[keep, h // 2].abs()
            assert ((out[i, h].double() - want).abs() <= 2.0 ** -11 * want.abs() + 2.0 ** -25 + 2.0 ** -9 * mass).all()


@pytest.mark.parametrize("dim", [64, 128])
def test_a_poisoned_prompt_does_not_hold_up_the_others_for_long(dim):
    """A row at a time, its rows took 90 ms over 9000 positions (0.3 us a position)."""
    lens, news = [9000, 700, 900, 800], [512, 700, 900, 800]
    p = Problem(lens, news, 32, 8, dim, 64, "bf16")
    q = p.randn(p.rows, 32, dim, dtype="bf16").cuda()
    clean = median_us(p, q, 32, dim, p.upload(afx))
    rows = p.rows_of(p.both, 0, 1).clone()
    rows[-1, :, 5] = math.inf
    p.cells(0, 1)[:] = rows
    hurt = median_us(p, q, 32, dim, p.upload(afx))
    print(f"clean {clean:.0f} us, poisoned {hurt:.0f}")
    assert hurt <= 9000


def test_a_prompt_over_a_cache_of_nan_is_soon_done():
    """Rows whose every sum is NaN are not taken again to their end."""
    p = Problem([6000], [3000], 32, 8, 64, 64, "bf16")
    q = p.randn(p.rows, 32, 64, dtype="bf16").cuda()
    clean = median_us(p, q, 32, 64, p.upload(afx))
    p.both[:] = math.nan
    hurt = median_us(p, q, 32, 64, p.upload(afx))
    print(f"clean {clean:.0f} us, NaN {hurt:.0f}")
    assert hurt <= 4 * clean
