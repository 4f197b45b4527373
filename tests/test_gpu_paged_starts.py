"""Starts that decrease or leave the rows are clamped to [largest start before, rows], by every kernel of the paged cache alike:
the same bits as with the clamped starts, and a report."""
import numpy as np
import pytest
import torch

from paged_util import Problem
from paper_2504_08378_b200 import afx
from test_gpu_paged_attn import attend

pytestmark = pytest.mark.gpu


def clamped(starts, rows):
    return np.clip(np.maximum.accumulate(starts), 0, rows)


def problem(starts, rows, dim=64, heads=4, kv=2, extra=5):
    news = np.diff(clamped(starts, rows))
    p = Problem([int(n) + 1 + (i * 7) % extra for i, n in enumerate(news)], [int(n) for n in news], heads, kv, dim, 16, "f16")
    p.rows = rows
    return p


def both(p, starts, call):
    """What `call` leaves with the starts and with the clamped ones, and the first one's report."""
    kvd = p.upload(afx)
    assert kvd.n_tokens == p.rows
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    p.d_start.copy_(torch.from_numpy(clamped(starts, p.rows).astype(np.int32)))
    want = call(kvd, status)
    assert status.item() == 0
    p.d_start.copy_(torch.from_numpy(np.asarray(starts, np.int32)))
    return call(kvd, status), want, status.item()


def attention(p):
    q = p.randn(p.rows, p.heads, p.dim, dtype="f16")
    return lambda kvd, status: attend(p, q, kvd, "f16", "f16", status=status)


def appending(p):
    H, kv, D = p.heads, p.kv, p.dim
    src = p.randn(p.rows, (H + 2 * kv) * D, dtype="f16").cuda()
    prep = afx.HeadPrep(x_dtype=afx.F16, n_heads=H, eps=1e-5)

    def call(kvd, status):
        p.d_both.fill_(7.0)
        q_out = torch.full((p.rows, H * D), 7.0, dtype=torch.float16, device="cuda")
        w = (H + 2 * kv) * D
        afx.afx_paged_append(kvd, prep, src, w, src.data_ptr() + H * D * 2, w, src.data_ptr() + (H + kv) * D * 2, w, q_out, "f16", dev_status=status)
        torch.cuda.synchronize()
        return p.d_both.cpu(), q_out.cpu()
    return call


def same(got, want):
    assert all(torch.equal(g.contiguous().view(torch.uint8), w.contiguous().view(torch.uint8)) for g, w in zip(got, want))


# the last sequence with a lower start has rows, so that every kernel reports it
CASES = [([0, 5, 3, 8], 8), ([0, 10, 5, 12], 14), ([0, 200, 60, 260], 260), ([0, 10, 2, 20, 3, 25], 25), ([-3, 4, 4, 60], 61), ([4, 0, 9, 7, 90], 90),
         ([0, 150, 20, 30, 170, 160, 300], 310), ([0, 3, 1, 900], 7)]


@pytest.mark.parametrize("starts,rows", CASES)
@pytest.mark.parametrize("kind", [attention, appending])
def test_starts_that_decrease_are_clamped(starts, rows, kind):
    p = problem(starts, rows)
    got, want, status = both(p, starts, kind(p))
    same(got, want)
    assert status == 1


@pytest.mark.parametrize("seed", range(6))
@pytest.mark.parametrize("n", [3, 100, 255, 256, 700])
@pytest.mark.parametrize("kind", [attention, appending])
def test_random_starts(seed, n, kind):
    r = np.random.default_rng(1000 * n + seed)
    rows = int(r.integers(n, 6 * n)) + 300
    starts = np.sort(r.integers(0, rows + 1, n + 1))
    if seed % 2:  # a long sequence among them
        starts[n // 2:] = np.minimum(starts[n // 2:] + 200, rows)
    hurt = r.integers(0, n + 1, 1 + n // 10)
    starts[hurt] = r.integers(-5, rows + 10, len(hurt))
    p = problem(starts, rows)
    got, want, _ = both(p, starts, kind(p))
    same(got, want)
