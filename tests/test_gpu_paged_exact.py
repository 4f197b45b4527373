"""Few new tokens, to the bits that their weights and queries are carried with: two halves of 16 bits each."""
import numpy as np
import pytest

from paged_util import HALF_STEP, Problem, attention_tolerance
from paper_2504_08378_b200 import afx
from test_gpu_paged_attn import attend

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cache", ["f16", "bf16"])
@pytest.mark.parametrize("q_type", ["cache", "f32"])
@pytest.mark.parametrize("heads,kv,dim,lens,news", [(4, 4, 128, [900], [1]), (32, 8, 128, [700, 40, 1300], [1, 1, 1]), (8, 2, 64, [500, 900], [8, 3]),
                                                    (48, 2, 64, [1500, 3], [1, 1]), (16, 4, 128, [400], [6])])
@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 4)])
def test_weights_lose_no_more_than_two_halves_do(cache, q_type, heads, kv, dim, lens, news, window, sinks):
    """A half leaves out at most half a step of itself: both together half a step squared, of a weight and of an fp32 query's
    value (whose share in the score's error counts twice, as the score's own).  fp16's low halves end at 2^-25 of the largest
    weight carried as 2^10, and of the largest value of a query row carried as 2^9.  The output is rounded to fp16."""
    p = Problem(lens, news, heads, kv, dim, 16, cache, seed=dim + len(lens))
    q_type = cache if q_type == "cache" else "f32"
    q = p.randn(p.rows, heads, dim, dtype=q_type)
    out, _ = attend(p, q, p.upload(afx), q_type, "f16", window, sinks)
    want, _, mass, size = p.attend(q, window, sinks)
    half = HALF_STEP[cache] ** 2
    tol = attention_tolerance(want, mass, size, dim, "f16") + 1.01 * half * mass
    if cache == "f16":  # every weight's, beside a sum of weights that is at least the largest
        tol = tol + 2.0 ** -35 * max(lens) * np.abs(mass).max()
    if q_type == "f32":
        big = q.abs().max().item() / np.sqrt(dim)
        tiny = 2.0 ** -34 * big * dim * 6 if cache == "f16" else 0.0  # (keys are below 6)
        tol = tol + 1.01 * 2 * (half * size + tiny)[..., None] * mass
    assert (np.abs(out.double().numpy() - want) <= tol).all()
