"""Hundreds of sequences that decode and a few chunks of prompts in one call."""
import pytest
import torch

from paged_util import Problem
from paper_2504_08378_b200 import afx
from test_gpu_paged_attn import check
from test_gpu_paged_poison import median_us

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,at,chunks", [(300, [0], [200]), (300, [299], [40]), (700, [5, 350, 690], [17, 300, 64]), (64, [10, 11], [9, 500])])
@pytest.mark.parametrize("window", [0, 33])
def test_chunks_among_decoding_sequences(n, at, chunks, window):
    lens, news = [1 + (i * 13) % 60 for i in range(n)], [1 if i % 5 else 0 for i in range(n)]
    for i, c in zip(at, chunks):
        lens[i], news[i] = c + 77, c
    check(Problem(lens, news, 4, 2, 64, 16, "bf16", pad=3), window=window, sinks=3 if window else 0)


@pytest.mark.parametrize("n,chunk", [(512, 512), (2000, 300)])
def test_a_chunk_beside_decoding_sequences_costs_what_it_costs_alone(n, chunk):
    """The search for the chunk's works does not look through all sequences for every place that the grid might have
    needed: 512 sequences and a chunk of 512 tokens once took 904 us instead of 84 and 30."""
    both, times = ([200] * n + [1000], [1] * n + [chunk]), []
    for lens, news in (both, (both[0][:n], both[1][:n]), (both[0][n:], both[1][n:])):
        p = Problem(lens, news, 32, 8, 64, 16, "bf16")
        q = p.randn(p.rows, 32, 64, dtype="bf16").cuda()
        times.append(median_us(p, q, 32, 64, p.upload(afx)))
    print([round(t) for t in times])
    assert times[0] <= 2 * (times[1] + times[2])


@pytest.mark.parametrize("lens,news", [([50, 60], [4, 4]), ([9, 3, 70], [1, 1, 1]), ([40, 41], [0, 2])])
def test_a_batch_with_fewer_tokens_than_a_prompt_has(lens, news):
    """max_new is an upper bound: a batch of a few tokens in all may come with that of a whole prompt."""
    check(Problem(lens, news, 8, 2, 64, 16, "bf16"), max_new=4096)
    check(Problem(lens, news, 1, 1, 64, 16, "bf16"), max_new=4096)
