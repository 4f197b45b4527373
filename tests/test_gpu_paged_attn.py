"""afx_paged_attn against its definition in 64 bits: few new tokens and prompts, masks, layouts, what lies at
positions that nobody sees."""
import math

import numpy as np
import pytest
import torch

from paged_util import TORCH, Problem, attention_tolerance
from paper_2504_08378_b200 import afx

pytestmark = pytest.mark.gpu

MARK = -1234.0


def workspace(kvd, heads):
    n = afx.afx_paged_attn_workspace_bytes(kvd, heads)
    # what an earlier call left there has no influence
    return torch.full((max(n, 1),), 0xFF, dtype=torch.uint8, device="cuda"), n


def attend(p, q, kvd, q_type, out_type, window=0, sinks=0, scale=0.0, lse=True, gap=0, status=None):
    H, D = p.heads, p.dim
    rows = torch.full((p.rows, H * D + gap), math.nan, dtype=TORCH[q_type], device="cuda")
    rows[:, :H * D] = q.reshape(p.rows, H * D).to(TORCH[q_type]).cuda()
    out = torch.full((p.rows, H, D), MARK, dtype=TORCH[out_type], device="cuda")
    l = torch.full((p.rows, H), MARK, device="cuda") if lse else None
    ws, n = workspace(kvd, H)
    afx.afx_paged_attn(kvd, rows, q_type, H * D + gap, H, scale, window, sinks, out, out_type, l, ws, n, dev_status=status)
    torch.cuda.synchronize()
    return out.cpu(), l.cpu() if lse else None


def check(p, q_type=None, out_type=None, window=0, sinks=0, scale=0.0, gap=0, size=1.5, max_new=None, start=True, q=None):
    q_type, out_type = q_type or p.cache, out_type or p.cache
    q = p.randn(p.rows, p.heads, p.dim, dtype=q_type, scale=size) if q is None else q
    kvd = p.upload(afx, max_new, start)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, lse = attend(p, q, kvd, q_type, out_type, window, sinks, scale, gap=gap, status=status)
    assert status.item() == 0
    want, want_lse, mass, norm = p.attend(q, window, sinks, scale or None)
    live = sum(p.news)
    o, l = out.double().numpy(), lse.double().numpy()
    assert (o[live:] == TORCH_MARK[out_type]).all() and (l[live:] == MARK).all()
    tol = attention_tolerance(want[:live], mass[:live], norm[:live], p.dim, out_type, p.cache)
    err = np.abs(o[:live] - want[:live])
    assert np.isfinite(o[:live]).all() and (err <= tol).all(), (err / np.maximum(tol, 1e-30)).max()
    empty = np.isinf(want_lse[:live])
    assert (l[:live][empty] == -np.inf).all()
    # the log of a sum whose terms are off as the weights are, and its own rounding
    ltol = 2 * ((p.dim + 4) * 2.0 ** -23 * norm[:live] + 2.0 ** -20) + 2.0 ** -22 * np.abs(want_lse[:live])
    assert (np.abs(l[:live] - want_lse[:live])[~empty] <= ltol[~empty]).all()
    return out, lse


TORCH_MARK = {t: float(torch.tensor(MARK).to(TORCH[t])) for t in ("f16", "bf16")}


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 200, 1000])
@pytest.mark.parametrize("heads,kv,dim", [(3, 3, 128), (8, 1, 64), (16, 2, 128), (5, 1, 64)])
def test_one_new_token_at_the_edges_of_tiles(n, heads, kv, dim):
    check(Problem([n], [1], heads, kv, dim, 16, "f16", seed=n))


@pytest.mark.parametrize("cache", ["f16", "bf16"])
@pytest.mark.parametrize("q_type", ["cache", "f32"])
@pytest.mark.parametrize("out_type", ["f16", "bf16"])
@pytest.mark.parametrize("heads,kv,dim", [(32, 32, 128), (64, 8, 128), (28, 4, 64), (40, 1, 64), (9, 1, 128)])
def test_types_and_head_layouts(cache, q_type, out_type, heads, kv, dim):
    check(Problem([77, 1, 300], [1, 1, 1], heads, kv, dim, 16, cache, pad=2), cache if q_type == "cache" else "f32", out_type)


@pytest.mark.parametrize("page", [1, 3, 16, 48, 64, 256])
@pytest.mark.parametrize("major", ["pos", "head"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("news", [[1, 1, 1, 1], [8, 1, 0, 3], [130, 1, 0, 48]])
def test_pages_of_any_size_and_order(page, major, interleaved, news):
    check(Problem([130, 1, 65, 497], news, 4, 2, 64, page, "f16", major, interleaved, pad=3))


@pytest.mark.parametrize("heads,kv,dim", [(4, 4, 128), (8, 1, 64), (12, 2, 128), (7, 1, 128), (6, 2, 64)])
@pytest.mark.parametrize("news", [[2, 5, 8], [1, 8, 7]])
@pytest.mark.parametrize("q_type", ["f16", "f32"])
def test_a_few_new_tokens_see_each_other_in_order(heads, kv, dim, news, q_type):
    check(Problem([9, 200, 8], news, heads, kv, dim, 16, "f16"), q_type)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 3), (5, 0), (16, 4), (64, 1), (100, 64), (1000, 4), (17, 1000)])
@pytest.mark.parametrize("news", [[1, 1, 1, 1], [4, 1, 8, 8], [300, 1, 20, 9], [1, 17, 64, 129]])
@pytest.mark.parametrize("cache", ["f16", "bf16"])
def test_window_and_first_positions(window, sinks, news, cache):
    check(Problem([300, 17, 64, 129], news, 4, 2, 64, 16, cache, pad=1), window=window, sinks=sinks)


@pytest.mark.parametrize("cache", ["f16", "bf16"])
@pytest.mark.parametrize("heads,kv,dim,page", [(4, 4, 128, 16), (8, 1, 128, 48), (6, 2, 64, 64), (3, 1, 64, 7), (16, 8, 128, 128), (40, 8, 64, 32)])
def test_prompts_alone_and_behind_a_prefix(cache, heads, kv, dim, page):
    check(Problem([140, 500, 1, 64, 257], [140, 129, 1, 9, 200], heads, kv, dim, page, cache, pad=2, seed=dim))


@pytest.mark.parametrize("n,new", [(9, 9), (31, 10), (127, 127), (128, 128), (129, 129), (256, 256), (257, 33), (384, 255), (700, 700), (1031, 518)])
@pytest.mark.parametrize("heads,kv", [(2, 2), (8, 2), (3, 1)])
def test_prompts_at_the_edges_of_tiles(n, new, heads, kv):
    check(Problem([n], [new], heads, kv, 128, 16, "bf16", seed=n))


@pytest.mark.parametrize("scale", [0.01, 0.5, -0.3, 4.0])
@pytest.mark.parametrize("new", [1, 100])
def test_scales(scale, new):
    check(Problem([150], [new], 4, 2, 64, 16, "f16"), scale=scale, size=1.0)


@pytest.mark.parametrize("new", [1, 64])
@pytest.mark.parametrize("cache", ["f16", "bf16"])
def test_scores_that_grow_along_the_sequence(new, cache):
    """The running maximum moves in every tile, by far (the rescaling of what has been summed)."""
    p = Problem([900], [new], 2, 1, 64, 16, cache)
    q = torch.zeros(p.rows, 2, 64)
    q[:, 0, 0], q[:, 1, 0] = 8.0, -8.0
    ramp = p.randn(900, 1, 64)
    ramp[:, 0, 0] = torch.linspace(-60, 60, 900)
    p.cells(0, 0)[:] = ramp
    check(p, q=q.to(TORCH[cache]))


def test_query_rows_with_a_stride_and_no_starts():
    check(Problem([90, 33], [1, 1], 8, 2, 128, 16, "f16", pad=1), gap=24, start=False)
    check(Problem([90, 33], [40, 9], 8, 2, 128, 16, "f16", pad=1), gap=24)


@pytest.mark.parametrize("news", [[0, 0], [0, 3], [0, 40]])
def test_sequences_without_new_tokens_or_positions(news):
    check(Problem([0, 50], news, 4, 2, 64, 16, "f16", pad=4), max_new=max(news + [1]))


@pytest.mark.parametrize("max_new", [1, 8, 33])
def test_tokens_that_see_nothing(max_new):
    """More new tokens than positions: the rows in front see nothing, the others what they should."""
    p = Problem([6, 20], [max_new, max_new], 4, 2, 64, 16, "f16") if max_new <= 6 else Problem([max_new, 40], [max_new, 3], 4, 2, 64, 16, "f16")
    q = p.randn(p.rows, 4, 64, dtype="f16")
    kvd = p.upload(afx)
    cut = 0 if max_new == 1 else 3
    p.d_len[0] = cut
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, lse = attend(p, q, kvd, "f16", "f16", status=status)
    assert status.item() == 1
    empty = p.news[0] - cut
    assert (out[:empty] == 0).all() and torch.isneginf(lse[:empty]).all()
    p2 = Problem([cut, p.lens[1]], [cut, p.news[1]], 4, 2, 64, 16, "f16")
    p2.table, p2.both = p.table, p.both
    want, _, mass, norm = p2.attend(q[empty:])
    tol = attention_tolerance(want, mass, norm, 64, "f16", "f16")
    assert (np.abs(out[empty:].double().numpy() - want) <= tol).all()


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("new,window,sinks", [(1, 20, 2), (6, 20, 2), (6, 0, 0), (100, 20, 2), (100, 0, 0), (100, 1, 0)])
@pytest.mark.parametrize("heads", [2, 20])
@pytest.mark.parametrize("cache,dim", [("f16", 64), ("bf16", 128)])
def test_what_a_token_does_not_see_has_no_influence(bad, new, window, sinks, heads, cache, dim):
    """NaN and infinities behind a token, in front of its window, and (everywhere in these tests) in the free cells of the
    pages.  A token that sees one gets what the formula gives."""
    n = 150
    p = Problem([n, 40], [new, 1], heads, 2, dim, 16, cache)
    hurt = [n - 3, n - new + 1, 5, 60] if new > 1 else [5, 60]
    for which in (0, 1):
        rows = p.rows_of(p.both, 0, which).clone()
        rows[hurt] = bad
        p.cells(0, which)[:] = rows
    q = p.randn(p.rows, heads, dim, dtype=cache)
    kvd = p.upload(afx)
    out, lse = attend(p, q, kvd, cache, cache, window, sinks)
    with np.errstate(all="ignore"):
        want, want_lse, mass, norm = p.attend(q, window, sinks)
    clean = np.isfinite(want).all((1, 2))
    assert clean.any()
    tol = attention_tolerance(want[clean], mass[clean], norm[clean], dim, cache, cache)
    assert (np.abs(out.double().numpy()[clean] - want[clean]) <= tol).all()
    sees = np.array([any(j <= pos and (not window or j > pos - window or j < sinks) for j in hurt) for pos in range(n - new, n)] + [False])
    assert np.array_equal(~sees, clean)
    if math.isnan(bad):
        assert torch.isnan(out[torch.from_numpy(sees)]).all()


def test_an_infinite_value_makes_its_dimension_infinite_and_nothing_else():
    for new in (1, 100):
        p = Problem([150], [new], 4, 2, 64, 16, "f16")
        rows = p.rows_of(p.both, 0, 1).clone()
        rows[3, :, 10], rows[20, :, 33] = math.inf, -math.inf
        p.cells(0, 1)[:] = rows
        q = p.randn(new, 4, 64, dtype="f16")
        out, _ = attend(p, q, p.upload(afx), "f16", "f16")
        want, _, mass, norm = p.attend(q)
        fin = np.isfinite(want)
        assert np.array_equal(out.double().numpy()[~fin], want[~fin]) and (~fin).any()
        mass[~fin] = 0
        tol = attention_tolerance(np.where(fin, want, 0), mass, norm, 64, "f16", "f16")
        assert (np.abs(out.double().numpy() - want)[fin] <= tol[fin]).all()


def test_bad_pages_are_left_out_and_reported():
    for new in (1, 5, 60):
        p = Problem([100, 70], [new, new], 4, 2, 64, 16, "f16")
        q = p.randn(p.rows, 4, 64, dtype="f16")
        kvd = p.upload(afx)
        p.d_table[0, 1], p.d_table[0, 4] = -1, p.n_pages  # positions 16..31 and 64..79
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        out, _ = attend(p, q, kvd, "f16", "f16", status=status)
        assert status.item() == 1
        gone = [j for j in range(100) if j // 16 in (1, 4)]
        K, V = (p.rows_of(p.both, 0, c).double() for c in (0, 1))
        for i in (0, new - 1):
            pos = 100 - new + i
            keep = torch.tensor([j for j in range(pos + 1) if j not in gone])
            for h in range(4):
                w = torch.softmax(K[keep, h // 2] @ q[i, h].double() / 8, 0)
                want, mass = w @ V[keep, h // 2], w @ V[keep, h // 2].abs()
                assert ((out[i, h].double() - want).abs() <= 2.0 ** -11 * want.abs() + 2.0 ** -25 + 2.0 ** -9 * mass).all()


def test_lengths_beyond_the_table_and_rows_beyond_max_new():
    p = Problem([64, 20], [4, 4], 4, 2, 64, 16, "f16")
    q = p.randn(p.rows, 4, 64, dtype="f16")
    kvd = p.upload(afx, max_new=3)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, _ = attend(p, q, kvd, "f16", "f16", status=status)
    assert status.item() == 3
    want, _, mass, norm = p.attend(q)
    tol = attention_tolerance(want, mass, norm, 64, "f16", "f16")
    rows = [0, 1, 2, 4, 5, 6]
    assert (np.abs(out.double().numpy() - want)[rows] <= tol[rows]).all()
    assert (out[[3, 7]] == TORCH_MARK["f16"]).all()
    kvd = p.upload(afx)
    p.d_len[0] = 1 << 30  # clamped to the table's 64
    status.zero_()
    out, _ = attend(p, q, kvd, "f16", "f16", status=status)
    assert status.item() == 3 and (np.abs(out.double().numpy() - want) <= tol).all()


@pytest.mark.parametrize("news", [[1] * 40, [8] * 40, [64] * 40])
def test_many_sequences(news):
    lens = [max(n, 1 + (i * 97) % 400) for i, n in enumerate(news)]
    check(Problem(lens, news, 4, 1, 64, 16, "bf16"))


@pytest.mark.parametrize("lens,heads,kv", [([20000], 8, 1), ([9000, 3, 1, 5000], 8, 2), ([30000, 1], 2, 2)])
def test_long_sequences_are_split_and_joined(lens, heads, kv):
    check(Problem(lens, [1] * len(lens), heads, kv, 128, 64, "bf16"))
    check(Problem(lens, [1] * len(lens), heads, kv, 64, 24, "f16"), "f32")


@pytest.mark.parametrize("news", [[1, 1, 1], [5, 1, 3], [200, 70, 9]])
def test_same_bits_again_on_other_streams_and_in_a_graph(news):
    p = Problem([2000, 70, 300], news, 8, 2, 128, 16, "bf16")
    q = p.randn(p.rows, 8, 128, dtype="bf16").cuda()
    kvd = p.upload(afx)
    outs = [torch.zeros((p.rows, 8, 128), dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    wss = [workspace(kvd, 8) for _ in range(3)]
    call = lambda i: afx.afx_paged_attn(kvd, q, "bf16", 1024, 8, 0.0, 0, 0, outs[i], "bf16", None, wss[i][0], wss[i][1])
    call(0)
    torch.cuda.synchronize()
    first = outs[0].clone()
    streams = [torch.cuda.Stream() for _ in range(3)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(10):  # calls that overlap, a workspace each
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                call(i)
    torch.cuda.synchronize()
    assert all(torch.equal(o, first) for o in outs)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=streams[0]):
        call(1)
    outs[1].zero_()
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[1], first)
    # lengths are read when the graph runs
    p.d_len.copy_(torch.tensor([1500, 70, 250], dtype=torch.int32))
    graph.replay()
    torch.cuda.synchronize()
    got = outs[1].cpu()
    p.lens = [1500, 70, 250]
    want, _, mass, norm = p.attend(q.cpu())
    assert (np.abs(got.double().numpy() - want) <= attention_tolerance(want, mass, norm, 128, "bf16", "bf16")).all()


def test_joining_two_caches_by_their_sums():
    """out and lse of two halves of a sequence give the whole sequence's."""
    p = Problem([300, 200], [1, 1], 4, 2, 64, 16, "f16")
    q = p.randn(2, 4, 64, dtype="f16")
    whole = Problem([500], [1], 4, 2, 64, 16, "f16")
    for c in (0, 1):
        whole.cells(0, c)[:] = torch.cat((p.rows_of(p.both, 0, c), p.rows_of(p.both, 1, c)))
    q[1] = q[0]
    out, lse = attend(p, q, p.upload(afx), "f16", "f16")
    want, want_lse, mass, norm = whole.attend(q[:1])
    w = torch.softmax(lse.double(), 0)
    joined = (w[..., None] * out.double()).sum(0).numpy()
    tol = attention_tolerance(want, mass, norm, 64, "f16", "f16")[0] + 2.0 ** -11 * (w[..., None] * out.double().abs()).sum(0).numpy()
    assert (np.abs(joined - want[0]) <= tol).all()
    assert np.abs(torch.logsumexp(lse.double(), 0).numpy() - want_lse[0]).max() <= 1e-4


@pytest.mark.parametrize("news", [[1, 1], [40, 7], [3, 60]])
def test_the_largest_windows_and_counts_of_first_positions(news):
    most = 2 ** 31 - 1
    for window, sinks in ((most, 0), (most, most), (5, most), (0, most)):
        p = Problem([200, 61], news, 4, 2, 64, 16, "f16")
        check(p, window=window if window < most else 10 ** 9, sinks=sinks if sinks < most else 10 ** 9)
        q = p.randn(p.rows, 4, 64, dtype="f16")
        kvd = p.upload(afx)
        assert torch.equal(attend(p, q, kvd, "f16", "f16", window, sinks)[0],
                           attend(p, q, kvd, "f16", "f16", min(window, 10 ** 9), min(sinks, 10 ** 9))[0])


@pytest.mark.parametrize("news", [[2, 1], [40, 9]])
def test_rows_in_front_of_the_first_sequence_stay(news):
    p = Problem([100, 61], news, 4, 2, 64, 16, "f16", pad=5)
    q = p.randn(p.rows, 4, 64, dtype="f16")
    kvd = p.upload(afx)
    p.d_start += 3  # three rows in front, two behind
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, lse = attend(p, q, kvd, "f16", "f16", status=status)
    assert status.item() == 0 and (out[:3] == TORCH_MARK["f16"]).all() and (out[-2:] == TORCH_MARK["f16"]).all()
    want, _, mass, norm = p.attend(torch.cat((q[3:], q[:3])))
    n = sum(news)
    tol = attention_tolerance(want[:n], mass[:n], norm[:n], 64, "f16", "f16")
    assert (np.abs(out[3:3 + n].double().numpy() - want[:n]) <= tol).all()


@pytest.mark.parametrize("every", [1, 7, 40])
def test_thousands_of_sequences_most_of_them_idle(every):
    """Every so many sequences has a token (or, seldom, a few dozen): the others take no part."""
    n = 3000
    news = [0 if i % every else (30 if i % (every * 50) == 0 else 1 + i % 3) for i in range(n)]
    lens = [max(m, 1 + (i * 13) % 60) for i, m in enumerate(news)]
    check(Problem(lens, news, 2, 1, 64, 16, "f16"))


@pytest.mark.parametrize("cache,dim,heads,kv", [("bf16", 128, 16, 2), ("f16", 64, 6, 3)])
def test_prompts_beside_decoding_sequences(cache, dim, heads, kv):
    check(Problem([700, 333, 900, 60, 1, 2000, 12], [300, 1, 9, 60, 1, 8, 12], heads, kv, dim, 16, cache, pad=1))
    check(Problem([700, 333, 900, 60, 1, 2000, 12], [300, 1, 9, 60, 1, 8, 12], heads, kv, dim, 48, cache, pad=1), window=100, sinks=5)


@pytest.mark.parametrize("heads,kv", [(8, 8), (16, 2), (40, 2)])
@pytest.mark.parametrize("cache,dim", [("f16", 128), ("bf16", 64)])
@pytest.mark.parametrize("lens", [[900], [900, 40]])
def test_one_token_over_an_infinite_value(heads, kv, cache, dim, lens):
    p = Problem(lens, [1] * len(lens), heads, kv, dim, 16, cache)
    rows = p.rows_of(p.both, 0, 1).clone()
    rows[0, :, 7], rows[700, :, 9] = math.inf, -math.inf
    p.cells(0, 1)[:] = rows
    q = p.randn(p.rows, heads, dim, dtype=cache)
    out, lse = attend(p, q, p.upload(afx), cache, cache)
    rows[0, :, 7] = rows[700, :, 9] = 0
    p.cells(0, 1)[:] = rows
    want, _, mass, norm = p.attend(q)
    tol = attention_tolerance(want, mass, norm, dim, cache, cache)
    o = out.double().numpy()
    assert (o[0, :, 7] == np.inf).all() and (o[0, :, 9] == -np.inf).all() and torch.isfinite(lse).all()
    o[0][:, [7, 9]] = want[0][:, [7, 9]]
    assert (np.abs(o - want) <= tol).all()
