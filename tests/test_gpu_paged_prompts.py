"""The tiles of 128 rows of afx_paged_attn at their edges.  Dozens of idle sequences beside the ones with new tokens make a
call busy, so that anything above AFX_MAX_T new tokens goes to the tiles; a single sequence goes there from some
256 rows on, a row tile to a work where works are few."""
import math

import numpy as np
import pytest
import torch

from paged_util import TORCH, Problem, attention_tolerance
from paper_2504_08378_b200 import afx
from test_gpu_paged_attn import attend, check

pytestmark = pytest.mark.gpu
IDLE = 80


def busy(lens, news):
    """Idle sequences in front of, between and behind the others."""
    a, b = [], []
    for n, m in zip(lens, news):
        a += [3] * (IDLE // len(lens) // 2) + [n] + [0] * (IDLE // len(lens) // 2)
        b += [0] * (IDLE // len(lens) // 2) + [m] + [0] * (IDLE // len(lens) // 2)
    return a + [2] * 4, b + [0] * 4


@pytest.mark.parametrize("n,new", [(9, 9), (31, 10), (64, 64), (127, 127), (128, 128), (129, 129), (200, 73), (256, 256), (257, 33), (384, 255), (513, 12)])
@pytest.mark.parametrize("heads,kv,dim", [(2, 2, 128), (8, 2, 64), (6, 2, 128)])
def test_edges_of_tiles_in_a_busy_call(n, new, heads, kv, dim):
    check(Problem(*busy([n], [new]), heads, kv, dim, 16, "bf16", seed=n))


@pytest.mark.parametrize("cache", ["f16", "bf16"])
@pytest.mark.parametrize("page,major", [(16, "pos"), (16, "head"), (48, "head"), (128, "pos"), (256, "head"), (7, "pos"), (24, "head")])
@pytest.mark.parametrize("dim", [64, 128])
def test_pages_and_types_in_a_busy_call(cache, page, major, dim):
    check(Problem(*busy([300, 140], [150, 20]), 4, 2, dim, page, cache, major, pad=3), out_type="f16" if cache == "bf16" else "bf16")


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 3), (5, 0), (40, 4), (64, 1), (128, 20), (129, 200), (1000, 4), (17, 1000)])
@pytest.mark.parametrize("page", [16, 64, 10])
def test_windows_in_a_busy_call(window, sinks, page):
    check(Problem(*busy([420, 140], [400, 20]), 4, 2, 64, page, "f16", pad=1), window=window, sinks=sinks)
    check(Problem(*busy([700, 60], [70, 9]), 6, 2, 128, page, "bf16"), window=window, sinks=sinks)


@pytest.mark.parametrize("n,new,heads,kv", [(600, 600, 1, 1), (900, 300, 1, 1), (400, 400, 8, 8), (300, 300, 40, 40), (1100, 257, 2, 2), (257, 257, 1, 1), (1500, 600, 12, 3)])
@pytest.mark.parametrize("dim", [64, 128])
def test_one_sequence_with_few_and_many_works(n, new, heads, kv, dim):
    check(Problem([n], [new], heads, kv, dim, 32, "f16", seed=new), window=0)
    check(Problem([n], [new], heads, kv, dim, 32, "f16", seed=new), window=200, sinks=5)


@pytest.mark.parametrize("scale", [0.01, 0.5, -0.3, 4.0])
def test_scales_in_a_busy_call(scale):
    check(Problem(*busy([350], [200]), 4, 2, 64, 16, "f16"), scale=scale, size=1.0)


@pytest.mark.parametrize("cache", ["f16", "bf16"])
def test_scores_that_grow_in_a_busy_call(cache):
    p = Problem(*busy([900], [64]), 2, 1, 64, 16, cache)
    b = p.lens.index(900)
    q = torch.zeros(p.rows, 2, 64)
    q[:, 0, 0], q[:, 1, 0] = 8.0, -8.0
    ramp = p.randn(900, 1, 64)
    ramp[:, 0, 0] = torch.linspace(-60, 60, 900)
    p.cells(b, 0)[:] = ramp
    check(p, q=q.to(TORCH[cache]))


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("window,sinks", [(20, 2), (0, 0), (1, 0), (150, 0)])
@pytest.mark.parametrize("cache,dim,page", [("f16", 64, 16), ("bf16", 128, 64), ("bf16", 64, 9)])
def test_what_a_token_does_not_see_has_no_influence_in_a_busy_call(bad, window, sinks, cache, dim, page):
    n, new = 350, 200
    p = Problem(*busy([n], [new]), 4, 2, dim, page, cache)
    b = p.lens.index(n)
    hurt = [5, 60, 180, n - 3]
    for which in (0, 1):
        rows = p.rows_of(p.both, b, which).clone()
        rows[hurt] = bad
        p.cells(b, which)[:] = rows
    q = p.randn(p.rows, 4, dim, dtype=cache)
    out, _ = attend(p, q, p.upload(afx), cache, cache, window, sinks)
    with np.errstate(all="ignore"):
        want, _, mass, norm = p.attend(q, window, sinks)
    sees = np.array([any(j <= pos and (not window or j > pos - window or j < sinks) for j in hurt) for pos in range(n - new, n)])
    clean = np.isfinite(want).all((1, 2))
    assert np.array_equal(~sees, clean)
    if clean.any():
        tol = attention_tolerance(want[clean], mass[clean], norm[clean], dim, cache, cache)
        assert (np.abs(out.double().numpy()[clean] - want[clean]) <= tol).all()
    if math.isnan(bad):
        assert torch.isnan(out[torch.from_numpy(sees)]).all()


@pytest.mark.parametrize("page", [16, 64, 12])
def test_bad_pages_are_left_out_in_a_busy_call(page):
    p = Problem(*busy([400], [120]), 4, 2, 64, page, "f16")
    b = p.lens.index(400)
    q = p.randn(p.rows, 4, 64, dtype="f16")
    kvd = p.upload(afx)
    p.d_table[b, 1], p.d_table[b, 4] = -1, p.n_pages
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, _ = attend(p, q, kvd, "f16", "f16", status=status)
    assert status.item() == 1
    K, V = (p.rows_of(p.both, b, c).double() for c in (0, 1))
    for i in (0, 60, 119):
        keep = torch.tensor([j for j in range(400 - 120 + i + 1) if j // page not in (1, 4)])
        for h in range(4):
            w = torch.softmax(K[keep, h // 2] @ q[i, h].double() / 8, 0)
            want, mass = w @ V[keep, h // 2], w @ V[keep, h // 2].abs()
            assert ((out[i, h].double() - want).abs() <= 2.0 ** -11 * want.abs() + 2.0 ** -25 + 2.0 ** -9 * mass).all()


def test_rows_that_see_nothing_in_a_busy_call():
    """More new tokens than positions: the rows in front see nothing, in tiles of their own and beside others."""
    p = Problem(*busy([300], [300]), 2, 1, 64, 16, "f16")
    b = p.lens.index(300)
    q = p.randn(p.rows, 2, 64, dtype="f16")
    kvd = p.upload(afx)
    p.d_len[b] = 20
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, lse = attend(p, q, kvd, "f16", "f16", status=status)
    assert status.item() == 1 and (out[:280] == 0).all() and torch.isneginf(lse[:280]).all()
    cut = Problem([20], [20], 2, 1, 64, 16, "f16")
    cut.table, cut.both = p.table[b:b + 1], p.both
    want, _, mass, norm = cut.attend(q[280:])
    assert (np.abs(out[280:].double().numpy() - want) <= attention_tolerance(want, mass, norm, 64, "f16", "f16")).all()


def test_same_bits_again_captured_and_beside_other_streams():
    p = Problem(*busy([700, 2000], [500, 300]), 8, 2, 128, 16, "bf16")
    q = p.randn(p.rows, 8, 128, dtype="bf16").cuda()
    kvd = p.upload(afx)
    nb = afx.afx_paged_attn_workspace_bytes(kvd, 8)
    outs = [torch.zeros((p.rows, 8, 128), dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    wss = [torch.empty(nb, dtype=torch.uint8, device="cuda") for _ in range(3)]
    call = lambda i: afx.afx_paged_attn(kvd, q, "bf16", 1024, 8, 0.0, 0, 0, outs[i], "bf16", None, wss[i], nb)
    call(0)
    torch.cuda.synchronize()
    first = outs[0].clone()
    streams = [torch.cuda.Stream() for _ in range(3)]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                call(i)
    torch.cuda.synchronize()
    assert all(torch.equal(o, first) for o in outs)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=streams[0]):
        for _ in range(3):
            call(1)
    outs[1].zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[1], first)


@pytest.mark.parametrize("dim,page,window", [(64, 16, 0), (128, 64, 0), (64, 32, 90)])
def test_more_works_than_multiprocessors(dim, page, window):
    """Several hundred works of unlike length: blocks take over others' places."""
    lens = [700, 300, 420, 301, 1000, 333]
    check(Problem(lens, [300, 300, 20, 290, 40, 333], 20, 20, dim, page, "bf16"), window=window, sinks=3)


@pytest.mark.parametrize("page", [16, 64, 10])
@pytest.mark.parametrize("lens,news", [([400], [1]), ([400, 333], [8, 3]), ([700], [300]), busy([700], [120])])
def test_pages_in_front_of_a_window_may_be_gone(page, lens, news):
    """What lies in front of every new token's window (and behind the first positions) is not touched, its pages' entries included."""
    window, sinks = 50, 5
    p = Problem(lens, news, 4, 2, 64, page, "f16")
    q = p.randn(p.rows, 4, 64, dtype="f16")
    kvd = p.upload(afx)
    gone = 0
    for b, (n, new) in enumerate(zip(p.lens, p.news)):
        low = max(0, n - new - window + 1) if new else 0
        for i in range(-(-sinks // page), low // page):
            p.d_table[b, i] = -1
            gone += 1
    assert gone > 0
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, _ = attend(p, q, kvd, "f16", "f16", window, sinks, status=status)
    assert status.item() == 0
    want, _, mass, norm = p.attend(q, window, sinks)
    assert (np.abs(out.double().numpy() - want) <= attention_tolerance(want, mass, norm, 64, "f16", "f16")).all()


def shifted(t):
    """The same values 16 bytes behind an allocation's start (which is a multiple of 256)."""
    room = torch.empty(t.untyped_storage().nbytes() + 16, dtype=torch.uint8, device="cuda")
    assert room.data_ptr() % 256 == 0
    flat = room[16:].view(t.dtype)
    out = torch.as_strided(flat, t.shape, t.stride())
    out.copy_(t)
    return out


@pytest.mark.parametrize("news", [[1, 1], [5, 8], [300, 20]])
@pytest.mark.parametrize("cache,dim", [("bf16", 128), ("f16", 64)])
def test_buffers_that_begin_on_any_16_bytes(news, cache, dim):
    p = Problem([320, 90], news, 4, 2, dim, 16, cache, pad=1)
    q = p.randn(p.rows, 4, dim, dtype=cache)
    kvd = p.upload(afx)
    pool = shifted(p.d_both)
    kvd.k_pages, kvd.v_pages = pool[:, 0].data_ptr(), pool[:, 1].data_ptr()
    dq, out = shifted(q.cuda()), shifted(torch.full((p.rows, 4, dim), 5.0, dtype=TORCH[cache], device="cuda"))
    n = afx.afx_paged_attn_workspace_bytes(kvd, 4)
    ws = torch.empty(max(n, 1), dtype=torch.uint8, device="cuda")
    afx.afx_paged_attn(kvd, dq, cache, 4 * dim, 4, 0.0, 0, 0, out, cache, None, ws, n)
    torch.cuda.synchronize()
    want, _, mass, norm = p.attend(q)
    live = sum(news)
    tol = attention_tolerance(want[:live], mass[:live], norm[:live], dim, cache, cache)
    assert (np.abs(out.cpu().double().numpy()[:live] - want[:live]) <= tol).all() and (out[live:] == 5.0).all()


@pytest.mark.parametrize("page,new", [(256, 300), (250, 300), (256, 40)])
def test_prompts_in_a_pool_beyond_32_bits(page, new):
    """A pool of more than 2^32 values: tensor copies, rows and the few tokens' split all reach its last pages."""
    kv, dim, n = 8, 128, 500
    n_pages = (1 << 32) // (kv * dim * page) + 8
    k = torch.zeros((n_pages, page, kv, dim), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    table = torch.tensor([[n_pages - 1, n_pages - 3]], dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(3)
    for c in (k, v):
        c[n_pages - 1] = torch.randn((page, kv, dim), generator=g, device="cuda").bfloat16()
        c[n_pages - 3] = torch.randn((page, kv, dim), generator=g, device="cuda").bfloat16()
    length = torch.tensor([n], dtype=torch.int32, device="cuda")
    start = torch.tensor([0, new], dtype=torch.int32, device="cuda")
    kvd = afx.PagedKV(dtype=1, n_kv_heads=kv, head_dim=dim, page_size=page, n_pages=n_pages, n_seqs=1, n_tokens=new, max_new=new,
                      page_stride=page * kv * dim, pos_stride=kv * dim, head_stride=dim, table_stride=2, k_pages=k.data_ptr(),
                      v_pages=v.data_ptr(), page_table=table.data_ptr(), seq_len=length.data_ptr(), tok_start=start.data_ptr())
    q = torch.randn((new, kv, dim), generator=g, device="cuda").bfloat16()
    out = torch.empty_like(q)
    nb = afx.afx_paged_attn_workspace_bytes(kvd, kv)
    ws = torch.empty(max(nb, 1), dtype=torch.uint8, device="cuda")
    afx.afx_paged_attn(kvd, q, "bf16", kv * dim, kv, 0.0, 0, 0, out, "bf16", None, ws, nb)
    K, V = (torch.cat((t[n_pages - 1], t[n_pages - 3]))[:n].double() for t in (k, v))
    s = torch.einsum("thd,phd->thp", q.double(), K) / dim ** 0.5
    pos = n - new + torch.arange(new, device="cuda")
    s = s.masked_fill(torch.arange(n, device="cuda")[None, None] > pos[:, None, None], -1e300)
    w = torch.softmax(s, -1)
    want, mass = torch.einsum("thp,phd->thd", w, V), torch.einsum("thp,phd->thd", w, V.abs())
    assert ((out.double() - want).abs() <= 2.0 ** -8 * want.abs() + 1.1 * 2.0 ** -8 * mass).all()
    del k, v, c
    torch.cuda.empty_cache()


@pytest.mark.parametrize("bad", [math.inf, math.nan])
@pytest.mark.parametrize("cache,dim", [("f16", 128), ("bf16", 64)])
def test_a_value_that_every_token_sees_spoils_its_dimension_alone(bad, cache, dim):
    p = Problem(*busy([1300], [1250]), 4, 2, dim, 16, cache)
    b = p.lens.index(1300)
    rows = p.rows_of(p.both, b, 1).clone()
    rows[0, :, 7] = bad
    p.cells(b, 1)[:] = rows
    q = p.randn(p.rows, 4, dim, dtype=cache)
    out, lse = attend(p, q, p.upload(afx), cache, cache)
    rows[0, :, 7] = 0
    p.cells(b, 1)[:] = rows
    want, want_lse, mass, norm = p.attend(q)
    tol = attention_tolerance(want, mass, norm, dim, cache, cache)
    o = out.double().numpy()
    assert not np.isfinite(o[..., 7]).any()
    rest = [d for d in range(dim) if d != 7]
    assert (np.abs(o - want)[..., rest] <= tol[..., rest]).all()
    assert np.abs(lse.double().numpy() - want_lse).max() <= 1e-3


def test_prompts_over_a_cache_of_nan_end_soon():
    """Everything NaN: the rows are taken again, but each ends with its first position."""
    n = 20000
    p = Problem([n], [4000], 8, 2, 64, 16, "bf16", filled=False)
    q = p.randn(p.rows, 8, 64, dtype="bf16")
    kvd = p.upload(afx)
    a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    a.record()
    out, _ = attend(p, q, kvd, "bf16", "bf16")
    b.record()
    torch.cuda.synchronize()
    assert torch.isnan(out).all()
    assert a.elapsed_time(b) < 20000  # (some milliseconds; 128000 rows of 20000 positions one after the other would be minutes)
