"""afx_paged_append against its definition in 64 bits."""
import numpy as np
import pytest
import torch

from paged_util import HALF_STEP, TINY, TORCH, Problem, rope_table, turn
from paper_2504_08378_b200 import afx

pytestmark = pytest.mark.gpu


def bits(t):
    return t.cpu().contiguous().view(torch.int16 if t.element_size() == 2 else torch.int32)


def check(p, x="f32", norm=(False, False), style="pairs", rotary=None, q_type=None, with_q=True, in_place=False, rope_len=None,
          start=True, seed=1):
    rotary = p.dim if rotary is None else rotary
    q_type = q_type or x
    H, kv, D = p.heads, p.kv, p.dim
    width = (H + 2 * kv) * D + 8
    src = p.randn(p.rows, width, dtype=x, scale=2.0)
    gq, gk = ((1 + 0.2 * p.randn(D)) if n else None for n in norm)
    n_pos = rope_len or max(p.lens + [1])
    cos, sin = rope_table(n_pos, rotary)
    kvd = p.upload(afx, start=start)
    d = src.cuda()
    dq = d[:, :H * D].contiguous() if in_place else d
    gains = [None if g is None else g.cuda() for g in (gq, gk)]
    dcos, dsin = cos.cuda(), sin.cuda()
    mark = -12345.0
    q_out = dq if in_place else torch.full((p.rows, H * D), mark, dtype=TORCH[q_type], device="cuda")
    prep = afx.HeadPrep(x_dtype=afx.DTYPES[x], n_heads=H, eps=1e-5, rope_style={"none": 0, "pairs": 1, "halves": 2}[style],
                        rotary_dim=rotary, rope_len=n_pos, g_q=None if gq is None else gains[0].data_ptr(),
                        g_k=None if gk is None else gains[1].data_ptr(), rope_cos=dcos.data_ptr(), rope_sin=dsin.data_ptr())
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    es = src.element_size()
    afx.afx_paged_append(kvd, prep, dq if with_q else None, H * D if in_place else width, d.data_ptr() + H * D * es, width,
                         d.data_ptr() + (H + kv) * D * es, width, q_out if with_q else None, q_type, dev_status=status)
    torch.cuda.synchronize()
    assert status.item() == 0
    got = torch.empty_strided(p.both.shape, p.both.stride(), dtype=p.both.dtype)
    got.copy_(p.d_both.cpu())
    touched = torch.zeros(p.both.shape, dtype=torch.bool)
    row = 0
    for b, (n, new) in enumerate(zip(p.lens, p.news)):
        pos = torch.arange(n - new, n)
        heads = src[row:row + new, :(H + 2 * kv) * D].view(new, H + 2 * kv, D)
        c, s = (cos[pos], sin[pos]) if style != "none" else (torch.ones(new, 0), torch.zeros(new, 0))
        page, slot = p.table[b, pos // p.page].long(), pos % p.page
        cells = lambda which, a: a[:, which][page, slot] if p.major == "pos" else a[:, which][page, :, slot]
        for name, part, gain in (("q", heads[:, :H], gq), ("k", heads[:, H:H + kv], gk)):
            if name == "q" and not with_q:
                continue
            want, size = turn(part, gain, 1e-5, c, s, style)
            t = q_type if name == "q" else p.cache
            have = q_out[row:row + new].cpu().view(new, H, D) if name == "q" else cells(0, got)
            # a norm: the sum of D squares, its root and quotient, two products (D / 16 lanes of 16 terms: chains of 20 additions);
            # the rotation: two products, their sum; then one rounding
            tol = HALF_STEP[t] * want.abs() + TINY[t] + 1.01 * (30 if gain is not None else 3) * 2.0 ** -24 * size
            assert ((have.double() - want).abs() <= tol).all(), (b, name, ((have.double() - want).abs() - tol).max())
        v = heads[:, H + kv:]
        assert torch.equal(bits(cells(1, got)), bits(v.to(TORCH[p.cache])))
        for which in (0, 1):
            if p.major == "pos":
                touched[:, which][page, slot] = True
            else:
                touched[:, which][page, :, slot] = True
        row += new
    untouched = ~touched
    assert torch.equal(bits(got[untouched]), bits(p.both[untouched]))  # NaN and all
    if with_q and not in_place:
        assert (q_out[row:].cpu().float() == torch.tensor(mark).to(TORCH[q_type]).float()).all()


@pytest.mark.parametrize("x", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("cache", ["f16", "bf16"])
@pytest.mark.parametrize("dim,heads,kv", [(128, 5, 1), (64, 6, 6), (128, 32, 32), (64, 64, 8)])
def test_types_and_head_layouts(x, cache, dim, heads, kv):
    check(Problem([9, 1, 40], [1, 1, 1], heads, kv, dim, 16, cache, pad=2), x)


@pytest.mark.parametrize("style", ["none", "pairs", "halves"])
@pytest.mark.parametrize("dim,rotary", [(128, 128), (128, 64), (128, 16), (128, 112), (64, 64), (64, 32), (64, 0)])
@pytest.mark.parametrize("norm", [(False, False), (True, True), (True, False), (False, True)])
def test_rotation_and_norm(style, dim, rotary, norm):
    check(Problem([70, 33], [3, 33], 6, 2, dim, 7, "bf16"), "bf16", norm, style, rotary)


@pytest.mark.parametrize("page", [1, 3, 16, 48, 64])
@pytest.mark.parametrize("major", ["pos", "head"])
@pytest.mark.parametrize("interleaved", [False, True])
def test_pages_of_any_size_and_order(page, major, interleaved):
    check(Problem([130, 1, 65, 49], [130, 1, 0, 48], 4, 2, 64, page, "f16", major, interleaved, pad=3), "f16", style="halves")


@pytest.mark.parametrize("q_type", ["f32", "f16", "bf16"])
def test_queries_in_another_type(q_type):
    check(Problem([20, 7], [2, 1], 8, 4, 128, 8, "f16"), "f32", q_type=q_type)


def test_without_queries_and_in_place():
    check(Problem([20, 7], [2, 1], 8, 4, 128, 8, "f16"), "f16", with_q=False)
    check(Problem([20, 7], [2, 1], 8, 4, 128, 8, "f16"), "f16", (True, True), "halves", in_place=True)


def test_one_row_per_sequence_without_starts():
    check(Problem([5, 1, 129], [1, 1, 1], 8, 2, 128, 16, "bf16", pad=1), "bf16", start=False)


def test_many_sequences_and_a_long_prompt():
    lens = [1 + (i * 37) % 61 for i in range(700)]
    check(Problem(lens, [1 if i % 3 else 0 for i in range(700)], 2, 1, 64, 16, "f16"), "f16")
    check(Problem([1, 3000, 5], [1, 3000, 0], 8, 2, 64, 16, "bf16"), "bf16", (True, True))


def test_bad_device_data_is_left_out():
    """A page id that is none, a position behind the table, more new tokens than positions, more than max_new: left out,
    reported, and nothing else is written."""
    for case, code in (("page", 1), ("rope", 3), ("negative", 1), ("max_new", 3), ("length", 3), ("length, rotated", 3), ("start", 1)):
        p = Problem([20, 33], [3, 4], 2, 1, 64, 8, "f16", seed=3)
        x = p.randn(p.rows, 4 * 64, dtype="f16")
        cos, sin = (t.cuda() for t in rope_table(40, 64))
        kvd = p.upload(afx, max_new=2 if case == "max_new" else None)
        live = {(0, 17), (0, 18), (0, 19), (1, 29), (1, 30), (1, 31), (1, 32)}
        rope_len = 33
        if case == "page":
            p.d_table[0, 2] = p.n_pages  # positions 16..23
            live -= {(0, 17), (0, 18), (0, 19)}
        elif case == "rope":
            rope_len = 31
            live -= {(1, 31), (1, 32)}
        elif case == "negative":
            p.d_len[0] = 1  # its three rows: positions -2, -1, 0
            live = {(0, 0)} | {t for t in live if t[0]}
        elif case == "max_new":
            live -= {(0, 19), (1, 31), (1, 32)}
        elif case.startswith("length"):
            p.d_len[1] = 1000  # the table has room for 40: positions 36..39, which the rotation's table of 33 does not reach
            p.d_table[1] = torch.arange(5, dtype=torch.int32)
            p.table[1] = torch.arange(5, dtype=torch.int32)
            p.d_table[0, 2] = p.table[0, 2] = 5
            live = {t for t in live if t[0] == 0}
            if case != "length":
                rope_len = 40
                live |= {(1, 36), (1, 37), (1, 38), (1, 39)}
        elif case == "start":
            p.d_start[2] = 100  # behind the last row: clamped, which here is what it was
        before = p.d_both.clone()
        prep = afx.HeadPrep(x_dtype=0, n_heads=2, eps=1e-5, rope_style=1, rotary_dim=64, rope_len=rope_len, rope_cos=cos.data_ptr(),
                            rope_sin=sin.data_ptr())
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        d = x.cuda()
        q_out = torch.zeros((p.rows, 128), dtype=torch.float16, device="cuda")
        afx.afx_paged_append(kvd, prep, d, 256, d.data_ptr() + 256, 256, d.data_ptr() + 384, 256, q_out, "f16", dev_status=status)
        torch.cuda.synchronize()
        assert status.item() == code, case
        a, b = (t.contiguous().view(torch.int16)[:, 1].cpu() for t in (p.d_both, before))
        changed = {tuple(c) for c in torch.nonzero((a != b).any(-1).any(-1)).tolist()}
        assert changed == {(p.table[s, pos // 8].item(), pos % 8) for s, pos in live}, case


def test_captured_and_on_another_stream():
    p = Problem([40, 9], [2, 1], 8, 4, 128, 16, "f16")
    x = p.randn(p.rows, 16 * 128, dtype="f32").cuda()
    cos, sin = (t.cuda() for t in rope_table(41, 128))
    kvd = p.upload(afx)
    prep = afx.HeadPrep(x_dtype=2, n_heads=8, eps=1e-5, rope_style=1, rotary_dim=128, rope_len=41, rope_cos=cos.data_ptr(),
                        rope_sin=sin.data_ptr())
    q_out = torch.zeros((p.rows, 1024), device="cuda")
    call = lambda: afx.afx_paged_append(kvd, prep, x, 2048, x.data_ptr() + 4096, 2048, x.data_ptr() + 6144, 2048, q_out, "f32")
    call()
    torch.cuda.synchronize()
    want, want_q = p.d_both.clone(), q_out.clone()
    p.d_both.copy_(p.both)
    q_out.zero_()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        call()
    assert not q_out.any()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(want.view(torch.int16), p.d_both.view(torch.int16)) and torch.equal(want_q, q_out)
    # new lengths on the device: the captured call follows them
    p.d_len.copy_(torch.tensor([41, 8], dtype=torch.int32))
    graph.replay()
    torch.cuda.synchronize()
    assert not torch.equal(want_q, q_out)


def test_offsets_beyond_32_bits():
    """A pool of more than 2^32 values: the last page's rows are written and read where they lie."""
    kv, dim, page = 8, 128, 256
    n_pages = (1 << 32) // (kv * dim * page) + 8
    k = torch.zeros((n_pages, page, kv, dim), dtype=torch.float16, device="cuda")
    v = torch.zeros_like(k)
    table = torch.tensor([[n_pages - 1, n_pages - 2]], dtype=torch.int32, device="cuda")
    length = torch.tensor([260], dtype=torch.int32, device="cuda")
    start = torch.tensor([0, 8], dtype=torch.int32, device="cuda")
    kvd = afx.PagedKV(dtype=0, n_kv_heads=kv, head_dim=dim, page_size=page, n_pages=n_pages, n_seqs=1, n_tokens=8, max_new=8,
                      page_stride=page * kv * dim, pos_stride=kv * dim, head_stride=dim, table_stride=2, k_pages=k.data_ptr(),
                      v_pages=v.data_ptr(), page_table=table.data_ptr(), seq_len=length.data_ptr(), tok_start=start.data_ptr())
    x = torch.randn((8, 3 * kv * dim), device="cuda").half()
    prep = afx.HeadPrep(x_dtype=0, n_heads=kv, eps=1e-5, rope_style=0)
    q = torch.empty((8, kv * dim), dtype=torch.float16, device="cuda")
    w = 3 * kv * dim
    afx.afx_paged_append(kvd, prep, x, w, x.data_ptr() + 2 * kv * dim, w, x.data_ptr() + 4 * kv * dim, w, q, "f16")
    torch.cuda.synchronize()
    want_k, want_v = x[:, kv * dim:2 * kv * dim].view(8, kv, dim), x[:, 2 * kv * dim:].view(8, kv, dim)
    assert torch.equal(k[n_pages - 1, 252:], want_k[:4]) and torch.equal(k[n_pages - 2, :4], want_k[4:])
    assert torch.equal(v[n_pages - 1, 252:], want_v[:4]) and torch.equal(v[n_pages - 2, :4], want_v[4:])
    out = torch.empty((8, kv, dim), dtype=torch.float16, device="cuda")
    nb = afx.afx_paged_attn_workspace_bytes(kvd, kv)
    ws = torch.empty(max(nb, 1), dtype=torch.uint8, device="cuda")
    afx.afx_paged_attn(kvd, q, "f16", kv * dim, kv, 0.0, 0, 0, out, "f16", None, ws, nb)
    K, V = (torch.cat((t[n_pages - 1], t[n_pages - 2, :4])).double() for t in (k, v))
    s = torch.einsum("thd,phd->thp", q.view(8, kv, dim).double(), K) / dim ** 0.5
    s = s.masked_fill(torch.arange(260, device="cuda")[None, None] > 252 + torch.arange(8, device="cuda")[:, None, None], -1e300)
    wgt = torch.softmax(s, -1)
    want = torch.einsum("thp,phd->thd", wgt, V)
    mass = torch.einsum("thp,phd->thd", wgt, V.abs())
    assert ((out.double() - want).abs() <= 2.0 ** -11 * want.abs() + 2.0 ** -25 + 2.0 ** -10 * mass).all()
    del k, v
    torch.cuda.empty_cache()


def test_buffers_that_begin_on_any_16_bytes():
    p = Problem([20, 7], [3, 1], 4, 2, 64, 8, "f16")
    x = p.randn(p.rows, 8 * 64, dtype="f16")
    kvd = p.upload(afx)
    cos, sin = (t.cuda() for t in rope_table(20, 64))
    outs = []
    for shift in (0, 16):
        p.d_both.copy_(p.both)
        room = [torch.zeros(n * 4 + 16, dtype=torch.uint8, device="cuda") for n in (x.numel(), 20 * 32, 20 * 32, p.rows * 256)]
        dx = room[0][shift:shift + x.numel() * 2].view(torch.float16).view(x.shape)
        dx.copy_(x)
        tabs = [r[shift:shift + 20 * 32 * 4].view(torch.float32).view(20, 32) for r in room[1:3]]
        tabs[0].copy_(cos)
        tabs[1].copy_(sin)
        q_out = room[3][shift:shift + p.rows * 512].view(torch.float16)
        prep = afx.HeadPrep(x_dtype=0, n_heads=4, eps=1e-5, rope_style=2, rotary_dim=64, rope_len=20, rope_cos=tabs[0].data_ptr(),
                            rope_sin=tabs[1].data_ptr())
        afx.afx_paged_append(kvd, prep, dx, 512, dx.data_ptr() + 512, 512, dx.data_ptr() + 768, 512, q_out, "f16")
        torch.cuda.synchronize()
        outs.append((p.d_both.clone().view(torch.int16), q_out.clone()))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1]) and outs[0][1].any()


@pytest.mark.parametrize("start", [True, False])
def test_rows_that_no_sequence_has_need_not_exist(start):
    """A batch padded far behind the live rows (and, with starts, begun behind its first ones): q, k, v and q_out hold the
    live rows alone."""
    H, kv, D, live, front = 8, 2, 128, 3, 4 if start else 0
    p = Problem([20, 7, 33], [1, 1, 1], H, kv, D, 16, "f16")
    src = p.randn(live, (H + 2 * kv) * D, dtype="f16").cuda()
    w = (H + 2 * kv) * D
    prep = afx.HeadPrep(x_dtype=afx.F16, n_heads=H, eps=1e-5)
    kvd = p.upload(afx, start=start)
    if start:
        p.d_start += front
    kvd.n_tokens = 100000
    q_out = torch.zeros((live, H * D), dtype=torch.float16, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    row = lambda t, first: t.data_ptr() + first * 2 - front * t.stride(0) * 2  # where row 0 would be
    afx.afx_paged_append(kvd, prep, row(src, 0), w, row(src, H * D), w, row(src, (H + kv) * D), w, row(q_out, 0), "f16", dev_status=status)
    torch.cuda.synchronize()
    assert status.item() == 0 and torch.equal(q_out, src[:, :H * D])
    for b, n in enumerate(p.lens):
        page, slot = p.table[b, (n - 1) // 16].item(), (n - 1) % 16
        got = p.d_both[page, :, slot].cpu()
        assert torch.equal(got.reshape(-1), src[b, H * D:].cpu())
