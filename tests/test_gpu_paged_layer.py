"""afx_layer_step_paged: a decoder layer over pages, every token row at its own position, against the stages of
afx_layer_step and the attention's definition in 64 bits; and a run of appending, prompts and decoding together."""
import numpy as np
import pytest
import torch

from paged_util import Problem, attention_tolerance, rope_table, turn
from paper_2504_08378_b200 import afx, synth
from paper_2504_08378_b200.model import DecoderModel

pytestmark = pytest.mark.gpu


def make(dt, heads, kvh, T, n_layers=1, max_seq=300, paged=True, mlp=512, **kw):
    hidden = 256
    layers = []
    for l in range(n_layers):
        L = synth.layer_weights(61, l, hidden, heads, kvh, mlp, dt)
        L["k"] = [hidden // 2, heads * 64, hidden // 2, mlp // 2]
        layers.append(L)
    return DecoderModel(dt, hidden, heads, kvh, mlp, max_seq, layers, T=T, paged=paged, **kw), layers


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("cache", ["f16", "bf16"])
@pytest.mark.parametrize("heads,kvh,lens,news", [(2, 2, [6], [1]), (8, 2, [200, 1, 37, 64], [1, 1, 1, 1]), (4, 1, [129, 50], [5, 2]), (4, 4, [7, 299, 16], [3, 4, 1])])
@pytest.mark.parametrize("norm,window,sinks", [(False, 0, 0), (True, 20, 3)])
def test_step_matches_its_stages(dt, cache, heads, kvh, lens, news, norm, window, sinks):
    T = sum(news)
    m, layers = make(dt, heads, kvh, T)
    plain, _ = make(dt, heads, kvh, T, paged=False)
    p = Problem(lens, news, heads, kvh, 128, 16, cache, seed=T)
    before = p.both.clone()
    kvd = p.upload(afx)
    h0 = torch.randn((T, m.hidden), generator=p.g)
    gq, gk = ((1 + 0.1 * p.randn(128)) for _ in range(2)) if norm else (None, None)
    dgq, dgk = (None if g is None else g.cuda() for g in (gq, gk))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    m.h.copy_(h0.cuda())
    m.layer_step_paged(0, kvd, window, sinks, dgq, dgk, dev_status=status)
    torch.cuda.synchronize()
    assert status.item() == 0
    # the operators around the attention are the ones of afx_layer_step, bit for bit
    plain.h.copy_(h0.cuda())
    plain.layer_kernel(0, 0, afx.STEP_QKV)
    assert torch.equal(plain.qkv, m.qkv)
    plain.bits(afx.BUF_ATTN).copy_(m.bits(afx.BUF_ATTN))
    for which in (afx.STEP_O, afx.STEP_GU, afx.STEP_DOWN):
        plain.layer_kernel(0, 0, which)
    torch.cuda.synchronize()
    assert torch.equal(plain.h, m.h)
    # new cache rows and the attention on the GPU's own q, k, v
    x = m.qkv.cpu().view(T, heads + 2 * kvh, 128)
    cos, sin = rope_table(300, 128)
    q64 = torch.zeros(T, heads, 128, dtype=torch.float64)
    got = torch.empty_strided(p.both.shape, p.both.stride(), dtype=p.both.dtype)
    got.copy_(p.d_both.cpu())
    row = 0
    for b, (n, new) in enumerate(zip(lens, news)):
        pos = torch.arange(n - new, n)
        part = x[row:row + new]
        q64[row:row + new], _ = turn(part[:, :heads], gq, 1e-5, cos[pos], sin[pos], "pairs")
        k64, size = turn(part[:, heads:heads + kvh], gk, 1e-5, cos[pos], sin[pos], "pairs")
        have = p.rows_of(got, b, 0)[n - new:].double()
        step = 2.0 ** (-8 if cache == "bf16" else -11)
        assert ((have - k64).abs() <= step * k64.abs() + 2.0 ** -25 + 31 * 2.0 ** -24 * size).all()
        assert torch.equal(p.rows_of(got, b, 1)[n - new:], part[:, heads + kvh:].to(p.both.dtype))
        for c in (0, 1):
            assert torch.equal(p.rows_of(got, b, c)[:n - new], p.rows_of(before, b, c)[:n - new])
        row += new
    want, _, mass, norm_size = p.attend(q64, window, sinks, both=got)
    out = m.bits(afx.BUF_ATTN).cpu().view(torch.bfloat16 if dt == "bf16" else torch.float16).view(T, heads, 128)
    # the kernel's queries are fp32: 32 roundings of what turn() adds up, on every product
    tol = attention_tolerance(want, mass, norm_size, 128, dt) + 2 * 40 * 2.0 ** -24 * norm_size[..., None] * mass
    assert (np.abs(out.double().numpy() - want) <= tol).all()
    m.close()
    plain.close()


def test_steps_in_a_row_captured_and_with_cross_layer_prediction():
    """Several layers and tokens without synchronisation, then the same in a graph: the same bits as step by step."""
    T, heads, kvh, n_layers, n_tok = 3, 4, 2, 3, 6
    lens0 = [40, 1, 17]
    states = []
    for mode in ("sync", "async", "graph"):
        m, _ = make("bf16", heads, kvh, T, n_layers, xl_depth=2, xl_mode=afx.XL_BOOKKEEP)
        probs = [Problem([n + n_tok for n in lens0], [1] * T, heads, kvh, 128, 16, "f16", seed=l) for l in range(n_layers)]
        kvs = [p.upload(afx) for p in probs]
        g = torch.Generator().manual_seed(5)
        hs = torch.randn((n_tok, T, m.hidden), generator=g).cuda()
        lens = torch.tensor(lens0, dtype=torch.int32, device="cuda")
        outs = torch.zeros((n_tok, T, m.hidden), device="cuda")
        cur = torch.zeros_like(hs[0])

        def step():
            lens.add_(1)
            for p in probs:
                p.d_len.copy_(lens)
            m.h.copy_(cur)
            if mode != "sync":
                m.decode_step_paged(kvs)
            else:
                for l in range(n_layers):
                    m.layer_step_paged(l, kvs[l])
                    torch.cuda.synchronize()

        if mode == "graph":
            step()  # warm
            torch.cuda.synchronize()
            lens.copy_(torch.tensor(lens0, dtype=torch.int32))
            m._view(afx.BUF_STATS, 0, torch.int32, (n_layers, 4, 4)).zero_()
            m.hints.zero_()
            for p in probs:
                p.d_both.copy_(p.both)
            s = torch.cuda.Stream()
            s.wait_stream(torch.cuda.current_stream())
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=s):
                step()
            run = graph.replay
        else:
            run = step
        for t in range(n_tok):
            cur.copy_(hs[t])
            run()
            outs[t].copy_(m.h)
        torch.cuda.synchronize()
        states.append((outs.clone(), [p.d_both.view(torch.int16).clone() for p in probs], m.stats.clone()))
        m.close()
    for other in states[1:]:
        assert torch.equal(states[0][0], other[0]) and all(torch.equal(a, b) for a, b in zip(states[0][1], other[1]))
        assert torch.equal(states[0][2][:, :, :3], other[2][:, :, :3])
    assert torch.isfinite(states[0][0]).all()


def test_refusals():
    m, _ = make("bf16", 4, 2, 2)
    p = Problem([9, 5], [1, 1], 4, 2, 128, 16, "f16")
    kvd = p.upload(afx)

    def status(**kw):
        d = afx.PagedKV.from_buffer_copy(kvd)
        ws, nb = kw.pop("ws", None), kw.pop("nb", None)
        args = dict(window=kw.pop("window", 0), sinks=kw.pop("sinks", 0), g=kw.pop("g", None))
        for k, v in kw.items():
            setattr(d, k, v)
        need = afx.afx_layer_paged_workspace_bytes(m.handle, kvd)
        buf = torch.empty(need + 256, dtype=torch.uint8, device="cuda")
        try:
            afx.afx_layer_step_paged(m.handle, 0, m.state, d, args["window"], args["sinks"], args["g"], None,
                                     (buf.data_ptr() + -buf.data_ptr() % 256) if ws is None else ws, need if nb is None else nb)
        except afx.AfxError as e:
            return e.status
        return 0

    h = m.h.clone()
    assert status(n_tokens=3) == 1 and status(n_kv_heads=4) == 1 and status(head_dim=64) == 1 and status(max_new=3) == 1
    assert status(ws=0) == 1 and status(ws=1 << 20 | 16) == 2 and status(nb=1) == 3
    assert status(dtype=2) == 4 and status(page_size=0) == 1 and status(n_seqs=-1) == 1 and status(n_seqs=70000) == 3
    assert status(window=-1) == 1 and status(g=p.d_len.data_ptr() + 4) == 2 and status(pos_stride=100) == 1
    assert afx.afx_layer_paged_workspace_bytes(0, kvd) == 0
    torch.cuda.synchronize()
    assert torch.equal(h, m.h)
    # layers without caches of their own refuse the steps that need them
    with pytest.raises(afx.AfxError):
        m.layer_step(0, 0)
    with pytest.raises(afx.AfxError):
        m.layer_kernel(0, 0, afx.STEP_ATTN)
    m.layer_kernel(0, 0, afx.STEP_QKV)
    torch.cuda.synchronize()
    m.close()


@pytest.mark.parametrize("cache,page,dim", [("bf16", 16, 128), ("f16", 7, 64)])
def test_prompts_chunks_drafts_and_tokens_together(cache, page, dim):
    """Two requests enter the cache as a prompt and in chunks, go on token by token and by drafted tokens, and each
    step's attention is that of the whole sequence so far."""
    heads, kv = 4, 2
    final = [190, 77]
    p = Problem(final, [0, 0], heads, kv, dim, page, cache, filled=False, seed=9)
    x = [p.randn(n, heads + 2 * kv, dim, dtype=cache, scale=1.5) for n in final]
    cos, sin = rope_table(max(final), dim)
    dcos, dsin = cos.cuda(), sin.cuda()
    done = [0, 0]
    full = Problem(final, final, heads, kv, dim, page, cache, seed=9)
    full.table = p.table
    # what the cache has to hold in the end, rounded once
    ref_q = []
    for b, n in enumerate(final):
        pos = torch.arange(n)
        k64, _ = turn(x[b][:, heads:heads + kv], None, 0, cos[pos], sin[pos], "halves")
        q64, _ = turn(x[b][:, :heads], None, 0, cos[pos], sin[pos], "halves")
        ref_q.append(q64)
    steps = [[100, 0], [0, 30], [30, 9], [1, 1], [1, 1], [4, 8], [1, 0], [40, 21], [1, 1], [8, 5], [4, 1]]
    for news in steps:
        lens = [d + n for d, n in zip(done, news)]
        q = Problem(lens, news, heads, kv, dim, page, cache, filled=False, seed=9)
        q.both, q.table, q.n_pages, q.width = p.both, p.table, p.n_pages, p.width
        if not hasattr(p, "pool"):
            q.upload(afx)
            p.pool = q.d_both
        kvd = q.upload(afx)
        kvd.k_pages, kvd.v_pages = p.pool[:, 0].data_ptr(), p.pool[:, 1].data_ptr()
        rows = torch.cat([x[b][done[b]:lens[b]] for b in range(2)]).reshape(sum(news), -1).contiguous().cuda()
        w, es = (heads + 2 * kv) * dim, 2
        prep = afx.HeadPrep(x_dtype=afx.DTYPES[cache], n_heads=heads, eps=0.0, rope_style=afx.ROPE_HALVES, rotary_dim=dim,
                            rope_len=max(final), rope_cos=dcos.data_ptr(), rope_sin=dsin.data_ptr())
        q_out = torch.empty((sum(news), heads, dim), dtype=rows.dtype, device="cuda")
        out = torch.empty_like(q_out)
        nb = afx.afx_paged_attn_workspace_bytes(kvd, heads)
        ws = torch.empty(max(nb, 1), dtype=torch.uint8, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        afx.afx_paged_append(kvd, prep, rows, w, rows.data_ptr() + heads * dim * es, w, rows.data_ptr() + (heads + kv) * dim * es, w,
                             q_out, cache, dev_status=status)
        afx.afx_paged_attn(kvd, q_out, cache, heads * dim, heads, 0.0, 50, 2, out, cache, None, ws, nb, dev_status=status)
        torch.cuda.synchronize()
        assert status.item() == 0
        done = lens
        now = torch.empty_strided(p.both.shape, p.both.stride(), dtype=p.both.dtype)
        now.copy_(p.pool.cpu())
        want, _, mass, size = q.attend(q_out.cpu(), 50, 2, both=now)
        tol = attention_tolerance(want, mass, size, dim, cache, cache)
        assert (np.abs(out.cpu().double().numpy() - want) <= tol).all()
    assert done == final
    step = 2.0 ** (-8 if cache == "bf16" else -11)
    for b, n in enumerate(final):
        pos = torch.arange(n)
        k64, size = turn(x[b][:, heads:heads + kv], None, 0, cos[pos], sin[pos], "halves")
        assert ((p.rows_of(now, b, 0).double() - k64).abs() <= step * k64.abs() + 2.0 ** -25 + 3.1 * 2.0 ** -24 * size).all()
        assert torch.equal(p.rows_of(now, b, 1), x[b][:, heads + kv:])


@pytest.mark.parametrize("news,window,sinks", [(1, 0, 0), (3, 0, 0), (1, 40, 3)])
def test_one_sequence_runs_on_as_it_goes_step_by_step(news, window, sinks):
    """Every layer's attention of a single sequence asks for its past before the new rows are stored: the bits are those
    of steps with the device idle between them."""
    heads, kvh, n_layers, n_tok, first = 4, 2, 3, 24, 110
    end = first + n_tok * news
    states = []
    for idle in (True, False):
        m, _ = make("f16", heads, kvh, news, n_layers)
        probs = [Problem([end], [news], heads, kvh, 128, 16, "f16", seed=l) for l in range(n_layers)]
        kvs = [p.upload(afx) for p in probs]
        hs = torch.randn((n_tok, news, m.hidden), generator=torch.Generator().manual_seed(5)).cuda()
        lens = torch.tensor([first], dtype=torch.int32, device="cuda")
        outs = torch.zeros((n_tok, news, m.hidden), device="cuda")
        for t in range(n_tok):
            lens.add_(news)
            for p in probs:
                p.d_len.copy_(lens)
            m.h.copy_(hs[t])
            for l in range(n_layers):
                m.layer_step_paged(l, kvs[l], window, sinks)
                if idle:
                    torch.cuda.synchronize()
            outs[t].copy_(m.h)
        torch.cuda.synchronize()
        states.append((outs.clone(), [p.d_both.view(torch.int16).clone() for p in probs]))
        m.close()
    assert torch.isfinite(states[0][0]).all()
    assert torch.equal(states[0][0], states[1][0]) and all(torch.equal(a, b) for a, b in zip(states[0][1], states[1][1]))


def test_sequences_that_share_pages_see_each_others_new_tokens():
    """Tokens of one text as sequences of one token each over the same pages: the second reads what the first stores in
    the same step.  The same cache as one sequence of two tokens gives the same rows up to the order of its sums."""
    heads, kvh, n = 4, 2, 150
    m, _ = make("f16", heads, kvh, 2)
    p = Problem([n], [2], heads, kvh, 128, 16, "f16", seed=3)
    one = p.upload(afx)
    h0 = torch.randn((2, m.hidden), generator=p.g).cuda()
    start = p.d_both.clone()
    m.h.copy_(h0)
    m.layer_step_paged(0, one)
    want, cache = m.bits(afx.BUF_ATTN).clone().view(torch.float16).double(), p.d_both.clone()
    two = afx.PagedKV.from_buffer_copy(one)
    lens = torch.tensor([n - 1, n], dtype=torch.int32, device="cuda")
    table = p.d_table.repeat(2, 1).contiguous()
    two.n_seqs, two.max_new, two.tok_start = 2, 1, None
    two.seq_len, two.page_table, two.table_stride = lens.data_ptr(), table.data_ptr(), table.shape[1]
    p.d_both.copy_(start)
    m.h.copy_(h0)
    m.layer_step_paged(0, two)
    got = m.bits(afx.BUF_ATTN).view(torch.float16).double()
    torch.cuda.synchronize()
    assert torch.equal(cache.view(torch.int16), p.d_both.view(torch.int16))
    # fp16 rows of values below 8: two roundings of half a step each, and sums of 150 weights in 32 bits
    assert (got - want).abs().max() <= 2 * 2.0 ** -11 * 8
    m.close()


@pytest.mark.parametrize("lens,news,out_of", [([40, 66], [1, 1], [1]), ([66], [4], [2, 3]), ([70, 9], [3, 2], [0, 1, 2])])
def test_tokens_beyond_max_seq_are_left_out(lens, news, out_of):
    """Their queries do not exist: the attention has nothing to take from what an earlier call left in the workspace."""
    T, heads, kvh = sum(news), 4, 2
    m, _ = make("f16", heads, kvh, T, max_seq=64)
    p = Problem(lens, news, heads, kvh, 128, 16, "f16", seed=3)
    kvd = p.upload(afx)
    h0 = torch.randn((T, m.hidden), generator=p.g).cuda()
    need = afx.afx_layer_paged_workspace_bytes(m.handle, kvd)
    results = []
    for fill in (0x00, 0x3C, 0xFF):  # zeros, ordinary numbers, NaN
        p.d_both.copy_(p.both)
        ws = torch.full((need + 256,), fill, dtype=torch.uint8, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        m.h.copy_(h0)
        m.bits(afx.BUF_ATTN).fill_(0x1234)
        afx.afx_layer_step_paged(m.handle, 0, m.state, kvd, 0, 0, None, None, ws.data_ptr() + -ws.data_ptr() % 256, need, dev_status=status)
        torch.cuda.synchronize()
        assert status.item() == 3
        attn = m.bits(afx.BUF_ATTN).cpu()
        for t in range(T):
            assert bool((attn[t] == 0x1234).all()) == (t in out_of)
        results.append((attn, m.h.cpu().clone()))
    assert all(torch.equal(a, results[0][0]) and torch.equal(h, results[0][1]) for a, h in results)
    # the cache rows of those tokens are as they were
    for b, n in enumerate(lens):
        for c in (0, 1):
            now = p.rows_of(p.d_both.cpu(), b, c)
            assert torch.equal(now[64:], p.rows_of(p.both, b, c)[64:])
    m.close()


@pytest.mark.parametrize("news", [[1], [1, 1, 1], [5, 3]])
def test_a_step_takes_no_memory(news):
    """The first step on a stream of the caller's must not be given memory that another stream may still be using."""
    m, _ = make("f16", 4, 2, sum(news))
    p = Problem([40 + i for i in range(len(news))], news, 4, 2, 128, 16, "f16")
    kvd = p.upload(afx)
    assert afx.afx_layer_paged_workspace_bytes(m.handle, kvd) == m._paged_bytes
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    before = torch.cuda.memory_stats()["allocation.all.allocated"]
    with torch.cuda.stream(s):
        m.layer_step_paged(0, kvd)
    torch.cuda.synchronize()
    assert torch.cuda.memory_stats()["allocation.all.allocated"] == before
    m.close()


@pytest.mark.parametrize("depth", [2, 3])
def test_cross_layer_reuse_over_pages(depth):
    """Channels predicted by an earlier layer, without synchronisation and step by step: the same bits; and not those of
    a model without prediction."""
    T, heads, kvh, n_layers, n_tok = 2, 4, 2, 4, 5
    runs = []
    for mode, idle in ((afx.XL_REUSE, True), (afx.XL_REUSE, False), (afx.XL_OFF, True)):
        m, _ = make("bf16", heads, kvh, T, n_layers, xl_depth=depth, xl_mode=mode) if mode != afx.XL_OFF else make("bf16", heads, kvh, T, n_layers)
        probs = [Problem([60 + n_tok, 9 + n_tok], [1] * T, heads, kvh, 128, 16, "f16", seed=l) for l in range(n_layers)]
        kvs = [p.upload(afx) for p in probs]
        hs = torch.randn((n_tok, T, m.hidden), generator=torch.Generator().manual_seed(5)).cuda()
        lens = torch.tensor([60, 9], dtype=torch.int32, device="cuda")
        outs = torch.zeros((n_tok, T, m.hidden), device="cuda")
        for t in range(n_tok):
            lens.add_(1)
            for p in probs:
                p.d_len.copy_(lens)
            m.h.copy_(hs[t])
            for l in range(n_layers):
                m.layer_step_paged(l, kvs[l])
                if idle:
                    torch.cuda.synchronize()
            outs[t].copy_(m.h)
        torch.cuda.synchronize()
        runs.append((outs.clone(), [p.d_both.view(torch.int16).clone() for p in probs]))
        m.close()
    assert torch.isfinite(runs[0][0]).all()
    assert torch.equal(runs[0][0], runs[1][0]) and all(torch.equal(a, b) for a, b in zip(runs[0][1], runs[1][1]))
    assert not torch.equal(runs[0][0], runs[2][0])
