"""Measured calls of the paged key-value cache operators: appending new tokens (with the norms of the heads and the
rotation of positions) and attention over the cache, for few new tokens and for prompts.

``run`` computes a case with the library's calls where ``own`` is true, in elementary torch operations otherwise.
Case fields: ``lens`` (positions of every sequence, the new ones included) and ``news`` (new tokens of every
sequence) are comma-separated lists; ``pad`` counts token rows behind the last sequence, which stay as they are.
"""
import math
import random

import torch

own = False

_T = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def _ints(text):
    return [int(t) for t in text.split(",")]


def _text(values):
    return ",".join(str(v) for v in values)


def _spread(n, lo, hi, key):
    """n whole numbers spread over the logarithm of [lo, hi]."""
    r = random.Random(key)
    return [max(lo, min(hi, round(math.exp(r.uniform(math.log(lo), math.log(hi)))))) for _ in range(n)]


def _append(name, lens, news, heads, kv, dim, page, x, cache, norm, style, rotary, pad=0):
    return dict(name=name, op="append", lens=_text(lens), news=_text(news), heads=heads, kv=kv, dim=dim, page=page, x=x,
                cache=cache, norm=norm, style=style, rotary=rotary, pad=pad)


def _attend(name, lens, news, heads, kv, dim, page, q, cache, window=0, sinks=0, major="pos", pad=0):
    return dict(name=name, op="attend", lens=_text(lens), news=_text(news), heads=heads, kv=kv, dim=dim, page=page, q=q,
                cache=cache, window=window, sinks=sinks, major=major, pad=pad)


def listed():
    return [
        # one new token of one sequence, q | k | v in fp32 as the layer's operator leaves them: pure latency
        _append("append_one_token", [2049], [1], 32, 32, 128, 64, "f32", "f16", False, "pairs", 128),
        # one new token of each of 96 requests, normed heads, padded batch
        _append("append_batch_normed", _spread(96, 1, 2000, 1), [1] * 96, 64, 8, 128, 16, "bf16", "bf16", True, "halves", 128, pad=32),
        # prompts of a few requests enter the cache at once, part of each head rotated
        _append("append_prompts", [4096, 777, 3111, 60], [4096, 777, 2048, 59], 40, 40, 128, 48, "bf16", "bf16", False, "halves", 64),
        # decode of one sequence, one query head per kv head (7B-shaped layer), fp32 queries
        _attend("attend_one_sequence", [2049], [1], 32, 32, 128, 64, "f32", "f16"),
        # the smallest call: a sequence that has only begun
        _attend("attend_short", [37], [1], 32, 8, 64, 16, "f16", "f16"),
        # a ragged decode batch (70B-shaped layer), padded
        _attend("attend_ragged_batch", _spread(61, 1, 8192, 2), [1] * 61, 64, 8, 128, 16, "bf16", "bf16", pad=3),
        # one very long context, pages stored head by head
        _attend("attend_long_context", [131072], [1], 64, 8, 128, 64, "bf16", "bf16", major="head"),
        # window and first tokens over long contexts
        _attend("attend_window_batch", _spread(64, 2000, 32000, 3), [1] * 64, 32, 8, 128, 32, "f16", "f16", window=4096, sinks=4),
        # a few drafted tokens per sequence checked at once
        _attend("attend_draft_check", _spread(16, 300, 6000, 4), _spread(16, 1, 8, 5), 32, 8, 128, 24, "bf16", "bf16"),
        # a whole prompt (70B-shaped layer)
        _attend("prompt_whole", [8192], [8192], 64, 8, 128, 64, "bf16", "bf16"),
        # chunks of several prompts behind cached prefixes, a page size that ends inside tiles
        _attend("prompt_ragged_chunks", [1500, 4096, 300, 2611, 17, 5000], [1500, 1024, 299, 2048, 17, 1], 32, 8, 128, 48, "f16", "f16", pad=7),
        # a long prompt with a window and first tokens
        _attend("prompt_window", [16384], [16384], 32, 8, 64, 128, "bf16", "bf16", window=1024, sinks=4),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    dim = rng.choice([64, 128])
    heads, kv = rng.choice([(32, 32), (40, 40), (64, 8), (32, 8), (8, 1), (28, 4), (15, 5), (6, 2)])
    page = rng.choice([1, 8, 16, 24, 32, 48, 64, 100, 128, 256])
    dtype = rng.choice(["f16", "bf16"])
    kind = rng.choice(["append", "append", "few", "few", "few", "prompt", "prompt"])
    if kind == "append":
        if rng.random() < 0.5:  # decode batch
            n = _log(rng, 1, 96)
            lens = [_log(rng, 1, 2000) for _ in range(n)]
            news = [1] * n
        else:
            n = rng.randint(1, 5)
            lens = [_log(rng, 1, 4000) for _ in range(n)]
            news = [rng.randint(1, m) for m in lens]
        return _append("drawn", lens, news, heads, kv, dim, page, rng.choice(["f32", dtype]), dtype, rng.random() < 0.5,
                       rng.choice(["pairs", "halves"]), rng.choice([dim, dim // 2]), pad=rng.choice([0, 0, 5]))
    if kind == "few":
        n = _log(rng, 1, 64)
        top = max(8, min(131072, int(1e9 / (4 * kv * dim * n))))  # at most a gigabyte of cache
        lens = [_log(rng, 1, top) for _ in range(n)]
        news = [1] * n if rng.random() < 0.6 else [min(m, rng.randint(1, 8)) for m in lens]
    else:
        n = rng.randint(1, 6)
        lens = [_log(rng, 1, 8192 // n) for _ in range(n)]
        lens[0] = max(lens[0], 9)
        news = [rng.randint(1, m) for m in lens]
        news[0] = max(news[0], 9)
    window, sinks = (_log(rng, 1, 4096), rng.choice([0, 1, 4, 16])) if rng.random() < 0.4 else (0, 0)
    q = rng.choice(["f32", dtype]) if kind == "few" else dtype
    return _attend("drawn", lens, news, heads, kv, dim, page, q, dtype, window, sinks, rng.choice(["pos", "pos", "head"]),
                   pad=rng.choice([0, 0, 5]))


def prepare(case, seed):
    """The cache, its page table in shuffled order, lengths on the device and on the host, the new tokens' rows,
    output buffers; the rotation's table; for the library also its descriptor and workspace."""
    dev = "cuda"
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    lens, news = _ints(case["lens"]), _ints(case["news"])
    n, page, kv, dim, heads = len(lens), case["page"], case["kv"], case["dim"], case["heads"]
    cache_t = _T[case["cache"]]
    pages = [-(-m // page) for m in lens]
    n_pages = sum(pages) + 3
    width = max(pages)
    order = torch.randperm(n_pages, generator=g, device=dev, dtype=torch.int32)
    owner = torch.repeat_interleave(torch.arange(n, device=dev), torch.tensor(pages, device=dev))
    first = torch.cumsum(torch.tensor([0] + pages[:-1], device=dev), 0)
    place = torch.arange(sum(pages), device=dev) - first[owner]
    table = torch.zeros((n, width), dtype=torch.int32, device=dev)
    table[owner, place] = order[:sum(pages)]
    major = case.get("major", "pos")
    shape = (n_pages, page, kv, dim) if major == "pos" else (n_pages, kv, page, dim)

    def normal(*s, dtype):
        return torch.randn(s, generator=g, device=dev, dtype=dtype)

    st = dict(case=case, lens=lens, news=news, table=table, k=normal(*shape, dtype=cache_t), v=normal(*shape, dtype=cache_t),
              seq_len=torch.tensor(lens, dtype=torch.int32, device=dev),
              start=torch.tensor([sum(news[:i]) for i in range(n + 1)], dtype=torch.int32, device=dev))
    rows = sum(news) + case["pad"]
    st["rows"] = rows
    if case["op"] == "append":
        x_t = _T[case["x"]]
        st["qkv"] = (1.5 * normal(rows, (heads + 2 * kv) * dim, dtype=torch.float32)).to(x_t)
        st["gq"] = 1 + 0.1 * normal(dim, dtype=torch.float32) if case["norm"] else None
        st["gk"] = 1 + 0.1 * normal(dim, dtype=torch.float32) if case["norm"] else None
        half = case["rotary"] // 2
        angle = torch.arange(max(lens), device=dev, dtype=torch.float64)[:, None] * 10000.0 ** (
            -torch.arange(half, device=dev, dtype=torch.float64) / half)
        st["cos"], st["sin"] = angle.cos().float(), angle.sin().float()
        st["q_out"] = torch.zeros((rows, heads, dim), dtype=x_t, device=dev)
    else:
        st["q"] = (1.5 * normal(rows, heads, dim, dtype=torch.float32)).to(_T[case["q"]])
        st["out"] = torch.zeros((rows, heads, dim), dtype=cache_t, device=dev)
    if own:
        from paper_2504_08378_b200 import afx
        st["afx"] = afx
        s = st["k"].stride()
        kvd = afx.PagedKV(dtype=afx.DTYPES[case["cache"]], n_kv_heads=kv, head_dim=dim, page_size=page, n_pages=n_pages, n_seqs=n,
                          n_tokens=rows, max_new=max(news), page_stride=s[0], pos_stride=s[1] if major == "pos" else s[2],
                          head_stride=s[2] if major == "pos" else s[1], table_stride=width, k_pages=st["k"].data_ptr(),
                          v_pages=st["v"].data_ptr(), page_table=table.data_ptr(), seq_len=st["seq_len"].data_ptr(),
                          tok_start=st["start"].data_ptr())
        st["kv_desc"] = kvd
        if case["op"] == "append":
            st["prep"] = afx.HeadPrep(x_dtype=afx.DTYPES[case["x"]], n_heads=heads, eps=1e-5,
                                      g_q=st["gq"].data_ptr() if case["norm"] else None,
                                      g_k=st["gk"].data_ptr() if case["norm"] else None,
                                      rope_style=afx.ROPE_PAIRS if case["style"] == "pairs" else afx.ROPE_HALVES,
                                      rotary_dim=case["rotary"], rope_len=max(lens), rope_cos=st["cos"].data_ptr(),
                                      rope_sin=st["sin"].data_ptr())
        else:
            nbytes = afx.afx_paged_attn_workspace_bytes(kvd, heads)
            st["work"] = torch.empty(max(nbytes, 1), dtype=torch.uint8, device=dev)
            st["work_bytes"] = nbytes
    else:
        # the token rows' sequences and positions, which a program in torch keeps beside the lengths
        seq = [i for i in range(n) for _ in range(news[i])]
        st["seq"] = torch.tensor(seq, device=dev)
        st["pos"] = torch.tensor([lens[i] - news[i] + j for i in range(n) for j in range(news[i])], device=dev)
    return st


# ------------------------------------------------------------------------------------------- plain forms


def _rotate(u, cos, sin, style):
    half = cos.shape[-1]
    rot, rest = u[..., :2 * half], u[..., 2 * half:]
    if style == "pairs":
        a, b = rot[..., 0::2], rot[..., 1::2]
        out = torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2)
    else:
        a, b = rot[..., :half], rot[..., half:]
        out = torch.cat((a * cos - b * sin, a * sin + b * cos), -1)
    return torch.cat((out, rest), -1)


def _plain_append(st):
    case = st["case"]
    heads, kv, dim, page = case["heads"], case["kv"], case["dim"], case["page"]
    live = st["pos"].numel()
    x = st["qkv"][:live].float().view(live, heads + 2 * kv, dim)
    q, k, v = x[:, :heads], x[:, heads:heads + kv], x[:, heads + kv:]
    if case["norm"]:
        q = q * torch.rsqrt((q * q).mean(-1, keepdim=True) + 1e-5) * st["gq"]
        k = k * torch.rsqrt((k * k).mean(-1, keepdim=True) + 1e-5) * st["gk"]
    cos, sin = st["cos"][st["pos"]][:, None], st["sin"][st["pos"]][:, None]
    q, k = _rotate(q, cos, sin, case["style"]), _rotate(k, cos, sin, case["style"])
    st["q_out"][:live] = q.to(st["q_out"].dtype)
    at = st["table"][st["seq"], st["pos"] // page].long()
    st["k"][at, st["pos"] % page] = k.to(st["k"].dtype)
    st["v"][at, st["pos"] % page] = v.to(st["v"].dtype)
    return st["q_out"], st["k"], st["v"]


def _gather(cache, table, seq, pos, page, major):
    """Rows [.., kv, dim] of the cache at positions pos of sequences seq, in fp32."""
    at = table[seq, pos // page].long()
    rows = cache[at, pos % page] if major == "pos" else cache[at, :, pos % page]
    return rows.float()


def _plain_attend(st):
    case = st["case"]
    heads, kv, dim, page = case["heads"], case["kv"], case["dim"], case["page"]
    window, sinks, rep, scale = case["window"], case["sinks"], heads // kv, 1.0 / math.sqrt(dim)
    lens, news, out, dev = st["lens"], st["news"], st["out"], st["q"].device
    if max(news) <= 8:  # all sequences at once, over the positions that some new token of them sees
        seqs, top = torch.arange(len(lens), device=dev), max(news)
        first = st["seq_len"].long() - torch.tensor(news, device=dev)
        low = (first - window + 1).clamp(min=0) if window else torch.zeros_like(first)
        few = torch.minimum(low, torch.full_like(low, sinks if window else 0))
        count = few + st["seq_len"].long() - low
        i = torch.arange(int(max(l - (max(l - m - window + 1, 0) - min(sinks, max(l - m - window + 1, 0)) if window else 0)
                                 for l, m in zip(lens, news))), device=dev)[None]
        pos = torch.where(i < few[:, None], i, i - few[:, None] + low[:, None])
        pos = torch.where(i < count[:, None], pos, torch.zeros_like(pos))
        t = torch.arange(top, device=dev)[None]
        row = (st["start"][:-1].long()[:, None] + t).clamp(max=st["rows"] - 1)
        q = st["q"][row].float().view(len(lens), top, kv, rep, dim)
        qpos = (first[:, None] + t)[:, :, None]
        p = pos[:, None]
        see = (i < count[:, None])[:, None] & (p <= qpos)
        if window:
            see &= (p > qpos - window) | (p < sinks)
        keys = _gather(st["k"], st["table"], seqs[:, None], pos, page, case["major"])
        s = torch.matmul(q.permute(0, 2, 1, 3, 4).reshape(len(lens), kv, top * rep, dim), keys.permute(0, 2, 3, 1)) * scale
        del keys
        s = s.view(len(lens), kv, top, rep, -1).masked_fill(~see[:, None, :, None], float("-inf"))
        e = torch.exp(s - s.amax(-1, keepdim=True))
        vals = _gather(st["v"], st["table"], seqs[:, None], pos, page, case["major"])
        o = torch.matmul(e.view(len(lens), kv, top * rep, -1), vals.permute(0, 2, 1, 3)).view(len(lens), kv, top, rep, dim)
        o = (o / e.sum(-1, keepdim=True)).permute(0, 2, 1, 3, 4).reshape(len(lens), top, heads, dim)
        out[:st["seq"].numel()] = o[st["seq"], st["pos"] - first[st["seq"]]].to(out.dtype)
        return out
    row = 0
    for b, (length, new) in enumerate(zip(lens, news)):
        keys = vals = None
        for c in range(0, new, 1024):
            m = min(1024, new - c)
            p0 = length - new + c
            low = max(0, p0 - window + 1) if window else 0
            few = min(low, sinks) if window else 0
            pos = torch.cat((torch.arange(few, device=dev), torch.arange(low, p0 + m, device=dev)))
            keys = _gather(st["k"], st["table"], b, pos, page, case["major"]).permute(1, 2, 0)
            vals = _gather(st["v"], st["table"], b, pos, page, case["major"]).permute(1, 0, 2)
            q = st["q"][row + c:row + c + m].float().view(m, kv, rep, dim).permute(1, 2, 0, 3).reshape(kv, rep * m, dim)
            s = (torch.matmul(q, keys) * scale).view(kv, rep, m, -1)
            qpos = torch.arange(p0, p0 + m, device=dev)[:, None]
            see = pos[None] <= qpos
            if window:
                see &= (pos[None] > qpos - window) | (pos[None] < sinks)
            s = s.masked_fill(~see, float("-inf"))
            e = torch.exp(s - s.amax(-1, keepdim=True))
            o = torch.matmul(e.view(kv, rep * m, -1), vals).view(kv, rep, m, dim) / e.sum(-1, keepdim=True)
            out[row + c:row + c + m] = o.permute(2, 0, 1, 3).reshape(m, heads, dim).to(out.dtype)
        row += new
    return out


def run(st):
    case = st["case"]
    if not own:
        return _plain_append(st) if case["op"] == "append" else _plain_attend(st)
    afx, heads, kv, dim = st["afx"], case["heads"], case["kv"], case["dim"]
    if case["op"] == "append":
        x, width = st["qkv"], (heads + 2 * kv) * dim
        es = x.element_size()
        base = x.data_ptr()
        afx.afx_paged_append(st["kv_desc"], st["prep"], base, width, base + heads * dim * es, width,
                             base + (heads + kv) * dim * es, width, st["q_out"], case["x"])
        return st["q_out"], st["k"], st["v"]
    afx.afx_paged_attn(st["kv_desc"], st["q"], case["q"], heads * dim, heads, 1.0 / math.sqrt(dim), case["window"], case["sinks"],
                       st["out"], case["cache"], None, st["work"], st["work_bytes"])
    return st["out"]


def work(case):
    lens, news = _ints(case["lens"]), _ints(case["news"])
    heads, kv, dim = case["heads"], case["kv"], case["dim"]
    tokens, n = sum(news), len(lens)
    if case["op"] == "append":
        xb = 4 if case["x"] == "f32" else 2
        per = (heads + 2 * kv) * dim * xb + heads * dim * xb + 2 * kv * dim * 2 + case["rotary"] * 4
        return {"bytes": tokens * per + 8 * n, "flops": tokens * dim * (heads + kv) * (6 if not case["norm"] else 10)}
    qb = 4 if case["q"] == "f32" else 2
    window, sinks = case["window"], case["sinks"]
    rows = pairs = 0
    for length, new in zip(lens, news):
        first = length - new
        if window:
            low = max(0, first - window + 1)
            rows += length - low + min(low, sinks)
            for p in range(first, length):
                lo = max(0, p - window + 1)
                pairs += p + 1 - lo + min(lo, sinks)
        else:
            rows += length
            pairs += new * first + new * (new + 1) // 2
    return {"bytes": rows * kv * dim * 4 + tokens * heads * dim * (qb + 2) + 4 * (rows // case["page"]) + 8 * n,
            "flops": 4 * dim * heads * pairs}


# ------------------------------------------------------------------------------------------- 64 bits


def exact(case, seed):
    """The definition, token by token (appending) or block of tokens by block (attention), in 64 bits."""
    if work(case)["flops"] > 2e13:
        return None
    st = prepare(case, seed)
    lens, news = st["lens"], st["news"]
    heads, kv, dim, page = case["heads"], case["kv"], case["dim"], case["page"]
    dev = st["table"].device
    d = torch.float64
    token = 0
    if case["op"] == "append":
        q_out, kc, vc = st["q_out"].to(d), st["k"].to(d), st["v"].to(d)
        half = case["rotary"] // 2
        if case["style"] == "pairs":
            ia, ib = torch.arange(half, device=dev) * 2, torch.arange(half, device=dev) * 2 + 1
        else:
            ia, ib = torch.arange(half, device=dev), torch.arange(half, device=dev) + half

        def turned(x, gain, pos):
            if gain is not None:
                x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / dim + 1e-5) * gain.to(d)
            c, s = st["cos"].to(d)[pos][:, None], st["sin"].to(d)[pos][:, None]
            y = x.clone()
            y[..., ia] = x[..., ia] * c - x[..., ib] * s
            y[..., ib] = x[..., ib] * c + x[..., ia] * s
            return y

        for b in range(len(lens)):
            pos = torch.arange(lens[b] - news[b], lens[b], device=dev)
            x = st["qkv"][token:token + news[b]].to(d).reshape(news[b], heads + 2 * kv, dim)
            q_out[token:token + news[b]] = turned(x[:, :heads], st["gq"], pos)
            page_of, slot = st["table"][b].long()[pos // page], pos % page
            kc[page_of, slot] = turned(x[:, heads:heads + kv], st["gk"], pos)
            vc[page_of, slot] = x[:, heads + kv:]
            token += news[b]
        return q_out, kc, vc
    out = torch.zeros_like(st["out"], dtype=d)
    for b in range(len(lens)):
        every = torch.arange(lens[b], device=dev)
        where = st["table"][b].long()[every // page]
        if case["major"] == "pos":
            keys, vals = st["k"][where, every % page], st["v"][where, every % page]
        else:
            keys, vals = st["k"][where, :, every % page], st["v"][where, :, every % page]
        for t0 in range(0, news[b], 256):
            n = min(256, news[b] - t0)
            at = torch.arange(lens[b] - news[b] + t0, lens[b] - news[b] + t0 + n, device=dev)
            hidden = every[None, :] > at[:, None]
            if case["window"]:
                hidden |= (every[None, :] <= at[:, None] - case["window"]) & (every[None, :] >= case["sinks"])
            for h in range(kv):
                group = slice(h * (heads // kv), (h + 1) * (heads // kv))
                q = st["q"][token + t0:token + t0 + n, group].to(d)
                s = torch.einsum("nrd,ld->nrl", q, keys[:, h].to(d)) / math.sqrt(dim)
                w = torch.softmax(s.masked_fill(hidden[:, None], -math.inf), -1)
                out[token + t0:token + t0 + n, group] = torch.einsum("nrl,ld->nrd", w, vals[:, h].to(d))
        token += news[b]
    return out
