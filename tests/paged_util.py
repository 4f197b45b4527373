"""A paged key-value cache on the CPU, in 64 bits: what the operators have to read and write, written from their
definitions, and the bounds of what 32-bit sums and one rounding may be off by."""
import math

import numpy as np
import torch

TORCH = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
HALF_STEP = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8, "f32": 2.0 ** -24}  # half a step, relative to the value
TINY = {"f16": 2.0 ** -25, "bf16": 2.0 ** -134, "f32": 2.0 ** -150}    # half a step of the subnormals


class Problem:
    """Sequences of ``lens`` positions, the last ``news`` of them new, over shuffled pages.  Every cell of the pool
    that belongs to no position holds NaN."""

    def __init__(self, lens, news, heads, kv, dim, page, cache="f16", major="pos", interleaved=False, pad=0, seed=0,
                 spare=2, filled=True):
        self.lens, self.news, self.heads, self.kv, self.dim, self.page = list(lens), list(news), heads, kv, dim, page
        self.cache, self.major, self.pad = cache, major, pad
        g = self.g = torch.Generator().manual_seed(seed)
        n_pages = [-(-n // page) for n in lens]
        self.n_pages = sum(n_pages) + spare
        self.width = max(n_pages + [1])
        order = torch.randperm(self.n_pages, generator=g).to(torch.int32)
        self.table = torch.full((len(lens), self.width), -1, dtype=torch.int32)
        at = 0
        for b, n in enumerate(n_pages):
            self.table[b, :n] = order[at:at + n]
            at += n
        shape = (self.n_pages, page, kv, dim) if major == "pos" else (self.n_pages, kv, page, dim)
        both = torch.full((self.n_pages, 2, *shape[1:]), math.nan, dtype=TORCH[cache])
        if not interleaved:
            both = torch.full((2, *shape), math.nan, dtype=TORCH[cache]).transpose(0, 1)
        self.both = both
        self.rows = sum(self.news) + pad
        if filled:
            for b, n in enumerate(lens):
                for c in range(2):
                    self.cells(b, c)[:] = torch.randn((n, kv, dim), generator=g)

    def cells(self, b, which):
        """Writable view-like access to sequence b's rows [position][kv][dim] of K (0) or V (1)."""
        return _Cells(self, b, which)

    def rows_of(self, both, b, which, n=None):
        p = torch.arange(self.lens[b] if n is None else n)
        page, slot = self.table[b, p // self.page].long(), p % self.page
        x = both[:, which]
        return x[page, slot] if self.major == "pos" else x[page, :, slot]

    def randn(self, *shape, dtype="f32", scale=1.0):
        return (scale * torch.randn(shape, generator=self.g)).to(TORCH[dtype])

    def start(self):
        return torch.tensor([sum(self.news[:i]) for i in range(len(self.news) + 1)], dtype=torch.int32)

    # ---- on the device

    def upload(self, afx, max_new=None, start=True):
        dev = "cuda"
        self.d_both = self.both.to(dev)
        # (a copy keeps neither layout: lay the pool out as on the host)
        if self.both.stride() != self.d_both.stride():
            self.d_both = torch.empty_strided(self.both.shape, self.both.stride(), dtype=self.both.dtype, device=dev)
            self.d_both.copy_(self.both.to(dev))
        self.d_table, self.d_len = self.table.to(dev), torch.tensor(self.lens, dtype=torch.int32, device=dev)
        self.d_start = self.start().to(dev) if start else None
        s = self.both.stride()
        return afx.PagedKV(dtype=afx.DTYPES[self.cache], n_kv_heads=self.kv, head_dim=self.dim, page_size=self.page,
                           n_pages=self.n_pages, n_seqs=len(self.lens), n_tokens=self.rows,
                           max_new=max_new or max(self.news + [1]), page_stride=s[0],
                           pos_stride=s[2] if self.major == "pos" else s[3], head_stride=s[3] if self.major == "pos" else s[2],
                           table_stride=self.width, k_pages=self.d_both[:, 0].data_ptr(), v_pages=self.d_both[:, 1].data_ptr(),
                           page_table=self.d_table.data_ptr(), seq_len=self.d_len.data_ptr(),
                           tok_start=self.d_start.data_ptr() if start else None)

    # ---- definitions in 64 bits

    def attend(self, q, window=0, sinks=0, scale=None, both=None):
        """(out, lse, sum of w |v|, largest sum of |q_i k_i| times the scale) per token row and head; NaN in padded rows."""
        both = self.both if both is None else both
        scale = 1 / math.sqrt(self.dim) if scale is None else scale
        rep = self.heads // self.kv
        shape = (self.rows, self.heads)
        out, mass = np.full((*shape, self.dim), np.nan), np.full((*shape, self.dim), np.nan)
        lse, size = np.full(shape, np.nan), np.zeros(shape)
        q = q.double().numpy()
        row = 0
        for b, (n, new) in enumerate(zip(self.lens, self.news)):
            K, V = (self.rows_of(both, b, c).double().numpy() for c in (0, 1))
            for i in range(new):
                p = n - new + i
                j = np.arange(n)
                see = j <= p
                if window:
                    see &= (j > p - window) | (j < sinks)
                for h in range(self.heads):
                    k, v = K[see, h // rep], V[see, h // rep]
                    if not len(k):
                        out[row, h], mass[row, h], lse[row, h] = 0, 0, -np.inf
                        continue
                    s = k @ q[row, h] * scale
                    w = np.exp(s - s.max())
                    lse[row, h] = s.max() + np.log(w.sum())
                    w /= w.sum()
                    out[row, h], mass[row, h] = w @ v, w @ np.abs(v)
                    size[row, h] = (np.abs(k) @ np.abs(q[row, h])).max() * abs(scale)
                row += 1
        return out, lse, mass, size


class _Cells:
    def __init__(self, prob, b, which):
        self.a = (prob, b, which)

    def __setitem__(self, key, value):
        prob, b, which = self.a
        p = torch.arange(prob.lens[b])[key]
        page, slot = prob.table[b, p // prob.page].long(), p % prob.page
        x = prob.both[:, which]
        value = value.to(x.dtype) if torch.is_tensor(value) else value
        if prob.major == "pos":
            x[page, slot] = value
        else:
            x[page, :, slot] = value


def attention_tolerance(out, mass, size, dim, out_type, weight_type=None):
    """A score is a sum of dim exact products in fp32 (each addition off by at most 2^-23 of the sum of magnitudes,
    where the hardware truncates), times a scale, off by a rounding or two; its error is the relative error of its
    weight, as are 2^-21 of the exponential and 2^-20 of the sums of weights (fixed chunks: short chains of fp32 additions).  Numerator and
    denominator: twice.  Weights that are rounded to 16 bits before they multiply the values: half a step of those.  The output is rounded once."""
    weights = 2 * ((dim + 4) * 2.0 ** -23 * size + 2.0 ** -20)[..., None]
    if weight_type is not None:
        weights = weights + HALF_STEP[weight_type]
    return HALF_STEP[out_type] * np.abs(out) + TINY[out_type] + 1.01 * weights * mass


def rope_table(n, rotary, theta=10000.0):
    half = rotary // 2
    ang = torch.arange(n, dtype=torch.float64)[:, None] * theta ** (-torch.arange(half, dtype=torch.float64) / max(half, 1))
    return ang.cos().float(), ang.sin().float()


def turn(x, gain, eps, cos, sin, style):
    """Norm and rotation of heads [rows][heads][dim] in 64 bits; and the size of what the rotation adds up."""
    x = x.double()
    if gain is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * gain.double()
    half = cos.shape[-1]
    i = torch.arange(half)
    ia, ib = (2 * i, 2 * i + 1) if style == "pairs" else (i, i + half)
    c, s = cos.double()[:, None], sin.double()[:, None]
    y, size = x.clone(), x.abs()
    y[..., ia] = x[..., ia] * c - x[..., ib] * s
    y[..., ib] = x[..., ib] * c + x[..., ia] * s
    size[..., ia] = size[..., ib] = x[..., ia].abs() + x[..., ib].abs()
    return y, size
