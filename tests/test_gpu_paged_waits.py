"""Waits of the prompts' attention that run out.  The kernel is built here with a limit that the test sets; the wait that it
cuts short is a real one: a warp that takes its rows again, because a value that they do not see is infinite."""
import ctypes
import math
import os
import subprocess

import numpy as np
import pytest
import torch

from paged_util import Problem, attention_tolerance
from paper_2504_08378_b200 import afx, build
from test_gpu_paged_attn import MARK, TORCH_MARK, attend

pytestmark = pytest.mark.gpu
HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def waits():
    src, so = os.path.join(HERE, "waits.cu"), os.path.join(HERE, "libafx_waits.so")
    inputs = [src, *build._inputs()]
    if not os.path.exists(so) or any(os.path.getmtime(p) > os.path.getmtime(so) for p in inputs):
        tmp = f"{so}.{os.getpid()}.tmp"
        subprocess.check_call([os.environ.get("NVCC", "nvcc"), *build.NVCC_FLAGS, "-I", os.path.join(build.ROOT, "include"), "-I", build.CSRC,
                               "-o", tmp, src])
        os.replace(tmp, so)
    L = ctypes.CDLL(so)
    L.waits_limit.argtypes = [ctypes.c_uint64]
    L.waits_prompt.argtypes = [ctypes.POINTER(afx.PagedKV), ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p,
                               ctypes.c_void_p]
    return L


HEADS, KV, DIM = 32, 8, 64


def problem(page):
    """More works than SMs, so that blocks take works over; one value that only the first sequence's last token sees is infinite."""
    p = Problem([40000, 700, 900, 800], [512, 700, 900, 800], HEADS, KV, DIM, page, "bf16")
    rows = p.rows_of(p.both, 0, 1).clone()
    rows[-1, :, 5] = math.inf
    p.cells(0, 1)[:] = rows
    return p


def run(L, p, q, kvd, ns):
    out = torch.full((p.rows, HEADS, DIM), MARK, dtype=torch.bfloat16, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    assert L.waits_limit(ns) == 0
    assert L.waits_prompt(kvd, q.data_ptr(), HEADS * DIM, HEADS, out.data_ptr(), None, status.data_ptr()) == 0
    torch.cuda.synchronize()
    return out.cpu(), status.item()


@pytest.mark.parametrize("page", [64, 24])
def test_a_wait_that_runs_out_is_reported_and_the_gpu_goes_on(waits, page):
    p = problem(page)
    q = p.randn(p.rows, HEADS, DIM, dtype="bf16").cuda()
    kvd = p.upload(afx)
    out, status = run(waits, p, q, kvd, 1)
    assert status == 6  # AFX_ERR_TIMEOUT
    whole, _ = attend(p, q.cpu(), kvd, "bf16", "bf16")
    # what was written is right, rows that were not are as they were
    stayed = (out == TORCH_MARK["bf16"]).all(2)
    assert stayed.any() and not stayed.all()
    same = torch.where(torch.isnan(whole), torch.isnan(out), out == whole).all(2)
    assert (stayed | same).all()
    again, status = run(waits, p, q, kvd, 2 * 10 ** 9)
    assert status == 0 and torch.equal(again.view(torch.int16), whole.view(torch.int16))


def test_rows_that_are_taken_again_keep_the_others_waiting(waits):
    """The first sequence's rows are taken again for longer than the limit, while blocks hold works of the other sequences:
    nobody gives up, and every row is right."""
    p = problem(64)
    q = p.randn(p.rows, HEADS, DIM, dtype="bf16").cuda()
    kvd = p.upload(afx)
    whole, _ = attend(p, q.cpu(), kvd, "bf16", "bf16")
    try:
        assert waits.waits_tell_every(1024) == 0
        out, status = run(waits, p, q, kvd, 5 * 10 ** 6)
    finally:
        assert waits.waits_tell_every(0x7FFFFFFF) == 0
    assert status == 0
    assert torch.equal(out.view(torch.int16), whole.view(torch.int16))
    # the rows in front of the infinite value, and those of the other sequences, by the definition
    rows = p.rows_of(p.both, 0, 1).clone()
    rows[-1, :, 5] = 0
    p.cells(0, 1)[:] = rows
    some = [0, 300, 505, 510]
    K, V = (p.rows_of(p.both, 0, c).double() for c in (0, 1))
    for i in some:
        pos = 40000 - 512 + i
        for h in (0, 5, 31):
            k, v = K[:pos + 1, h // 4], V[:pos + 1, h // 4]
            s = k @ q[i, h].double().cpu() / 8
            w = torch.softmax(s, 0)
            size = (k.abs() @ q[i, h].double().cpu().abs()).max().item() / 8
            tol = attention_tolerance((w @ v).numpy(), (w @ v.abs()).numpy(), np.float64(size), DIM, "bf16", "bf16")
            assert (np.abs(out[i, h].double().numpy() - (w @ v).numpy()) <= tol).all()
    assert torch.isposinf(out[511, :, 5]).all() and torch.isfinite(out[:511]).all() and torch.isfinite(out[512:]).all()
