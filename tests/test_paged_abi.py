"""The paged cache's entry points refuse bad arguments on the host; their descriptors have the header's layout."""
import ctypes
import os
import re
import subprocess

import pytest

from paper_2504_08378_b200 import afx

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 1 << 20  # aligned, never dereferenced on the host


def desc(**kw):
    d = dict(dtype=0, n_kv_heads=8, head_dim=128, page_size=16, n_pages=100, n_seqs=4, n_tokens=4, max_new=1,
             page_stride=16 * 8 * 128, pos_stride=8 * 128, head_stride=128, table_stride=32, k_pages=FAKE, v_pages=FAKE,
             page_table=FAKE, seq_len=FAKE, tok_start=None)
    d.update(kw)
    return afx.PagedKV(**d)


def prep(**kw):
    d = dict(x_dtype=1, n_heads=32, eps=1e-5, rope_style=1, rotary_dim=128, rope_len=512, g_q=FAKE, g_k=FAKE, rope_cos=FAKE,
             rope_sin=FAKE)
    d.update(kw)
    return afx.HeadPrep(**d)


def status(fn, *a, **kw):
    try:
        fn(*a, stream=0, **kw)
    except afx.AfxError as e:
        return e.status
    return 0


def append(kv=None, p=None, q=FAKE, ldq=32 * 128, k=FAKE, ldk=8 * 128, v=FAKE, ldv=8 * 128, q_out=FAKE + 4096, q_type=1, **kw):
    return status(afx.afx_paged_append, kv or desc(), p or prep(), q, ldq, k, ldk, v, ldv, q_out, q_type, **kw)


def attn(kv=None, q=FAKE, q_type=0, ldq=32 * 128, heads=32, scale=0.0, window=0, sinks=0, out=FAKE, out_type=0, lse=None,
         ws=FAKE, ws_bytes=1 << 40, **kw):
    return status(afx.afx_paged_attn, kv or desc(), q, q_type, ldq, heads, scale, window, sinks, out, out_type, lse, ws, ws_bytes, **kw)


BAD_DESC = [(dict(dtype=2), 4), (dict(dtype=9), 4), (dict(head_dim=96), 4), (dict(head_dim=256), 4), (dict(n_kv_heads=0), 1), (dict(page_size=0), 1),
            (dict(n_pages=0), 1), (dict(n_seqs=-1), 1), (dict(n_tokens=-1), 1), (dict(max_new=0), 1), (dict(table_stride=0), 1),
            (dict(n_seqs=70000, n_tokens=70000), 3), (dict(page_size=(1 << 20) + 1), 3), (dict(n_tokens=(1 << 24) + 1), 3),
            (dict(k_pages=None), 1), (dict(v_pages=None), 1), (dict(page_table=None), 1), (dict(seq_len=None), 1),
            (dict(max_new=2), 1), (dict(n_tokens=3), 1), (dict(pos_stride=120), 1), (dict(head_stride=64), 1), (dict(page_stride=0), 1),
            (dict(pos_stride=1028), 2), (dict(head_stride=132), 2), (dict(page_stride=16 * 1024 + 4), 2), (dict(k_pages=FAKE + 8), 2),
            (dict(v_pages=FAKE + 2), 2), (dict(page_table=FAKE + 2), 2), (dict(seq_len=FAKE + 1), 2),
            (dict(tok_start=FAKE + 2), 2)]


@pytest.mark.parametrize("bad,code", BAD_DESC)
def test_bad_descriptors(bad, code):
    assert append(desc(**bad)) == code
    assert attn(desc(**bad)) == code
    if code != 2:
        assert afx.afx_paged_attn_workspace_bytes(desc(**bad), 32) == 0


def test_append_refusals():
    for name in ("k", "v", "q_out"):
        assert append(**{name: None}) == 1
    assert append(q=None) == 1
    assert append(p=prep(x_dtype=3)) == 4 and append(q_type=5) == 4 and append(p=prep(rope_style=3)) == 4
    assert append(p=prep(n_heads=12)) == 1 and append(p=prep(n_heads=0)) == 1
    assert append(p=prep(eps=-1.0)) == 1 and append(p=prep(eps=float("nan"))) == 1
    assert append(ldq=32 * 128 - 8) == 1 and append(ldk=8) == 1 and append(ldv=8) == 1
    assert append(p=prep(rotary_dim=136)) == 1 and append(p=prep(rotary_dim=-16)) == 1 and append(p=prep(rope_len=0)) == 1
    assert append(p=prep(rope_cos=None)) == 1 and append(p=prep(rope_sin=None)) == 1
    assert append(p=prep(rotary_dim=24)) == 2 and append(p=prep(rope_cos=FAKE + 4)) == 2 and append(p=prep(g_q=FAKE + 4)) == 2
    assert append(ldq=32 * 128 + 4) == 2 and append(ldk=8 * 128 + 1) == 2 and append(q=FAKE + 8) == 2 and append(k=FAKE + 2) == 2
    assert append(q_out=FAKE + 4) == 2 and append(dev_status=FAKE + 1) == 2
    # in place only row upon row, in one type
    assert append(q_out=FAKE, ldq=33 * 128) == 1 and append(q_out=FAKE, q_type=0) == 1
    with pytest.raises(afx.AfxError):
        afx._check("afx_paged_append", afx.lib().afx_paged_append(None, None, FAKE, 4096, FAKE, 1024, FAKE, 1024, FAKE, 0, None, 0))


def test_attention_refusals():
    for name in ("q", "out"):
        assert attn(**{name: None}) == 1
    assert attn(heads=12) == 1 and attn(heads=0) == 1 and attn(heads=8 * 2000) == 3 or attn(heads=8 * 2000, ldq=8 * 2000 * 128) == 3
    assert attn(window=-1) == 1 and attn(sinks=-1) == 1 and attn(scale=float("nan")) == 1 and attn(ldq=128) == 1
    assert attn(q_type=1) == 4 and attn(out_type=2) == 4 and attn(out_type=7) == 4
    assert attn(desc(max_new=9, tok_start=FAKE, n_tokens=36), q_type=2) == 4  # fp32 queries of more than a few tokens
    assert attn(ldq=32 * 128 + 4) == 2 and attn(q=FAKE + 8) == 2 and attn(out=FAKE + 8) == 2 and attn(lse=FAKE + 2) == 2
    assert attn(ws=FAKE + 16) == 2 and attn(dev_status=FAKE + 2) == 2


def test_nothing_to_do_is_no_error():
    assert append(desc(n_seqs=0, n_tokens=0)) == 0 and attn(desc(n_seqs=0, n_tokens=0)) == 0
    assert append(desc(n_seqs=0, n_tokens=9)) == 0 and attn(desc(n_tokens=0, tok_start=FAKE)) == 0


def test_descriptors_have_the_headers_layout(tmp_path):
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "afx.h"', "int main(void) {"]
    pairs = {"afx_paged_kv": afx.PagedKV, "afx_head_prep": afx.HeadPrep}
    for c, cls in pairs.items():
        lines.append(f'  printf("{c} %zu", sizeof({c}));')
        lines += [f'  printf(" %zu", offsetof({c}, {n}));' for n, _ in cls._fields_]
        lines.append('  printf("\\n");')
    src = tmp_path / "layout.c"
    src.write_text("\n".join(lines + ["  return 0;", "}"]))
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), "-o", str(tmp_path / "layout"), str(src)])
    for ln in subprocess.check_output([str(tmp_path / "layout")], text=True).splitlines():
        c, size, *offs = ln.split()
        assert ctypes.sizeof(pairs[c]) == int(size)
        assert [getattr(pairs[c], n).offset for n, _ in pairs[c]._fields_] == [int(o) for o in offs]
    hdr = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "afx.h")).read(), flags=re.S)
    for c, cls in pairs.items():  # no field of the header is missing in the binding
        body = re.search(r"typedef struct \{([^}]*)\}\s*" + c + r"\s*;", hdr).group(1)
        names = [re.search(r"(\w+)\s*$", part).group(1) for decl in body.split(";") if decl.strip() for part in decl.split(",")]
        assert names == [n for n, _ in cls._fields_]


def test_counts_of_query_heads_are_checked_one_by_one():
    assert attn(heads=12) == 1
    assert attn(heads=0) == 1
    assert attn(heads=-8) == 1
    assert attn(heads=16000, ldq=16000 * 128) == 3
    assert attn(desc(n_seqs=1, n_tokens=1 << 23, max_new=1 << 23, tok_start=FAKE), heads=512, ldq=512 * 128) == 3  # rows times heads
