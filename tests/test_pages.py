"""Refusals of the operators on 4-bit pages, sizes and launch plans: host code only, nothing is launched."""
import ctypes as C
import math
import os
import subprocess

import numpy as np
import pytest

import pages_ref as R
import paper_2604_05417_amd as M
from paper_2604_05417_amd import binding as B
from paper_2604_05417_amd.build import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK = 1 << 20      # an aligned address that nothing is read from


@pytest.fixture(scope="module")
def lib():
    build(force=False)
    return M.load_library()


def pages(**kw):
    d = dict(n_kv_heads=2, head_dim=64, page=16, n_pages=4, pool=OK, page_stride=2 * 17 * 64)
    d.update(kw)
    return B._Pages(*[d[k] for k in ("n_kv_heads", "head_dim", "page", "n_pages", "pool", "page_stride")])


def refused(lib, rc, text):
    assert rc in (-1, -5) and text.encode() in lib.metasd_last_error(None), lib.metasd_last_error(None)


def test_page_bytes(lib):
    assert M.page_bytes(32, 128, 64) == 32 * 64 * 128 * 2 * 17 // 32      # 4.25 bits per value
    assert M.page_bytes(1, 32, 16) == 17 * 32
    for bad in ((0, 64, 16), (1, 48, 16), (1, 64, 24), (1, 64, 8), (1, 64, 2048)):
        with pytest.raises(M.MetaSDError):
            M.page_bytes(*bad)


@pytest.mark.parametrize("kw,text", [(dict(batch=0), "batch"), (dict(batch=4097), "batch"), (dict(width=0), "width"), (dict(batch=4096, width=1 << 20), "31 bits"), (dict(page=17), "power of two"),
                                     (dict(n_pages=0), "n_pages"), (dict(n_pages=1 << 27), "31 bits"), (dict(rows=-1), "rows"), (dict(null=5), "NULL"), (dict(null=6), "NULL")])
def test_plan_refusals(lib, kw, text):
    a = dict(batch=2, width=4, n_pages=8, page=16, rows=8, null=None)
    a.update(kw)
    p = [OK] * 10
    if a["null"] is not None:
        p[a["null"]] = None
    refused(lib, lib.metasd_page_plan(p[0], a["batch"], a["width"], p[1], p[2], a["n_pages"], p[3], p[4], p[5], a["page"], a["rows"], p[6], p[7], p[8], p[9], None), text)


PAGE_REFUSALS = [(dict(head_dim=96), "head_dim"), (dict(page=8), "page"), (dict(n_kv_heads=0), "n_kv_heads"), (dict(pool=None), "pool"), (dict(pool=OK + 8), "16-byte"),
                 (dict(n_pages=0), "n_pages"), (dict(n_pages=1 << 28), "31 bits"), (dict(page_stride=2 * 17 * 64 - 16), "page_stride"), (dict(page_stride=2 * 17 * 64 + 8), "page_stride")]


@pytest.mark.parametrize("kw,text", PAGE_REFUSALS)
def test_bad_pages_are_refused(lib, kw, text):
    p = pages(**kw)
    r = M.Rope("half", 64)
    refused(lib, lib.metasd_rope_append(C.byref(r.c), C.byref(p), 0, 4, 2, OK, 128, OK, 128, OK, 128, OK, 128, OK, OK, None), text)
    refused(lib, lib.metasd_kv_rows(C.byref(p), OK, 4, 0, OK, OK, None), text)
    refused(lib, lib.metasd_attn_pages(C.byref(p), 0, 4, 2, OK, 128, 2 * OK, 128, OK, 2, 3, OK, OK, 4, 40, 1.0, OK, 1 << 30, None), text)


@pytest.mark.parametrize("kw,text", [(dict(q=None), "NULL"), (dict(v=None), "NULL"), (dict(slots=None), "NULL"), (dict(pos=None), "NULL"), (dict(q=None, q_out=None, k=None, v=None), "NULL"),
                                     (dict(dtype=2), "dtype"), (dict(rows=0), "rows"), (dict(H=0), "n_heads"), (dict(q=OK + 4), "rows of q"), (dict(q_ld=127), "rows of q"),
                                     (dict(q_ld=130), "rows of q"), (dict(q_out_ld=64), "rows of q_out"), (dict(k=OK + 8), "rows of k"), (dict(v_ld=64), "rows of v"),
                                     (dict(rows=(1 << 22) + 1), "rows"), (dict(q_out_ld=256), "rows of q_out")])
def test_append_refusals(lib, kw, text):
    a = dict(dtype=0, rows=4, H=2, q=OK, q_ld=128, q_out=OK, q_out_ld=128, k=OK, k_ld=128, v=OK, v_ld=128, pos=OK, slots=OK)
    a.update(kw)
    refused(lib, lib.metasd_rope_append(C.byref(M.Rope("half", 64).c), C.byref(pages()), a["dtype"], a["rows"], a["H"], a["q"], a["q_ld"], a["q_out"], a["q_out_ld"], a["k"], a["k_ld"],
                                        a["v"], a["v_ld"], a["pos"], a["slots"], None), text)


@pytest.mark.parametrize("kw,text", [(dict(rot_dim=7), "rot_dim"), (dict(rot_dim=66), "rot_dim"), (dict(rot_dim=-2), "rot_dim"), (dict(theta=1.0), "theta"), (dict(theta=math.nan), "theta"),
                                     (dict(gain=0.0), "gain"), (dict(gain=math.inf), "gain"), (dict(scaling="linear", factor=0.0), "factor"), (dict(scaling="wave", low=4.0), "low"),
                                     (dict(scaling="index", orig_ctx=0), "orig_ctx"), (dict(scaling="index", low=0.0), "low")])
def test_rope_refusals(lib, kw, text):
    r = M.Rope(**{**dict(style="half", rot_dim=64), **kw})
    refused(lib, lib.metasd_rope_append(C.byref(r.c), C.byref(pages()), 0, 4, 2, OK, 128, OK, 128, OK, 128, OK, 128, OK, OK, None), text)
    for field, value in (("style", 2), ("scaling", 4)):
        r = M.Rope("half", 64)
        setattr(r.c, field, value)
        refused(lib, lib.metasd_rope_append(C.byref(r.c), C.byref(pages()), 0, 4, 2, OK, 128, OK, 128, OK, 128, OK, 128, OK, OK, None), field)


@pytest.mark.parametrize("kw,text", [(dict(q=None), "NULL"), (dict(lens=None), "NULL"), (dict(dtype=3), "dtype"), (dict(rows=0), "rows"), (dict(H=3), "n_heads"), (dict(batch=0), "batch"),
                                     (dict(batch=65536), "batch"), (dict(width=0), "width"), (dict(width=1 << 28), "31 bits"), (dict(max_new=0), "max_new"), (dict(max_len=0), "max_len"),
                                     (dict(scale=0.0), "scale"), (dict(scale=math.nan), "scale"), (dict(q_ld=129), "rows of q"), (dict(out=OK + 4), "rows of out"), (dict(out=OK), "which is q"),
                                     (dict(rows=(1 << 22) + 1), "rows"), (dict(batch=65535, max_new=1 << 14), "one launch")])
def test_attention_refusals(lib, kw, text):
    a = dict(dtype=0, rows=4, H=2, q=OK, q_ld=128, out=2 * OK, out_ld=128, table=OK, batch=2, width=3, start=OK, lens=OK, max_new=2, max_len=40, scale=1.0)
    a.update(kw)
    refused(lib, lib.metasd_attn_pages(C.byref(pages()), a["dtype"], a["rows"], a["H"], a["q"], a["q_ld"], a["out"], a["out_ld"], a["table"], a["batch"], a["width"], a["start"], a["lens"],
                                       a["max_new"], a["max_len"], a["scale"], OK, 1 << 30, None), text)


@pytest.mark.parametrize("kw,text", [(dict(P=None), "NULL"), (dict(w=None), "NULL"), (dict(rows=0), "rows"), (dict(rows=(1 << 24) + 1), "rows"), (dict(gamma=0), "gamma"),
                                     (dict(gamma=1025), "gamma"), (dict(V=0), "V 1"), (dict(V=(1 << 20) + 1), "V 1"), (dict(p_pos=99), "overlap"), (dict(q_row=5), "overlap")])
def test_accept_refusals(lib, kw, text):
    a = dict(P=OK, p_row=400, p_pos=100, Q=OK, q_row=300, q_pos=100, d=OK, n=OK, u=OK, w=OK, rows=2, gamma=3, V=100)
    a.update(kw)
    refused(lib, lib.metasd_accept_probs(a["P"], a["p_row"], a["p_pos"], a["Q"], a["q_row"], a["q_pos"], a["d"], a["n"], a["u"], a["w"], a["rows"], a["gamma"], a["V"], OK, OK, None), text)


def test_reference_quantiser():
    """The rules in small: the scale's border at 7, ties to the even code, saturation at 6."""
    assert [R.scale_exponent(a) for a in (7.0, np.nextafter(7.0, 8.0), 3.5, 3.6, 1e-300, 1e300)] == [0, 1, -1, 0, -125, 125]
    assert [R.GRID[R.nearest_code(a)] for a in (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0)] == [0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, 6.0]
    x = np.zeros(32)
    x[:3] = 6.9, -0.3, 0.2
    assert R.quantise(x)[0][:3].tolist() == [6.0, -0.5, 0.0]
