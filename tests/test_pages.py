"""Refusals of the operators on 4-bit pages, sizes and launch plans: host code only, nothing is launched."""
import ctypes as C
import math
import os
import subprocess

import numpy as np
import pytest
import torch

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


@pytest.mark.parametrize("scaling", ["linear", "wave", "index"])
def test_rope_refuses_angles_beyond_its_reduction(lib, scaling):
    """Positions times frequencies over a tiny factor would leave the range that the sines are reduced from."""
    for factor in (2.0 ** -17, 1e-30, -1.0, math.nan, math.inf):
        r = M.Rope("half", 64, scaling=scaling, factor=factor)
        refused(lib, lib.metasd_rope_append(C.byref(r.c), C.byref(pages()), 0, 4, 2, OK, 128, OK, 128, OK, 128, OK, 128, OK, OK, None), "factor")


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


def test_wrappers_refuse_what_is_missing():
    q, i = torch.zeros(2, 4, 64), torch.zeros(2, dtype=torch.int32)
    pool = torch.zeros(4, M.page_bytes(2, 64, 16), dtype=torch.uint8)
    for args in ((None, None, None, i, i, pool), (None, q, None, i, i, pool), (q, q, q, i, None, pool), (q, q, q, i, i, None)):
        with pytest.raises(ValueError, match="k with v, slots and pool"):
            M.rope_append(*args, 16, 2, 64, M.Rope())
    for call in (lambda: M.rope_append(q, None, None, i, None, None, 16, 2, 64, M.Rope()), lambda: M.kv_rows(pool, i, 16, 2, 64),
                 lambda: M.attn_pages(q, pool, i.reshape(2, 1), i, i, 16, 2, 0.1, 1, 16), lambda: M.page_plan(i.reshape(2, 1), i, i, i, i, i, 16, 2),
                 lambda: M.accept_probs(torch.zeros(2, 2, 8), None, i.reshape(2, 1), None, torch.zeros(2, 1), torch.zeros(2))):
        with pytest.raises(ValueError, match="no CPU fallback"):
            call()


PLAN_SRC = '''#include "pages_plan.h"
extern "C" void plan(int B, int KH, int G, int hd, int max_new, int max_len, int terms, int n_cu, size_t limit, long* o) {
    const msd::PagesPlan p = msd::plan_pages(B, KH, G, hd, max_new, max_len, terms, n_cu, limit);
    const long x[] = {p.wide, p.ct, p.pack, p.cols, p.nw, p.ncg, p.spw, p.nsp, (long)msd::pages_records(p, B, KH, hd)};
    for (int i = 0; i < 9; ++i) o[i] = x[i];
}'''


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("pages_plan")
    (d / "p.cpp").write_text(PLAN_SRC)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2604_05417_amd", "csrc"), "-o", str(d / "p.so"), str(d / "p.cpp")], check=True)
    f = C.CDLL(str(d / "p.so")).plan
    f.argtypes = [C.c_int] * 8 + [C.c_size_t, C.POINTER(C.c_long)]

    def call(*a, n_cu=256, limit=2 ** 63):
        o = (C.c_long * 9)()
        f(*a, n_cu, limit, o)
        return dict(zip(("wide", "ct", "pack", "cols", "nw", "ncg", "spw", "nsp", "records"), o))
    return call


@pytest.mark.parametrize("terms", [1, 3])
@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("B,KH,G", [(1, 1, 1), (1, 32, 1), (24, 8, 4), (3, 2, 8), (1, 1, 256), (4096, 8, 1), (4096, 1024, 1), (65535, 64, 1)])
def test_attention_plan(plan, B, KH, G, hd, terms):
    """Every column and every position has its workgroup, a launch holds the grid, and records stay within the room that there is."""
    for max_new in (1, 2, 3, 7, 16, 17, 200, 1000, 1 << 20):
        if B * KH * G * max_new > 1 << 26:
            continue
        for max_len in (1, 31, 33, 500, 513, 4000, 100001, 2 ** 31 - 1):
            for n_cu in (256, 64, 1):
                p = plan(B, KH, G, hd, max_new, max_len, terms, n_cu=n_cu)
                nsub = max(1, (max_len + 31) // 32)
                assert p["cols"] == (64 if p["wide"] else 16 * p["ct"] // p["pack"]) and p["ncg"] * p["cols"] >= max_new * G > (p["ncg"] - 1) * p["cols"]
                assert p["nsp"] * p["spw"] >= nsub > (p["nsp"] - 1) * p["spw"] and p["spw"] % (2 if p["wide"] else p["nw"]) == 0
                assert p["pack"] == 1 or (terms == 3 and max_new * G <= 16 // p["pack"])
                assert p["nw"] == 4 or p["nsp"] == 1
                units = -(-B * KH // 8) * 8 if p["wide"] else B * KH
                assert units * p["ncg"] * p["nsp"] * 64 * p["nw"] < 1 << 32
                assert p["records"] == (0 if p["nsp"] == 1 else B * KH * p["ncg"] * p["nsp"] * p["cols"] * (hd + 4))
                for limit in (0, p["records"] // 2, p["records"]):
                    r = plan(B, KH, G, hd, max_new, max_len, terms, n_cu=n_cu, limit=limit)
                    assert r["records"] <= limit and r["nsp"] * r["spw"] >= nsub
                    assert limit < p["records"] or r == p


@pytest.mark.parametrize("ncg,nsp", [(5, 1), (24, 1), (63, 1), (24, 3), (7, 16), (600, 1)])
def test_order_of_long_blocks(ncg, nsp):
    """The order that attn_pages_long_kernel gives its workgroups, written out: every (pair, column group, span) once."""
    for units in (1, 2, 4, 5, 40, 130):
        per, seen = ncg * nsp, set()
        most = min(units, (511 + per) // per)
        for y in range(units * per):
            bundle = y // (most * per)
            n_units, z = min(most, units - bundle * most), y - bundle * most * per
            rnd = z >> 5
            place = min(32 * rnd + 31, n_units * per - 1) - (z & 31) if rnd & 1 else z
            seen.add((bundle * most + place // nsp % n_units, ncg - 1 - place // (nsp * n_units), place % nsp))
        assert seen == {(u, c, s) for u in range(units) for c in range(ncg) for s in range(nsp)}


def test_reference_quantiser():
    """The rules in small: the scale's border at 7, ties to the even code, saturation at 6."""
    assert [R.scale_exponent(a) for a in (7.0, np.nextafter(7.0, 8.0), 3.5, 3.6, 1e-300, 1e300)] == [0, 1, -1, 0, -125, 125]
    assert [R.GRID[R.nearest_code(a)] for a in (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0)] == [0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, 6.0]
    x = np.zeros(32)
    x[:3] = 6.9, -0.3, 0.2
    assert R.quantise(x)[0][:3].tolist() == [6.0, -0.5, 0.0]
