"""Operators on 4-bit pages against a plain 64-bit reference (pages_ref.py, where the tolerances are derived)."""
import math

import numpy as np
import pytest
import torch

import pages_ref as R

pytestmark = pytest.mark.gpu

M = pytest.importorskip("paper_2604_05417_amd")
DEV = "cuda:0"


def dev(x, dt=torch.int32):
    return torch.as_tensor(np.asarray(x)).to(dt).to(DEV)


# ---- block tables and slots

def plan_state(rng, B, width, n_pages, page, held=None):
    held = np.zeros(B, np.int64) if held is None else np.asarray(held, np.int64)
    ids = rng.permutation(n_pages)
    table = np.full((B, width), -7, np.int64)
    k = 0
    for b in range(B):
        table[b, :held[b]] = ids[k:k + held[b]]
        k += held[b]
    head = int(rng.integers(0, n_pages))
    ring = np.full(n_pages, -9, np.int64)
    ring[(head + np.arange(n_pages - k)) % n_pages] = ids[k:]
    return table, held, ring, np.array([head, n_pages - k, 0, 0], np.int64)


def check_plan(g, h, lens, n_new, page, rows):
    """One call on the device arrays g and on the host arrays h (table, held, ring, state)."""
    out = M.page_plan(*g, dev(lens), dev(n_new), page, rows)
    want = R.page_plan(*h, np.asarray(lens, np.int64), np.asarray(n_new, np.int64), page, rows)
    for name, w in zip(("slots", "pos", "start", "served"), want):
        assert np.array_equal(out[name].cpu().numpy(), w), name
    for name, a, b in zip(("table", "held", "ring", "state"), g, h):
        assert np.array_equal(a.cpu().numpy(), b), name
    return out


@pytest.mark.parametrize("B,page,width,n_pages,most", [(1, 16, 8, 8, 40), (3, 16, 6, 30, 30), (33, 32, 5, 120, 90), (64, 64, 40, 4000, 1500), (300, 16, 12, 2500, 120),
                                                       (1025, 16, 3, 3075, 30), (4096, 128, 2, 6000, 200)])
def test_plan_rounds(B, page, width, n_pages, most):
    """Rounds of growing, shrinking, ending and starting requests on one pool, which runs empty in some of them."""
    rng = np.random.default_rng(B)
    h = plan_state(rng, B, width, n_pages, page)
    g = [dev(x) for x in h]
    lens = np.zeros(B, np.int64)
    for step in range(6):
        n_new = rng.integers(0, most, B) * (rng.random(B) < 0.8)
        total = int(n_new.sum())
        rows = max(1, total + int(rng.integers(-3, 60)) if step % 2 else total)
        check_plan(g, h, lens, n_new, page, rows)
        held = sorted(int(x) for b in range(B) for x in h[0][b, :h[1][b]])
        free = [int(h[2][(h[3][0] + i) % n_pages]) for i in range(h[3][1])]
        assert sorted(held + free) == list(range(n_pages))              # every page is held by one request or free
        lens = np.minimum(h[1] * page, lens + rng.integers(0, most + 1, B) * (n_new > 0))
        lens[rng.random(B) < 0.2] = 0


@pytest.mark.parametrize("B,rows", [(256, 1024), (257, 1023), (1024, 1024), (1024, 1025), (1023, 257), (1025, 1024), (1025, 300)])
def test_plan_on_both_sides_of_its_forms(B, rows):
    """Few requests and rows go to workgroups of 256 threads, others to 1024: the border, several requests of a thread, several workgroups."""
    rng = np.random.default_rng(B + rows)
    h = plan_state(rng, B, 4, 3 * B, 16)
    g = [dev(x) for x in h]
    lens = np.zeros(B, np.int64)
    for step in range(4):
        n_new = rng.integers(0, 12, B) * (rng.random(B) < min(1.0, rows / (4 * B)))
        check_plan(g, h, lens, n_new, 16, rows)
        lens = np.minimum(np.minimum(h[1] * 16, lens + n_new), 50)
        lens[rng.random(B) < 0.3] = 0


@pytest.mark.parametrize("lens,n_new,held,rows", [([0], [0], [0], 5), ([0], [1], [0], 1), ([5], [0], [1], 2), ([15], [1], [1], 1), ([16], [1], [1], 1), ([40], [3], [6], 3),
                                                  ([-4, 3], [2, -5], [0, 1], 4), ([0, 0, 0], [9, 1, 200], [0, 0, 0], 64), ([2 ** 31 - 1, 1], [2 ** 31 - 1, 3], [2, 0], 9)])
def test_plan_edges(lens, n_new, held, rows):
    rng = np.random.default_rng(4)
    h = plan_state(rng, len(lens), 6, 20, 16, held)
    # (positions are 32-bit numbers: those of a request whose rows do not fit are not compared beyond that)
    if max(lens) > 2 ** 30:
        g = [dev(x) for x in h]
        out = M.page_plan(*g, dev(lens), dev(n_new), 16, rows)
        assert out["served"].tolist() == [0, 0] and (out["slots"] == -1).all() and g[1].tolist() == [2, 0]
        return
    check_plan([dev(x) for x in h], h, lens, n_new, 16, rows)


def test_plan_serves_later_requests_that_need_nothing():
    rng = np.random.default_rng(5)
    h = plan_state(rng, 4, 8, 9, 16, [1, 2, 2, 1])                       # three pages free
    g = [dev(x) for x in h]
    out = check_plan(g, h, [16, 32, 30, 16], [20, 40, 2, 1], 16, 63)     # wants 2, 3, 0, 1: only the first and the third get theirs
    assert out["served"].tolist() == [1, 0, 1, 0]


def test_plan_without_rows_only_gives_back():
    h = plan_state(np.random.default_rng(6), 3, 4, 12, 16, [3, 1, 2])
    g = [dev(x) for x in h]
    out = check_plan(g, h, [16, 0, 32], [0, 0, 0], 16, 0)
    assert out["slots"].numel() == 0 and g[1].tolist() == [1, 0, 2]


def test_nothing_to_do():
    """Calls without rows return without a launch."""
    pool, _ = new_pool(1, 2, 64, 16)
    none = torch.zeros(0, dtype=torch.int32, device=DEV)
    q = torch.zeros((0, 4, 64), device=DEV)
    k = torch.zeros((0, 2, 64), device=DEV)
    assert M.rope_append(q, k, k, none, none, pool, 16, 2, 64, M.Rope("half", 64)).shape == (0, 4, 64)
    assert M.kv_rows(pool, none, 16, 2, 64)[0].shape == (0, 2, 64)
    assert M.attn_pages(q, pool, dev([[0]]), dev([0, 0]), dev([0]), 16, 2, 1.0, 1, 1).shape == (0, 4, 64)


# ---- rotation and append

def new_pool(n_pages, KH, hd, page, pad=0, fill=0xA5):
    full = torch.full((n_pages, M.page_bytes(KH, hd, page) + pad), fill, dtype=torch.uint8, device=DEV)
    return full[:, :M.page_bytes(KH, hd, page)], full


def held_by(pool, slots, page, KH, hd):
    k, v = M.kv_rows(pool, slots, page, KH, hd, torch.float32)
    return k.double().cpu().numpy(), v.double().cpu().numpy()


@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("page", [16, 64, 1024])
def test_append_holds_the_nearest_values(hd, page):
    """Without rotation codes and scales are exact: zeros, ties, the largest and smallest numbers, signs."""
    KH, rows = 3, 37
    g = torch.Generator().manual_seed(hd)
    k = torch.randn((rows, KH, hd), generator=g)
    v = torch.randn((rows, KH, hd), generator=g) * torch.exp(4 * torch.randn((rows, KH, 1), generator=g))
    k[0] = 0.0
    k[1, 0] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0] * (hd // 8)) * torch.tensor([1.0, -1.0]).repeat(hd // 2)      # ties
    k[2] *= 2.0 ** -130
    v[2] *= 2.0 ** -140
    k[3, 1] *= 1e37
    v[3, 0, :] = 3.4e38
    v[4, 2, 5] = 7.0 * 2.0 ** 9
    v[5, 2, 5] = float(np.nextafter(np.float32(7.0 * 2.0 ** 9), np.float32(1e9)))
    pool, full = new_pool(5 if page < 1024 else 2, KH, hd, page, pad=48)
    n_slots = pool.shape[0] * page
    slots = torch.randperm(n_slots, generator=g)[:rows].to(torch.int32).to(DEV)
    before = full.clone()
    M.rope_append(None, k.to(DEV), v.to(DEV), torch.zeros(rows, dtype=torch.int32, device=DEV), slots, pool, page, KH, hd, M.Rope())
    hk, hv = held_by(pool, slots, page, KH, hd)
    for x, got in ((k, hk), (v, hv)):
        for r in range(rows):
            for h in range(KH):
                want, _ = R.quantise(x[r, h].numpy())
                assert np.array_equal(got[r, h], want), (r, h)
    assert torch.equal(full[:, pool.shape[1]:], before[:, pool.shape[1]:])          # nothing between the pages
    # every other slot is as it was: read all slots before and after
    rest = torch.ones(n_slots, dtype=torch.bool)
    rest[slots.cpu().long()] = False
    others = rest.nonzero()[:, 0].to(torch.int32).to(DEV)
    a, b = M.kv_rows(pool, others, page, KH, hd), M.kv_rows(before[:, :pool.shape[1]], others, page, KH, hd)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_append_marks_what_is_not_finite():
    KH, hd, page = 2, 64, 16
    k, v = torch.ones((4, KH, hd)), torch.ones((4, KH, hd))
    k[0, 0, 3], k[1, 1, 60], v[2, 0, 40] = math.nan, math.inf, -math.inf
    pool, _ = new_pool(1, KH, hd, page)
    slots = torch.arange(4, dtype=torch.int32, device=DEV)
    M.rope_append(None, k.to(DEV), v.to(DEV), slots, slots, pool, page, KH, hd, M.Rope())
    for x in held_by(pool, slots, page, KH, hd):
        bad = np.isnan(x).all(-1)
        assert bad.tolist() == [[True, False], [False, True], [True, False], [False, False]]
        assert (x[~bad] == 1.0).all()


SPECS = [dict(style="half", rot_dim=0), dict(style="half", rot_dim=32), dict(style="pairs", rot_dim=32), dict(style="half", rot_dim=10), dict(style="pairs", rot_dim=2, gain=0.5),
         dict(style="half", rot_dim=32, scaling="linear", factor=4.0), dict(style="pairs", rot_dim=32, scaling="wave", theta=500000.0, factor=8.0, orig_ctx=2048),
         dict(style="half", rot_dim=32, scaling="index", factor=16.0, low=1.0, high=32.0, orig_ctx=512, gain=1.25)]


@pytest.mark.parametrize("spec", SPECS)
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("hd,H,KH,rows", [(32, 4, 4, 1), (64, 6, 2, 19), (128, 4, 1, 7), (32, 3, 1, 2100)])
def test_rope_append(spec, dt, hd, H, KH, rows):
    page = 32
    g = torch.Generator().manual_seed(rows + H)
    qkv = torch.randn((rows, (H + 2 * KH) * hd), generator=g).to(dt)
    pos = torch.randint(0, 3000, (rows,), generator=g).to(torch.int32)
    pos[-1] = 2 ** 31 - 1 if rows > 1 else 1
    n_pages = -(-rows // page) + 2
    slots = torch.randperm(n_pages * page, generator=g)[:rows].to(torch.int32)
    if rows > 5:
        slots[2], slots[3] = -1, n_pages * page                           # nothing is appended
    pool, full = new_pool(n_pages, KH, hd, page)
    d = qkv.to(DEV)
    q, k, v = d[:, :H * hd], d[:, H * hd:(H + KH) * hd], d[:, (H + KH) * hd:]
    out = M.rope_append(q, k, v, pos.to(DEV), slots.to(DEV), pool, page, KH, hd, M.Rope(**spec))
    x = qkv.double().numpy()
    want, err = R.rotate(x[:, :H * hd].reshape(rows, H, hd), pos.numpy(), spec)
    got = out.double().cpu().numpy()
    assert (np.abs(got - want) <= err + (R.H8 * 1.01 * np.abs(want) if dt == torch.bfloat16 else 0)).all()
    hk, hv = held_by(pool, slots.to(DEV), page, KH, hd)
    ky, kerr = R.rotate(x[:, H * hd:(H + KH) * hd].reshape(rows, KH, hd), pos.numpy(), spec)
    for y, e, held in ((ky, kerr, hk), (x[:, (H + KH) * hd:].reshape(rows, KH, hd), 0 * kerr, hv)):
        for r in range(rows) if rows < 50 else range(0, rows, 211):
            if slots[r] < 0 or slots[r] >= n_pages * page:
                assert (held[r] == 0).all()
                continue
            for h in range(KH):
                for c in range(hd // 32):
                    at = slice(32 * c, 32 * c + 32)
                    b, ee = y[r, h, at], e[r, h, at]
                    top = np.abs(b).max()
                    ok = False                                            # next to a border of the scale either one is right
                    for s in {R.scale_exponent(float(top - ee.max())), R.scale_exponent(float(top + ee.max()))}:
                        a = np.abs(b) / 2.0 ** s
                        ok = ok or (np.abs(held[r, h, at] - b) <= R.half_step(a + ee / 2.0 ** s) * 2.0 ** s + ee).all()
                    assert ok, (r, h, c)
    # in place, and the same bits from rows of their own
    again = q.clone()
    M.rope_append(again.view(rows, H, hd), None, None, pos.to(DEV), None, None, page, KH, hd, M.Rope(**spec), out=again.view(rows, H, hd))
    assert torch.equal(again.view(rows, H, hd), out)
    other, _ = new_pool(n_pages, KH, hd, page)
    M.rope_append(None, k.contiguous(), v.contiguous().view(rows, KH, hd), pos.to(DEV), slots.to(DEV), other, page, KH, hd, M.Rope(**spec))
    assert torch.equal(other, full)


# ---- attention

def filled(rng, lens, KH, hd, page, extra=2, bad_rest=True):
    """A pool with requests of these lengths, appended by the library from N(0, 1) rows; what the pages hold elsewhere are bytes 255."""
    B = len(lens)
    width = max(1, max(-(-L // page) for L in lens)) + 1
    pages = [-(-L // page) for L in lens]
    n_pages = sum(pages) + extra
    ids = rng.permutation(n_pages)
    table = np.full((B, width), 2 ** 31 - 1 if bad_rest else 0, np.int64)
    k = 0
    for b in range(B):
        table[b, :pages[b]] = ids[k:k + pages[b]]
        k += pages[b]
    pool, _ = new_pool(n_pages, KH, hd, page, fill=255)
    K, V = [], []
    g = torch.Generator().manual_seed(int(rng.integers(1 << 30)))
    for b, L in enumerate(lens):
        if L == 0:
            K.append(np.zeros((0, KH, hd)))
            V.append(np.zeros((0, KH, hd)))
            continue
        p = np.arange(L)
        slots = dev(table[b, p // page] * page + p % page)
        x = torch.randn((2, L, KH, hd), generator=g).to(DEV)
        M.rope_append(None, x[0], x[1], slots, slots, pool, page, KH, hd, M.Rope())
        kk, vv = held_by(pool, slots, page, KH, hd)
        K.append(kk)
        V.append(vv)
    return pool, dev(table), K, V


def check_attn(q, pool, table, K, V, lens, n_new, page, KH, scale, max_new=None, max_len=None):
    rows = q.shape[0]
    start = np.concatenate([[0], np.cumsum(n_new)])
    out = torch.full((rows + 3, q.shape[1], q.shape[2]), 77.0, dtype=q.dtype, device=DEV)
    more = torch.cat([q, torch.full_like(out[:3], math.nan)])             # rows behind the last request
    M.attn_pages(more, pool, table, dev(start), dev(lens), page, KH, scale, max_new or max(1, max(n_new)), max_len or max(1, max(lens)), out=out)
    want, bound = R.attention(q.double().cpu().numpy(), K, V, lens, n_new, scale, q.dtype == torch.bfloat16)
    got = out[:rows].double().cpu().numpy()
    assert (out[rows:] == 77.0).all()
    assert np.array_equal(np.isnan(got), np.isnan(want))
    fine = ~np.isnan(want)
    worst = (np.abs(got - want) / np.maximum(bound, 1e-300))[fine]
    assert (np.abs(got - want)[fine] <= bound[fine]).all(), float(worst.max())
    return out[:rows]


EDGES = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 257]


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("H,KH,hd", [(4, 4, 32), (8, 2, 64), (3, 1, 128), (2, 2, 128), (12, 12, 64)])
@pytest.mark.parametrize("page", [16, 64])
def test_attention_of_single_tokens(dt, H, KH, hd, page):
    rng = np.random.default_rng(H * hd + page)
    pool, table, K, V = filled(rng, EDGES, KH, hd, page)
    q = torch.randn((len(EDGES), H, hd), generator=torch.Generator().manual_seed(1)).to(dt).to(DEV)
    check_attn(q, pool, table, K, V, EDGES, [1] * len(EDGES), page, KH, 1 / math.sqrt(hd))


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("H,KH,hd,page", [(4, 4, 32, 32), (8, 2, 64, 16), (5, 1, 128, 128), (2, 2, 128, 16)])
def test_attention_of_ragged_blocks(dt, H, KH, hd, page):
    """Blocks of 0 to 40 rows; requests without positions, rows that see nothing, blocks longer than their context."""
    rng = np.random.default_rng(hd + page)
    lens = [0, 5, 40, 3, 0, 70, 150, 16, 33, 64, 1]
    n_new = [0, 5, 40, 7, 4, 1, 17, 16, 9, 0, 1]
    pool, table, K, V = filled(rng, lens, KH, hd, page)
    q = torch.randn((sum(n_new), H, hd), generator=torch.Generator().manual_seed(2)).to(dt).to(DEV)
    check_attn(q, pool, table, K, V, lens, n_new, page, KH, 0.3)


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("H,KH,hd,L,n", [(2, 2, 128, 1500, 6), (4, 1, 64, 3000, 1), (4, 4, 32, 900, 3), (8, 1, 64, 700, 16), (2, 1, 64, 300, 130)])
def test_attention_of_long_contexts(dt, H, KH, hd, L, n):
    """One request whose context is split over workgroups and merged; hints on the lengths that are off change nothing."""
    rng = np.random.default_rng(L)
    pool, table, K, V = filled(rng, [L], KH, hd, 64)
    q = torch.randn((n, H, hd), generator=torch.Generator().manual_seed(3)).to(dt).to(DEV)
    check_attn(q, pool, table, K, V, [L], [n], 64, KH, 1 / math.sqrt(hd))
    for hint in (1, L // 3, 4 * L):
        check_attn(q, pool, table, K, V, [L], [n], 64, KH, 1 / math.sqrt(hd), max_new=n + 5, max_len=hint)


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("H,KH,hd,page", [(2, 2, 32, 16), (4, 2, 64, 64), (2, 1, 128, 32), (1, 1, 64, 128)])
def test_attention_of_prompts(dt, H, KH, hd, page):
    """Long blocks among short and empty ones: prompts, the rest of a prompt behind its prefix, rows that see nothing."""
    rng = np.random.default_rng(hd + page)
    lens, n_new = [0, 300, 350, 17, 600, 1, 250], [0, 300, 260, 17, 30, 1, 270]
    pool, table, K, V = filled(rng, lens, KH, hd, page)
    q = torch.randn((sum(n_new), H, hd), generator=torch.Generator().manual_seed(6)).to(dt).to(DEV)
    check_attn(q, pool, table, K, V, lens, n_new, page, KH, 1 / math.sqrt(hd))


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("H,KH,hd,L,n", [(2, 1, 128, 2000, 300), (1, 1, 64, 4100, 257), (4, 2, 32, 900, 700)])
def test_attention_of_prompts_behind_long_contexts(dt, H, KH, hd, L, n):
    """Long blocks whose positions are split over workgroups and merged."""
    rng = np.random.default_rng(L)
    pool, table, K, V = filled(rng, [L], KH, hd, 64)
    q = torch.randn((n, H, hd), generator=torch.Generator().manual_seed(7)).to(dt).to(DEV)
    for hint in (L, 50, 3 * L):
        check_attn(q, pool, table, K, V, [L], [n], 64, KH, 1 / math.sqrt(hd), max_len=hint)


@pytest.mark.parametrize("dt,B,H,KH,n", [(torch.bfloat16, 6, 16, 16, 500), (torch.float32, 3, 16, 16, 300), (torch.bfloat16, 1120, 256, 1, 1), (torch.float32, 700, 256, 1, 1)])
def test_attention_of_many_long_blocks(dt, B, H, KH, n):
    """More workgroups than CUs, in several rounds and bundles."""
    rng = np.random.default_rng(B)
    lens = rng.integers(1, 60, B) + (n if n > 1 else 0)
    n_new = [int(rng.integers(max(1, n - 100), n + 1)) for _ in range(B)]
    pool, table, K, V = filled(rng, lens, KH, 32, 16)
    q = torch.randn((sum(n_new), H, 32), generator=torch.Generator().manual_seed(8)).to(dt).to(DEV)
    check_attn(q, pool, table, K, V, lens, n_new, 16, KH, 0.2, max_new=n)


def test_attention_with_large_scores_and_marked_positions():
    """Scores of hundreds (the weight is on one position); a marked position makes the rows that see it NaN and no others."""
    rng = np.random.default_rng(8)
    KH, hd, page, L, n = 2, 64, 16, 90, 5
    pool, table, K, V = filled(rng, [L, L], KH, hd, page)
    q = (torch.randn((2 * n, 4, hd), generator=torch.Generator().manual_seed(4)) * 60).to(DEV)
    check_attn(q, pool, table, K, V, [L, L], [n, n], page, KH, 1.0)
    at = table[1, (L - 3) // page].item() * page + (L - 3) % page        # request 1, position L - 3: rows 2, 3, 4 see it
    bad = torch.ones((1, KH, hd), device=DEV)
    bad[0, 1, 7] = math.nan
    slot = dev([at])
    M.rope_append(None, torch.ones_like(bad), bad, slot, slot, pool, page, KH, hd, M.Rope())
    K[1][L - 3, 0] = V[1][L - 3, 0] = 1.0
    K[1][L - 3, 1] = np.nan
    V[1][L - 3, 1] = 0.0
    out = check_attn((q / 60), pool, table, K, V, [L, L], [n, n], page, KH, 1.0)
    nan = torch.isnan(out).all(-1)
    assert nan.sum().item() == 3 * 2 and nan[n + 2:, 2:].all()


def test_attention_strides_and_far_pages():
    """Rows of q and out inside wider buffers; a pool longer than 4 GiB with the pages at its end."""
    rng = np.random.default_rng(9)
    KH, hd, page, L, n, H = 2, 128, 64, 150, 3, 4
    pool, table, K, V = filled(rng, [L], KH, hd, page, bad_rest=False)
    wide = torch.randn((n, 7 * hd), generator=torch.Generator().manual_seed(5)).to(DEV)
    q = wide[:, hd:5 * hd].unflatten(1, (H, hd))
    buf = torch.zeros((n, 6 * hd), device=DEV)
    out = buf[:, 2 * hd:].unflatten(1, (H, hd))
    start, lens = dev([0, n]), dev([L])
    M.attn_pages(q, pool, table, start, lens, page, KH, 0.1, n, L, out=out)
    flat = M.attn_pages(q.contiguous(), pool, table, start, lens, page, KH, 0.1, n, L)
    assert torch.equal(out, flat) and (buf[:, :2 * hd] == 0).all()
    want, bound = R.attention(q.double().cpu().numpy(), K, V, [L], [n], 0.1, False)
    assert (np.abs(flat.double().cpu().numpy() - want) <= bound).all()
    stride = 1 << 30                                                     # pages a GiB apart: as many layers share a table
    far = torch.empty((6, stride), dtype=torch.uint8, device=DEV)[:, 4096:4096 + pool.shape[1]]
    far[1:].copy_(pool)
    assert torch.equal(M.attn_pages(q.contiguous(), far, table + 1, start, lens, page, KH, 0.1, n, L), flat)
    slots = dev([5 * page + 3])
    x = torch.randn((2, 1, KH, hd), device=DEV)
    M.rope_append(None, x[0], x[1], slots, slots, far, page, KH, hd, M.Rope())
    near, _ = new_pool(1, KH, hd, page)
    M.rope_append(None, x[0], x[1], slots, dev([3]), near, page, KH, hd, M.Rope())
    a, b = M.kv_rows(far, slots, page, KH, hd), M.kv_rows(near, dev([3]), page, KH, hd)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


# ---- verification

def laws(rng, rows, gamma, V, sharp=2.0):
    def soft(x):
        e = np.exp(x - x.max(-1, keepdims=True))
        return (e / e.sum(-1, keepdims=True)).astype(np.float32)
    z = rng.standard_normal((rows, gamma + 1, V)) * sharp
    return soft(z), soft(z[:, :gamma] + 0.7 * rng.standard_normal((rows, gamma, V)))


def check_accept(P, Q, d, n, u, w):
    t = lambda x, dt=torch.float32: None if x is None else torch.as_tensor(x).to(dt).to(DEV)  # noqa: E731
    out = M.accept_probs(t(P), t(Q), t(d, torch.int32), t(n, torch.int32), t(u), t(w))
    acc, tokens = R.accept(P, Q, d, n, u, w)
    assert out["n_acc"].tolist() == acc.tolist()
    assert np.array_equal(out["tokens"].cpu().numpy(), tokens)
    return out


@pytest.mark.parametrize("V", [1, 2, 3, 7, 64, 1000, 4095, 4096, 4097, 8190, 32000])
@pytest.mark.parametrize("rows,gamma,onehot", [(1, 1, False), (17, 4, False), (9, 3, True)])
def test_accept_probs(V, rows, gamma, onehot):
    rng = np.random.default_rng(V + rows)
    P, Q = laws(rng, rows, gamma, V)
    d = np.stack([[rng.choice(V, p=Q[b, j].astype(np.float64) / Q[b, j].astype(np.float64).sum()) for j in range(gamma)] for b in range(rows)])
    if rows > 3:
        d[1, 0], d[2, gamma - 1] = -1, V                                  # drafts outside the vocabulary fail
    n = rng.integers(-1, gamma + 2, rows)
    u, w = rng.random((rows, gamma)).astype(np.float32), rng.random(rows).astype(np.float32)
    w[0] = 0.0
    if rows > 2:
        w[1] = np.nextafter(np.float32(1), np.float32(0))
    check_accept(P, None if onehot else Q, d, n, u, w)
    check_accept(P, None if onehot else Q, d, None, u * 0, w)             # u = 0: every draft with a positive probability passes


def test_accept_probs_borders():
    """Laws with zeros, equal laws, laws without a weight, NaN, infinite ties: dyadic numbers, so that every sum is exact."""
    V, G = 4100, 2
    P, Q = np.zeros((8, G + 1, V), np.float32), np.zeros((8, G, V), np.float32)
    P[:, :, 4098], P[:, :, 5] = 0.5, 0.5
    Q[:, :, 5] = 1.0
    d = np.full((8, G), 5)
    u = np.full((8, G), 0.5, np.float32)                                  # u q = p exactly: not accepted
    w = np.zeros(8, np.float32)
    P[1], Q[1] = 0.0, 0.0                                                 # nothing anywhere
    P[2] = np.nan
    Q[3] = P[3, :G]                                                       # equal laws, the test fails for u = 1: nothing is left of the residual
    u[3] = 1.0
    u[4] = np.nextafter(np.float32(0.5), np.float32(0))                   # just below: accepted
    w[4] = 0.5                                                            # the sum up to 5 is exactly half: the next token
    P[5, 0, 7] = np.nan                                                   # a NaN beside the rest counts as nothing
    P[6, 0, 7] = -1.0
    w[7] = np.nextafter(np.float32(1), np.float32(0))
    check_accept(P, Q, d, None, u, w)
    check_accept(P, None, d, [0, 0, 1, 1, 2, 2, 0, 0], u, w)


@pytest.mark.parametrize("V", [70000, 300001, 1 << 20])
def test_accept_probs_of_long_laws(V):
    """Sixteen tokens of one weight at the borders of the wavefronts' spans and pieces: every one of them is drawn, at and just below its border."""
    span = -(-V // 4096) * 256
    at = np.unique(np.minimum([0, 255, 256, 4095, 4096, span - 1, span, span + 255, span + 256, span + 4095, span + 4096, 2 * span - 1, 9 * span + 3, 15 * span - 1, V - 2, V - 1], V - 1))
    P = np.zeros((32, 2, V), np.float32)
    P[:, :, at] = 1 / 16
    w = np.arange(32, dtype=np.float32) // 2 / 16
    w[1::2] = np.nextafter(w[1::2], np.float32(0))
    w[1] = 0
    Q = np.zeros((32, 1, V), np.float32)
    Q[:, 0, at[::2]] = 1 / 16                                             # behind a rejection: every second of them
    check_accept(P, Q, np.full((32, 1), at[3]), None, np.zeros((32, 1), np.float32), w)
    check_accept(P, Q, np.full((32, 1), at[0]), None, np.ones((32, 1), np.float32), w)
    check_accept(P, None, np.full((32, 1), at[-1]), None, np.ones((32, 1), np.float32), w)


def test_accept_probs_strided_and_unaligned():
    rng = np.random.default_rng(3)
    P, Q = laws(rng, 5, 3, 1003)
    wide = torch.zeros((4, 5, 1100), device=DEV)                          # positions outside, rows inside, and 4 bytes off
    p = wide[:, :, 1:1004].transpose(0, 1)
    p.copy_(torch.as_tensor(P))
    d = rng.integers(0, 1003, (5, 3))
    u, w = rng.random((5, 3)).astype(np.float32) * 0.3, rng.random(5).astype(np.float32)
    out = M.accept_probs(p, torch.as_tensor(Q).to(DEV), dev(d), None, torch.as_tensor(u).to(DEV), torch.as_tensor(w).to(DEV))
    acc, tokens = R.accept(P, Q, d, None, u, w)
    assert out["n_acc"].tolist() == acc.tolist() and np.array_equal(out["tokens"].cpu().numpy(), tokens)


def test_accept_probs_is_lossless():
    """Over 200000 draws the first emitted token follows p whatever q is (V = 8): every count within 5 sigma."""
    rng = np.random.default_rng(6)
    n = 65000
    P1, Q1 = laws(rng, 1, 1, 8, sharp=1.0)
    P, Q = np.repeat(P1, n, 0), np.repeat(Q1, n, 0)
    counts = np.zeros(8)
    for seed in range(3):
        r = np.random.default_rng(seed)
        q = Q1[0, 0].astype(np.float64)
        d = r.choice(8, size=(n, 1), p=q / q.sum())
        t = lambda x, dt=torch.float32: torch.as_tensor(x).to(dt).to(DEV)  # noqa: E731
        out = M.accept_probs(t(P), t(Q), t(d, torch.int32), None, t(r.random((n, 1))), t(r.random(n)))
        counts += np.bincount(out["tokens"][:, 0].cpu().numpy(), minlength=8)
    p = P1[0, 0].astype(np.float64)
    p /= p.sum()
    N = 3 * n
    assert (np.abs(counts - N * p) <= 5 * np.sqrt(N * p * (1 - p))).all()


# ---- a run of them together

def test_a_batch_is_served():
    """Rounds of a batch through plan, append, attention and verification, against a host that keeps every request's rows in full: lengths
    follow the verification, requests end and start, the pool is smaller than all requests at their longest.  Each round is also captured
    once into a graph and replayed after the eager call has moved on."""
    rng = np.random.default_rng(11)
    B, H, KH, hd, page, gamma, V, width, n_pages = 5, 4, 2, 64, 16, 3, 50, 8, 24
    spec = dict(style="half", rot_dim=hd)
    scale = 1 / math.sqrt(hd)
    h = plan_state(rng, B, width, n_pages, page)
    g = [dev(x) for x in h]
    pool, _ = new_pool(n_pages, KH, hd, page, fill=255)
    lens = np.zeros(B, np.int64)
    K = [np.zeros((0, KH, hd)) for _ in range(B)]
    V_ = [np.zeros((0, KH, hd)) for _ in range(B)]
    rope = M.Rope(**spec)
    for step in range(8):
        n_new = np.where(lens == 0, rng.integers(1, 40, B), gamma + 1)
        rows = int(n_new.sum()) + 2
        out = check_plan(g, h, lens, n_new, page, rows)
        served, start, slots, pos = (out[k].cpu().numpy() for k in ("served", "start", "slots", "pos"))
        x = torch.randn((rows, (H + 2 * KH) * hd), generator=torch.Generator().manual_seed(step)).to(DEV)
        q, k, v = x[:, :H * hd], x[:, H * hd:(H + KH) * hd], x[:, (H + KH) * hd:]
        now = np.where(served > 0, lens + n_new, 0)
        qr = M.rope_append(q, k, v, out["pos"], out["slots"], pool, page, KH, hd, rope)
        y = M.attn_pages(qr, pool, g[0], out["start"], dev(now), page, KH, scale, int(n_new.max()), int(max(1, now.max())))
        hk, hv = held_by(pool, out["slots"], page, KH, hd)
        for b in range(B):
            if served[b]:
                at = slice(int(start[b]), int(start[b + 1]))
                K[b], V_[b] = np.concatenate([K[b][:lens[b]], hk[at]]), np.concatenate([V_[b][:lens[b]], hv[at]])
                assert (slots[at] >= 0).all() and (pos[at] == lens[b] + np.arange(n_new[b])).all()
        counts = [int(n) if served[b] else 0 for b, n in enumerate(n_new)]
        live = np.concatenate([np.arange(start[b], start[b + 1]) for b in range(B) if served[b]]).astype(np.int64)
        want, bound = R.attention(qr[live].double().cpu().numpy(), K, V_, now, counts, scale, False)
        assert (np.abs(y[live].double().cpu().numpy() - want) <= bound).all()
        P, Q = laws(rng, B, gamma, V, 1.0)
        d, u, w = rng.integers(0, V, (B, gamma)), rng.random((B, gamma)).astype(np.float32) * 0.5, rng.random(B).astype(np.float32)
        nd = np.where(n_new == gamma + 1, gamma, 0)
        acc = check_accept(P, Q, d, nd, u, w)["n_acc"].cpu().numpy()
        lens = np.where(served > 0, np.where(nd > 0, lens + 1 + acc, now), lens)
        ended = (lens > width * page - gamma - 2) | (rng.random(B) < 0.1)
        lens[ended] = 0
    assert h[1].sum() + h[3][1] == n_pages


@pytest.mark.parametrize("side", [False, True])
def test_a_step_replays_from_a_graph(side):
    """A captured step gives on every replay what the eager calls give for the inputs it finds, on the default and on another stream, with
    eager work and synchronisations between the replays."""
    rng = np.random.default_rng(12)
    B, H, KH, hd, page, gamma, V, width, n_pages = 3, 4, 4, 128, 16, 4, 6000, 90, 300
    h = plan_state(rng, B, width, n_pages, page)
    g = [dev(x) for x in h]
    pool, _ = new_pool(n_pages, KH, hd, page, fill=0)
    lens, n_new, rows = dev([700, 0, 1200]), dev([gamma + 1] * B), B * (gamma + 1)
    now = lens + n_new
    x = torch.randn((rows, 3 * H * hd), device=DEV)
    P, Q = (torch.as_tensor(a).to(DEV) for a in laws(rng, B, gamma, V))
    d, u, w = dev(rng.integers(0, V, (B, gamma))), torch.rand((B, gamma), device=DEV), torch.rand(B, device=DEV)
    rope = M.Rope("half", hd)

    def step():
        s = M.page_plan(*g, lens, n_new, page, rows)
        q = M.rope_append(x[:, :H * hd], x[:, H * hd:2 * H * hd], x[:, 2 * H * hd:], s["pos"], s["slots"], pool, page, KH, hd, rope)
        y = M.attn_pages(q, pool, g[0], s["start"], now, page, KH, 0.1, gamma + 1, width * page)
        t = M.accept_probs(P, Q, d, None, u, w)
        return [s["slots"], s["pos"], q, y, t["n_acc"], t["tokens"]]

    stream = torch.cuda.Stream() if side else torch.cuda.current_stream()
    with torch.cuda.stream(stream):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream if side else None):
        got = step()
    for i in range(4):
        x.normal_()
        u.uniform_()
        w.uniform_()
        lens.copy_(dev([700 - 3 * i, 17 * i, 1200 + i]))
        now.copy_(lens + n_new)
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            graph.replay()
        torch.cuda.synchronize()
        want = step()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)
