"""Contexts whose target keeps its cache in 4-bit pages: every round's target logits against a 64-bit forward pass over the values that the
pages hold (read back), the held values against the pass's own K and V, the book against its rules."""
import ctypes as C

import numpy as np
import pytest
import torch

import pages_ref as R
import workloads as W

pytestmark = pytest.mark.gpu

M = pytest.importorskip("paper_2604_05417_amd")
TOL = 3e-2                                              # of the logits of a bf16 model, as everywhere


def small(d=256, heads=4, kv_heads=2, layers=2, vocab=1024, act=W.SWIGLU, ffn=512):
    td = W.model_desc(layers, d, heads, kv_heads, ffn, vocab, act, W.BF16)
    dd = W.model_desc(1, 128, 2, 2, 256, vocab, W.SWIGLU, W.BF16)
    return (td, W.gen_weights(td, 11, std=0.05)), [(dd, W.gen_weights(dd, 20 + k, std=0.05)) for k in range(2)]


class Reference:
    def __init__(self, desc, weights):
        self.d = desc
        self.w = [None if x is None else x.double().numpy() for x in weights]
        self.hd = desc["d_model"] // desc["n_heads"]
        half = self.hd // 2
        self.paired = np.stack([np.arange(half), np.arange(half) + half], 1).reshape(-1)      # rotary pairs next to each other

    def norm(self, h, g):
        return h / np.sqrt((h * h).mean(-1, keepdims=True) + self.d["rms_eps"]) * g

    def forward(self, tokens, pos, held):
        """tokens at positions pos ..; held(L): K and V [positions, KH, hd] up to the block's end as the pages hold them.  Returns logits and the
        block's own K (rotated, paired order) and V per layer."""
        d, hd = self.d, self.hd
        H, KH, G = d["n_heads"], d["n_kv_heads"], d["n_heads"] // d["n_kv_heads"]
        h, own = self.w[0][tokens], []
        at = pos + np.arange(len(tokens))
        for L in range(d["n_layers"]):
            an, wq, wk, wv, wo, fn, wg, wu, wd = self.w[1 + 9 * L: 10 + 9 * L]
            x = self.norm(h, an)
            q, k, v = (x @ w.T for w in (wq, wk, wv))
            rope = dict(style="half", rot_dim=hd, theta=d["rope_theta"])
            q = R.rotate(q.reshape(-1, H, hd), at, rope)[0][..., self.paired]
            k = R.rotate(k.reshape(-1, KH, hd), at, rope)[0][..., self.paired]
            own.append((k, v.reshape(-1, KH, hd)))
            K, V = held(L)
            o = np.zeros((len(tokens), H, hd))
            for i, p in enumerate(at):
                for hh in range(H):
                    s = K[:p + 1, hh // G] @ q[i, hh] / np.sqrt(hd)
                    e = np.exp(s - s.max())
                    o[i, hh] = e @ V[:p + 1, hh // G] / e.sum()
            h = h + o.reshape(len(tokens), -1) @ wo.T
            x = self.norm(h, fn)
            if d["act"] == W.SWIGLU:
                a = x @ wg.T
                x = a / (1 + np.exp(-a)) * (x @ wu.T)
            else:
                from math import erf
                a = x @ wu.T
                x = 0.5 * a * (1 + np.vectorize(erf)(a / np.sqrt(2)))
            h = h + x @ wd.T
        return self.norm(h, self.w[-2]) @ self.w[-1].T, own


def read_back(g, seq, upto, page):
    td = g.tdesc
    hd, lb = td["d_model"] // td["n_heads"], g.page_pool.shape[1] // td["n_layers"]
    p = torch.arange(upto, device="cuda")
    slots = (g.page_table[seq][p // page] * page + p % page).to(torch.int32)
    out = []
    for L in range(td["n_layers"]):
        k, v = M.kv_rows(g.page_pool[:, L * lb:(L + 1) * lb], slots, page, td["n_kv_heads"], hd, torch.float32)
        out.append((k.double().cpu().numpy(), v.double().cpu().numpy()))
    return out


def check_held(held, own, pos):
    """Held rows are the nearest values to the pass's own: half a step, and what the projections' two-term arithmetic may be off by."""
    for (K, V), (k, v) in zip(held, own):
        for y, z in ((k, K[pos:pos + len(k)]), (v, V[pos:pos + len(k)])):
            eps = 2e-3 * np.abs(y).max()
            for i in range(len(y)):
                for h in range(y.shape[1]):
                    for c in range(y.shape[2] // 32):
                        b, s = y[i, h, 32 * c:32 * c + 32], z[i, h, 32 * c:32 * c + 32]
                        top = np.abs(b).max()
                        assert any((np.abs(s - b) <= R.half_step((np.abs(b) + eps) / 2.0 ** e) * 2.0 ** e + eps).all()
                                   for e in {R.scale_exponent(top - eps), R.scale_exponent(top + eps)})


def book_is_consistent(g, batch, n_pages, lens, page):
    pages = [-(-n // page) for n in lens]
    listed = [int(x) for b in range(batch) for x in g.page_table[b][:pages[b]]]
    assert len(set(listed)) == len(listed) and all(0 <= x < n_pages for x in listed)


@pytest.mark.parametrize("shape,T", [(dict(), 1.0), (dict(d=256, heads=8, kv_heads=8, act=W.GELU), 0.0), (dict(d=512, heads=4, kv_heads=1, layers=1), 1.0)])
@pytest.mark.parametrize("batch,page", [(1, 16), (3, 32)])
def test_rounds_against_the_values_the_pages_hold(shape, T, batch, page):
    target, drafters = small(**shape)
    ref = Reference(*target)
    gamma, max_ctx = 4, 160
    n_pages = batch * 6 if page == 32 else batch * 11
    g = M.MetaSD(target, drafters, gamma_max=gamma, max_ctx=max_ctx, temperature=T, seed=5, batch=batch, target_pages=(n_pages, page))
    prompts = [W.prompt_tokens(n, target[0]["vocab"], 60 + n) for n in (40, 17, 98)[:batch]]
    hist = [list(int(t) for t in p) for p in prompts]
    for b, p in enumerate(prompts):
        g.set_context(p, seq=b)
    for b, p in enumerate(prompts):                     # the prefill's own rows
        if len(p) > 1:
            held = read_back(g, b, len(p) - 1, page)
            _, own = ref.forward(np.array(p[:-1]), 0, lambda L: held[L])
            check_held(held, own, 0)
    for rnd in range(4):
        arms = [g.bandit_select(seq=b) for b in range(batch)]
        g.draft(arms if batch > 1 else arms[0], gamma)
        g.verify(gamma)
        torch.cuda.synchronize()
        P = g.peek("P", gamma).clone().cpu().numpy().reshape(batch, -1, target[0]["vocab"])
        D = g.peek("draft", gamma).clone().cpu().numpy().reshape(batch, -1)
        for b in range(batch):
            l = len(hist[b])
            block = np.array([hist[b][-1]] + [int(t) for t in D[b][:gamma]])
            held = read_back(g, b, l + gamma, page)
            logits, own = ref.forward(block, l - 1, lambda L: held[L])
            assert np.abs(P[b][:gamma + 1] - logits).max() <= TOL
            check_held(held, own, l - 1)
        book_is_consistent(g, batch, n_pages, [len(h) + gamma for h in hist], page)
        n, tok, _, _ = g.accept(gamma)
        n, tok = np.atleast_1d(n), np.atleast_1d(tok)
        for b in range(batch):
            hist[b] += [int(t) for t in D[b][:n[b]]] + [int(tok[b])]
            g.bandit_update(arms[b], int(n[b]), gamma, seq=b)
            assert g.state(-1, seq=b)[:2] == (len(hist[b]), len(hist[b]) - 1)
    if batch > 1:                                       # a new query in one place: its pages go back, the others' stay as they were
        before = read_back(g, 2, len(hist[2]) - 1, page)
        g.set_context(W.prompt_tokens(50, target[0]["vocab"], 99), seq=0)
        for (a, b), (c, d) in zip(before, read_back(g, 2, len(hist[2]) - 1, page)):
            assert np.array_equal(a, c) and np.array_equal(b, d)
        g.draft([0] * batch, gamma)
        g.verify(gamma)
        g.accept(gamma)
    g.close()


def test_a_long_prompt_and_a_prefilled_one():
    """A prompt that goes through in one long block, and a context whose pages the caller fills from the table."""
    target, drafters = small(layers=1)
    ref, page, gamma, n = Reference(*target), 64, 3, 330
    toks = W.prompt_tokens(n, target[0]["vocab"], 5)
    g = M.MetaSD(target, drafters, gamma_max=gamma, max_ctx=400, temperature=1.0, seed=5, target_pages=(7, page))
    g.set_context(toks)
    held = read_back(g, 0, n - 1, page)
    _, own = ref.forward(toks[:-1], 0, lambda L: held[L])
    check_held(held, own, 0)
    g.draft(0, gamma)
    g.verify(gamma)
    torch.cuda.synchronize()
    P, D = g.peek("P").clone().cpu().numpy(), g.peek("draft").clone().cpu().numpy()
    held = read_back(g, 0, n + gamma, page)
    logits, _ = ref.forward(np.concatenate([toks[-1:], D[:gamma]]), n - 1, lambda L: held[L])
    assert np.abs(P[:gamma + 1] - logits).max() <= TOL
    g.accept(gamma)
    # the same query again, its K and V given: rows of the caller's, in the order that the pages keep
    g.set_context(toks, kv_prefilled=True)
    p = torch.arange(n - 1, device="cuda")
    slots = (g.page_table[0][p // page] * page + p % page).to(torch.int32)
    kv = torch.randn((2, n - 1, 2, 64), generator=torch.Generator().manual_seed(1)).to("cuda")
    M.rope_append(None, kv[0], kv[1], slots, slots, g.page_pool, page, 2, 64, M.Rope())
    for b in g.kv_drafters:
        b.zero_()
    g.draft(1, gamma)
    g.verify(gamma)
    torch.cuda.synchronize()
    P, D = g.peek("P").clone().cpu().numpy(), g.peek("draft").clone().cpu().numpy()
    held = read_back(g, 0, n + gamma, page)
    assert np.array_equal(held[0][0][:n - 1], read_back(g, 0, n - 1, page)[0][0])
    logits, _ = ref.forward(np.concatenate([toks[-1:], D[:gamma]]), n - 1, lambda L: held[L])
    assert np.abs(P[:gamma + 1] - logits).max() <= TOL
    g.close()


def test_too_few_pages_and_other_refusals():
    target, drafters = small(layers=1)
    vocab = target[0]["vocab"]
    # 30 and 33 tokens and four drafts take ceil(34 / 16) + ceil(37 / 16) = 6 pages: five are refused before the first round, six last for some
    five = M.MetaSD(target, drafters, gamma_max=4, max_ctx=160, temperature=1.0, seed=5, batch=2, target_pages=(5, 16))
    five.set_context(W.prompt_tokens(30, vocab, 1), seq=0)
    for n in (60, 33):
        with pytest.raises(M.MetaSDError) as e:
            five.set_context(W.prompt_tokens(n, vocab, 2), seq=1)
        assert e.value.code == -2 and "pages" in str(e.value)
    five.close()
    g = M.MetaSD(target, drafters, gamma_max=4, max_ctx=160, temperature=1.0, seed=5, batch=2, target_pages=(6, 16))
    g.set_context(W.prompt_tokens(30, vocab, 1), seq=0)
    g.set_context(W.prompt_tokens(33, vocab, 2), seq=1)
    rounds = 0
    with pytest.raises(M.MetaSDError) as e:
        while rounds < 40:
            g.draft([0, 1], 4)
            g.verify(4)
            g.accept(4)
            rounds += 1
    assert e.value.code == -2 and "pages" in str(e.value) and 1 <= rounds < 40
    g.set_context(W.prompt_tokens(5, vocab, 3), seq=0)                   # a shorter query: its predecessor's pages are free again
    g.draft([0, 1], 4)
    g.verify(4)
    g.accept(4)
    g.close()
    one = M.MetaSD(target, drafters, gamma_max=4, max_ctx=160, temperature=1.0, seed=5, target_pages=(11, 16))
    one.set_context(W.prompt_tokens(30, vocab, 1))
    with pytest.raises(M.MetaSDError):
        one.draft_tree(0, [-1, 0, 0], [0, 0, 1])
    with pytest.raises(M.MetaSDError) as e:                              # no second pool behind a running query
        M.binding._check(one.L.metasd_set_target_pages(one._h, one.page_pool.data_ptr(), 11, 16, one._book.data_ptr(), one._book.numel() * 4), one._h)
    assert e.value.code == -3
    one.close()
    with pytest.raises(ValueError):
        M.MetaSD(target, [W.early_exit_drafter(target[0], target[1], 1, 0.02, 3)], gamma_max=4, max_ctx=160, temperature=1.0, seed=5, share_target_kv=True, target_pages=(11, 16))


def test_a_context_without_a_cache_waits_for_its_pages():
    target, drafters = small(layers=1)
    g = M.MetaSD(target, drafters, gamma_max=2, max_ctx=64, temperature=0.0, seed=1)
    h = C.c_void_p()
    B = M.binding
    tptr = (C.c_void_p * len(g._tw))(*g._tw)
    dptrs = [(C.c_void_p * len(t))(*t) for t in g._dw]
    dtab = (C.POINTER(C.c_void_p) * 2)(*[C.cast(p, C.POINTER(C.c_void_p)) for p in dptrs])
    dkv = (C.c_void_p * 2)(*[t.data_ptr() for t in g.kv_drafters])
    B._check(g.L.metasd_create(C.byref(h), C.byref(g.cfg), C.byref(g._tdesc_c), g._ddesc_c, tptr, dtab, None, dkv, g.workspace.data_ptr(), g.workspace.numel(),
                               torch.cuda.current_stream().cuda_stream))
    tok = np.zeros(3, np.int32)
    assert g.L.metasd_set_context(h, 0, tok.ctypes.data_as(C.c_void_p), 3, 0) == -3
    assert b"metasd_set_target_pages" in g.L.metasd_last_error(h)
    assert g.L.metasd_set_target_pages(h, None, 4, 16, None, 0) == -1
    assert g.L.metasd_set_target_pages(h, 1 << 20, 4, 17, 1 << 20, 1 << 20) == -1
    assert g.L.metasd_set_target_pages(h, 1 << 20, 4, 16, 1 << 20, 8) == -5
    g.L.metasd_destroy(h)
    g.close()
