"""ctypes binding of include/metasd.h.  Names follow the C ABI; argument marshalling only."""
from __future__ import annotations

import ctypes as C
import functools
import os

import numpy as np
import torch

HERE = os.path.dirname(os.path.abspath(__file__))
PER_LAYER = 9
MATRIX_SLOTS = (1, 2, 3, 4, 6, 7, 8)          # wq wk wv wo w_gate w_up w_down within a layer

EXPORTS = ["metasd_kv_bytes", "metasd_workspace_bytes", "metasd_pack_weight", "metasd_create", "metasd_destroy",
           "metasd_set_context", "metasd_swap_weight", "metasd_bandit_select", "metasd_bandit_update",
           "metasd_bandit_state", "metasd_draft", "metasd_verify", "metasd_accept", "metasd_draft_tree", "metasd_verify_tree", "metasd_accept_tree", "metasd_accept_logits",
           "metasd_accept_logits_noalloc", "metasd_sample_logits", "metasd_philox_words", "metasd_stream_read", "metasd_profile", "metasd_profile_read", "metasd_profile_shapes", "metasd_peek", "metasd_state", "metasd_state_seq", "metasd_accept_fallbacks", "metasd_set_drafter_head", "metasd_last_error",
           "metasd_page_bytes", "metasd_page_plan", "metasd_rope_append", "metasd_kv_rows", "metasd_attn_pages_scratch", "metasd_attn_pages", "metasd_accept_probs",
           "metasd_target_pages_bytes", "metasd_set_target_pages"]


class MetaSDError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"metasd error {code}: {msg}")
        self.code = code


class _Desc(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("d_model", C.c_int32), ("n_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("d_ffn", C.c_int32), ("vocab", C.c_int32), ("act", C.c_int32), ("dtype", C.c_int32),
                ("rms_eps", C.c_float), ("rope_theta", C.c_float)]


class _Config(C.Structure):
    _fields_ = [("K", C.c_int32), ("gamma_max", C.c_int32), ("batch", C.c_int32), ("max_ctx", C.c_int32),
                ("temperature", C.c_float), ("reward", C.c_int32), ("ucb_beta", C.c_double), ("seed", C.c_uint64),
                ("policy", C.c_int32), ("policy_window", C.c_int32), ("policy_param", C.c_double),
                ("stream_sink", C.c_int32), ("stream_window", C.c_int32), ("feature_heads", C.c_int32)]


class _Tree(C.Structure):
    _fields_ = [("n", C.c_int32), ("parent", C.c_int32 * 16), ("rank", C.c_int32 * 16)]


class _Pages(C.Structure):
    _fields_ = [("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("page", C.c_int32), ("n_pages", C.c_int32), ("pool", C.c_void_p), ("page_stride", C.c_size_t)]


class _RopeSpec(C.Structure):
    _fields_ = [("style", C.c_int32), ("rot_dim", C.c_int32), ("scaling", C.c_int32), ("orig_ctx", C.c_int32), ("theta", C.c_float),
                ("factor", C.c_float), ("low", C.c_float), ("high", C.c_float), ("gain", C.c_float)]


def lib_path() -> str:
    return os.path.join(HERE, "libmetasd.so")


_lib = None


def load_library():
    """Load libmetasd.so (built by ``paper_2604_05417_amd.build`` / ``__graft_entry__.build``)."""
    global _lib
    if _lib is not None:
        return _lib
    path = lib_path()
    if not os.path.exists(path):
        raise FileNotFoundError(f"{path} is missing: run `python -m paper_2604_05417_amd.build` (hipcc, gfx950) first")
    L = C.CDLL(path)
    vp, i32, u32, u64, f32, f64, sz, i64 = C.c_void_p, C.c_int32, C.c_uint32, C.c_uint64, C.c_float, C.c_double, C.c_size_t, C.c_int64
    sig = {
        "metasd_kv_bytes": [C.POINTER(_Desc), i32, C.POINTER(sz)],
        "metasd_workspace_bytes": [C.POINTER(_Config), C.POINTER(_Desc), C.POINTER(_Desc), C.POINTER(sz)],
        "metasd_pack_weight": [vp, vp, i32, i32, i32, vp],
        "metasd_create": [C.POINTER(vp), C.POINTER(_Config), C.POINTER(_Desc), C.POINTER(_Desc), C.POINTER(vp),
                          C.POINTER(C.POINTER(vp)), vp, C.POINTER(vp), vp, sz, vp],
        "metasd_destroy": [vp],
        "metasd_set_context": [vp, i32, vp, i32, i32],
        "metasd_swap_weight": [vp, i32, i32, vp],
        "metasd_bandit_select": [vp, i32, C.POINTER(i32)],
        "metasd_bandit_update": [vp, i32, i32, i32, i32, f64],
        "metasd_bandit_state": [vp, i32, vp, vp, C.POINTER(i32)],
        "metasd_set_drafter_head": [vp, i32, vp],
        "metasd_draft": [vp, C.POINTER(i32), i32],
        "metasd_verify": [vp, i32],
        "metasd_accept": [vp, i32, vp, vp, vp, vp],
        "metasd_draft_tree": [vp, i32, C.POINTER(_Tree)],
        "metasd_verify_tree": [vp],
        "metasd_accept_tree": [vp, C.POINTER(i32), C.POINTER(i32), vp],
        "metasd_accept_logits": [vp, vp, vp, i32, i32, i32, f32, u64, u32, u32, vp, vp, vp, vp, vp, vp],
        "metasd_accept_logits_noalloc": [vp, vp, vp, i32, i32, i32, f32, u64, u32, u32, vp, vp, vp, vp, vp],
        "metasd_sample_logits": [vp, i32, i32, f32, u64, u32, u32, u32, vp, vp],
        "metasd_philox_words": [u64, u32, i32, u32, u32, u32, vp, vp],
        "metasd_stream_read": [vp, C.c_size_t, vp, vp],
        "metasd_profile": [vp, i32],
        "metasd_profile_read": [vp, i32, C.POINTER(f64), C.POINTER(C.c_int64), C.POINTER(f64)],
        "metasd_profile_shapes": [vp, i32, i32, vp, vp, vp, vp, vp, vp, C.POINTER(i32)],
        "metasd_peek": [vp, i32, C.POINTER(vp), C.POINTER(sz)],
        "metasd_state": [vp, i32, C.POINTER(i32), C.POINTER(i32), C.POINTER(i32)],
        "metasd_state_seq": [vp, i32, i32, C.POINTER(i32), C.POINTER(i32), C.POINTER(i32)],
        "metasd_accept_fallbacks": [vp, C.POINTER(C.c_int64)],
        "metasd_target_pages_bytes": [C.POINTER(_Config), C.POINTER(_Desc), i32, i32, C.POINTER(sz), C.POINTER(sz)],
        "metasd_set_target_pages": [vp, vp, i32, i32, vp, sz],
        "metasd_page_bytes": [i32, i32, i32, C.POINTER(sz)],
        "metasd_page_plan": [vp, i32, i32, vp, vp, i32, vp, vp, vp, i32, i32, vp, vp, vp, vp, vp],
        "metasd_rope_append": [C.POINTER(_RopeSpec), C.POINTER(_Pages), i32, i32, i32, vp, i64, vp, i64, vp, i64, vp, i64, vp, vp, vp],
        "metasd_kv_rows": [C.POINTER(_Pages), vp, i32, i32, vp, vp, vp],
        "metasd_attn_pages_scratch": [i32, i32, i32, i32, i32, i32, i32, C.POINTER(sz)],
        "metasd_attn_pages": [C.POINTER(_Pages), i32, i32, i32, vp, i64, vp, i64, vp, i32, i32, vp, vp, i32, i32, f32, vp, sz, vp],
        "metasd_accept_probs": [vp, i64, i64, vp, i64, i64, vp, vp, vp, vp, i32, i32, i32, vp, vp, vp],
    }
    for name, args in sig.items():
        fn = getattr(L, name)
        fn.argtypes = args
        fn.restype = i32
    L.metasd_last_error.argtypes = [vp]
    L.metasd_last_error.restype = C.c_char_p
    _lib = L
    return L


def _check(rc: int, ctx=None):
    if rc != 0:
        raise MetaSDError(rc, load_library().metasd_last_error(ctx).decode())


def _require_gpu():
    if not torch.cuda.is_available():
        raise RuntimeError("the MetaSD library needs a GPU (MI355X); there is no CPU fallback")


def _stream_ptr(stream=None) -> int:
    s = stream if stream is not None else torch.cuda.current_stream()
    return int(s.cuda_stream)


def _desc(d: dict) -> _Desc:
    return _Desc(d["n_layers"], d["d_model"], d["n_heads"], d["n_kv_heads"], d["d_ffn"], d["vocab"], d["act"], d["dtype"],
                 d.get("rms_eps", 1e-5), d.get("rope_theta", 10000.0))


def pack_weight(w: torch.Tensor, rope_head_dim: int = 0, stream=None) -> torch.Tensor:
    """Row-major bf16 matrix [n_out, n_in] on the GPU -> streaming-tile order (same shape container).
    rope_head_dim: the head dimension for the q and k projections, 0 for every other matrix."""
    _require_gpu()
    assert w.is_cuda and w.dtype == torch.bfloat16 and w.dim() == 2 and w.is_contiguous()
    out = torch.empty_like(w)
    _check(load_library().metasd_pack_weight(out.data_ptr(), w.data_ptr(), w.shape[0], w.shape[1], rope_head_dim,
                                             _stream_ptr(stream)))
    return out


POLICIES = {"ucb": 0, "ducb": 1, "swucb": 2, "exp3": 3, "sh": 4, "random": 5}


class MetaSD:
    """One MetaSD context: a target, K drafters, their KV caches and the workspace (all torch-owned)."""

    def __init__(self, target, drafters, gamma_max: int, max_ctx: int, temperature: float, seed: int,
                 ucb_beta: float = 1.0, reward: str = "BE", device: str = "cuda:0", policy: str = "ucb",
                 policy_param: float = 0.0, policy_window: int = 0, batch: int = 1, share_target_kv: bool = False,
                 stream=None, heads=None, target_pages=None):
        """target_pages = (n_pages, page): the target's cache lies in 4-bit pages (metasd_set_target_pages): `page_pool` [n_pages, bytes of a
        page], `page_table` [batch, pages of max_ctx] int32.
        stream = (sinks, window): drafters with caches of their own keep a streaming cache (metasd_config.stream_*).
        heads = {k: W_fc [d, 2 d]}: drafter k is a head on the target's hidden states (metasd_set_drafter_head)."""
        _require_gpu()
        self.L = load_library()
        self.device = torch.device(device)
        self.K = len(drafters)
        self.gamma_max = gamma_max
        self.max_ctx = max_ctx
        self.batch = batch
        if target_pages and share_target_kv:
            raise ValueError("drafters that share the target's cache read it in bf16, not in 4-bit pages")
        self._packed = {}       # data_ptr of a row-major matrix -> packed tensor (early-exit drafters share the target's)
        self._keep = []
        tdesc, tw = target
        self.tdesc = dict(tdesc)
        self.ddescs = [dict(d) for d, _ in drafters]
        self.cfg = _Config(self.K, gamma_max, batch, max_ctx, temperature, 1 if reward == "BD" else 0, ucb_beta, seed,
                           POLICIES[policy], policy_window, policy_param, 0 if stream is None else int(stream[0]),
                           0 if stream is None else int(stream[1]), 1 if heads else 0)
        self._tdesc_c = _desc(tdesc)
        self._ddesc_c = (_Desc * self.K)(*[_desc(d) for d in self.ddescs])
        self._tw = self._table(tdesc, tw)
        self._dw = [self._table(d, w) for d, w in drafters]
        self.kv_target = None if target_pages else self._alloc_kv(self._tdesc_c, tdesc)
        # share_target_kv: a drafter whose layer tensors ARE the target's first layers (early exit) gets the target's cache
        # itself (metasd.h, "shared" strategy); every other drafter gets a cache of its own
        self.kv_shared = [share_target_kv and d["n_layers"] <= tdesc["n_layers"] and
                          all(a is b for a, b in zip(w[: 1 + PER_LAYER * d["n_layers"]], tw)) for d, w in drafters]
        self.kv_drafters = [self.kv_target if self.kv_shared[k] else self._alloc_kv(self._ddesc_c[k], self.ddescs[k]) for k in range(self.K)]
        nbytes = C.c_size_t(0)
        _check(self.L.metasd_workspace_bytes(C.byref(self.cfg), C.byref(self._tdesc_c), self._ddesc_c, C.byref(nbytes)))
        self.workspace = torch.zeros(nbytes.value, dtype=torch.uint8, device=self.device)
        self.stream = torch.cuda.current_stream(self.device)
        tptr = (C.c_void_p * len(self._tw))(*self._tw)
        dptrs = [(C.c_void_p * len(t))(*t) for t in self._dw]
        dtab = (C.POINTER(C.c_void_p) * self.K)(*[C.cast(p, C.POINTER(C.c_void_p)) for p in dptrs])
        dkv = (C.c_void_p * self.K)(*[t.data_ptr() for t in self.kv_drafters])
        h = C.c_void_p()
        torch.cuda.synchronize(self.device)
        _check(self.L.metasd_create(C.byref(h), C.byref(self.cfg), C.byref(self._tdesc_c), self._ddesc_c, tptr, dtab,
                                    None if target_pages else self.kv_target.data_ptr(), dkv, self.workspace.data_ptr(), nbytes.value,
                                    _stream_ptr(self.stream)))
        self._h = h
        if target_pages:
            n_pages, page = (int(v) for v in target_pages)
            pb, bb = C.c_size_t(0), C.c_size_t(0)
            _check(self.L.metasd_target_pages_bytes(C.byref(self.cfg), C.byref(self._tdesc_c), page, n_pages, C.byref(pb), C.byref(bb)))
            self.page_pool = torch.empty((n_pages, pb.value), dtype=torch.uint8, device=self.device)
            self._book = torch.zeros(bb.value // 4, dtype=torch.int32, device=self.device)
            width = -(-max_ctx // page)
            self.page_table = self._book[:batch * width].view(batch, width)
            torch.cuda.synchronize(self.device)
            _check(self.L.metasd_set_target_pages(self._h, self.page_pool.data_ptr(), n_pages, page, self._book.data_ptr(), bb.value), self._h)
        for k, fc in (heads or {}).items():
            want = torch.bfloat16 if tdesc["dtype"] == 1 else torch.float32
            assert fc.dtype == want and tuple(fc.shape) == (tdesc["d_model"], 2 * tdesc["d_model"])
            t = fc.to(self.device).contiguous()
            if tdesc["dtype"] == 1:
                t = pack_weight(t)
            self._keep.append(t)
            _check(self.L.metasd_set_drafter_head(self._h, int(k), t.data_ptr()), self._h)

    # ---- construction helpers
    def _prepare(self, desc, index, w):
        """Device tensor for weight-table entry `index`.  Tensors shared between tables (early-exit
        drafters reuse the target's) are uploaded, and bf16 matrices packed, once."""
        if w is None:
            return None
        want = torch.bfloat16 if desc["dtype"] == 1 else torch.float32
        assert w.dtype == want, (index, w.dtype)
        nl = desc["n_layers"]
        is_matrix = (index == 2 + PER_LAYER * nl) or (1 <= index <= PER_LAYER * nl and (index - 1) % PER_LAYER in MATRIX_SLOTS)
        pack = desc["dtype"] == 1 and is_matrix
        is_qk = 1 <= index <= PER_LAYER * nl and (index - 1) % PER_LAYER in (1, 2)
        rope_hd = desc["d_model"] // desc["n_heads"] if (pack and is_qk) else 0
        key = (w.data_ptr(), tuple(w.shape), pack, rope_hd)
        if key not in self._packed:
            dev = w.to(self.device).contiguous()
            self._packed[key] = (pack_weight(dev, rope_hd) if pack else dev, w)   # keep the source alive: the key stays unique
        return self._packed[key][0]

    def _table(self, desc, weights):
        assert len(weights) == 1 + PER_LAYER * desc["n_layers"] + 2
        out = []
        for i, w in enumerate(weights):
            t = self._prepare(desc, i, w)
            self._keep.append(t)
            out.append(None if t is None else t.data_ptr())
        return out

    def _alloc_kv(self, desc_c, desc):
        nbytes = C.c_size_t(0)
        _check(self.L.metasd_kv_bytes(C.byref(desc_c), self.max_ctx, C.byref(nbytes)))
        dt = torch.bfloat16 if desc["dtype"] == 1 else torch.float32
        hd = desc["d_model"] // desc["n_heads"]
        t = torch.zeros((self.batch, desc["n_layers"], 2, desc["n_kv_heads"], self.max_ctx, hd), dtype=dt, device=self.device)
        assert t.numel() * t.element_size() == nbytes.value * self.batch
        return t[0] if self.batch == 1 else t

    # ---- C ABI, same names
    def close(self):
        if getattr(self, "_h", None):
            torch.cuda.synchronize(self.device)
            self.L.metasd_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def set_context(self, tokens, kv_prefilled: bool = False, seq: int = 0):
        tok = np.ascontiguousarray(tokens, np.int32)
        _check(self.L.metasd_set_context(self._h, seq, tok.ctypes.data_as(C.c_void_p), tok.shape[0], int(kv_prefilled)), self._h)

    def swap_weight(self, model: int, index: int, tensor: torch.Tensor):
        """tensor must already be in device layout (bf16 matrices: packed with pack_weight)."""
        self._keep.append(tensor)
        _check(self.L.metasd_swap_weight(self._h, model, index, tensor.data_ptr()), self._h)

    def bandit_select(self, seq: int = 0) -> int:
        k = C.c_int32(-1)
        _check(self.L.metasd_bandit_select(self._h, seq, C.byref(k)), self._h)
        return int(k.value)

    def bandit_update(self, k: int, n_acc: int, gamma: int, bd_reward: float = float("nan"), seq: int = 0):
        _check(self.L.metasd_bandit_update(self._h, seq, k, n_acc, gamma, bd_reward), self._h)

    def bandit_state(self, seq: int = 0):
        mu = np.zeros(self.K, np.float64)
        n = np.zeros(self.K, np.int32)
        t = C.c_int32(0)
        _check(self.L.metasd_bandit_state(self._h, seq, mu.ctypes.data_as(C.c_void_p), n.ctypes.data_as(C.c_void_p), C.byref(t)))
        return mu, n, int(t.value)

    def draft(self, k, gamma: int):
        """k: the arm (batch 1) or one arm per sequence."""
        ks = [k] * self.batch if np.isscalar(k) else list(k)
        assert len(ks) == self.batch
        kk = (C.c_int32 * self.batch)(*[int(v) for v in ks])
        _check(self.L.metasd_draft(self._h, kk, gamma), self._h)

    def verify(self, gamma: int):
        _check(self.L.metasd_verify(self._h, gamma), self._h)

    def accept(self, gamma: int):
        """batch 1: (n_acc, token, mask, bd); otherwise four arrays of `batch` entries."""
        B = self.batch
        n, tok, mask, bd = np.zeros(B, np.int32), np.zeros(B, np.int32), np.zeros(B, np.uint32), np.zeros(B, np.float64)
        _check(self.L.metasd_accept(self._h, gamma, n.ctypes.data_as(C.c_void_p), tok.ctypes.data_as(C.c_void_p),
                                    mask.ctypes.data_as(C.c_void_p), bd.ctypes.data_as(C.c_void_p)), self._h)
        if B == 1:
            return int(n[0]), int(tok[0]), int(mask[0]), float(bd[0])
        return n, tok, mask, bd

    # ---- tree rounds (greedy for temperature 0, sampled otherwise): parent[i], rank[i] per node, node 0 the root
    def draft_tree(self, k: int, parent, rank):
        n = len(parent)
        assert len(rank) == n and n <= 16
        t = _Tree(n, (C.c_int32 * 16)(*[int(v) for v in parent]), (C.c_int32 * 16)(*[int(v) for v in rank]))
        _check(self.L.metasd_draft_tree(self._h, k, C.byref(t)), self._h)

    def verify_tree(self):
        _check(self.L.metasd_verify_tree(self._h), self._h)

    def accept_tree(self):
        """(n_acc, token, path): path = the accepted nodes."""
        n, tok = C.c_int32(0), C.c_int32(0)
        path = np.zeros(16, np.int32)
        _check(self.L.metasd_accept_tree(self._h, C.byref(n), C.byref(tok), path.ctypes.data_as(C.c_void_p)), self._h)
        return int(n.value), int(tok.value), [int(v) for v in path[: n.value]]

    def peek(self, what: str, gamma: int | None = None) -> torch.Tensor:
        """View of an internal device buffer: 'P' [gamma_max+1, V], 'Q' [gamma_max, V], 'hist' [max_ctx], 'bd' [gamma_max],
        'draft' [gamma_max].  batch > 1: pass the gamma of the last round; the views are P [batch, gamma+1, V],
        Q [batch, gamma, V], hist [batch, max_ctx], bd / draft [batch, gamma]."""
        code = {"P": 0, "Q": 1, "hist": 2, "bd": 3, "draft": 4, "feat": 5}[what]
        p, n = C.c_void_p(), C.c_size_t(0)
        _check(self.L.metasd_peek(self._h, code, C.byref(p), C.byref(n)), self._h)
        off = p.value - self.workspace.data_ptr()
        raw = self.workspace[off: off + n.value]
        V = self.tdesc["vocab"]
        if what == "feat":
            return raw.view(torch.float32).view(self.max_ctx, self.tdesc["d_model"])
        if self.batch > 1:
            B, g = self.batch, gamma
            if what == "hist":
                return raw.view(torch.int32).view(B, self.max_ctx)
            assert g is not None
            if what == "P":
                return raw.view(torch.float32)[: B * (g + 1) * V].view(B, g + 1, V)
            if what == "Q":
                return raw.view(torch.float32)[: B * g * V].view(B, g, V)
            if what == "draft":
                return raw.view(torch.int32)[: B * g].view(B, g)
            return raw.view(torch.float64)[: B * g].view(B, g)
        if what == "P":
            return raw.view(torch.float32).view(self.gamma_max + 1, V)
        if what == "Q":
            return raw.view(torch.float32).view(self.gamma_max, V)
        if what in ("hist", "draft"):
            return raw.view(torch.int32)
        return raw.view(torch.float64)

    def profile(self, max_records: int):
        _check(self.L.metasd_profile(self._h, max_records), self._h)

    def profile_read(self, kind: str) -> dict:
        ms, n, by = C.c_double(0), C.c_int64(0), C.c_double(0)
        _check(self.L.metasd_profile_read(self._h, {"gemm": 0, "attn": 1, "accept": 2}[kind], C.byref(ms), C.byref(n), C.byref(by)), self._h)
        return dict(ms=ms.value, launches=n.value, bytes=by.value)

    def profile_shapes(self, target_only: bool = True, max_rows: int = 64) -> list:
        """Recorded GEMM launches by shape: dicts N, K, m, launches, avg_us, bytes_per_launch, GBs."""
        n, k, m = (np.zeros(max_rows, np.int32) for _ in range(3))
        ms, by, cnt = np.zeros(max_rows, np.float64), np.zeros(max_rows, np.float64), np.zeros(max_rows, np.int64)
        rows = C.c_int32(0)
        vp = lambda a: a.ctypes.data_as(C.c_void_p)
        _check(self.L.metasd_profile_shapes(self._h, int(target_only), max_rows, vp(n), vp(k), vp(m), vp(ms), vp(cnt), vp(by), C.byref(rows)), self._h)
        out = []
        for i in range(rows.value):
            out.append(dict(N=int(n[i]), K=int(k[i]), m=int(m[i]), launches=int(cnt[i]), avg_us=ms[i] / cnt[i] * 1e3,
                            bytes_per_launch=by[i] / cnt[i], GBs=by[i] / (ms[i] * 1e-3) / 1e9 if ms[i] > 0 else 0.0))
        return out

    def state(self, model: int = -1, seq: int = 0):
        l, kv, r = C.c_int32(0), C.c_int32(0), C.c_int32(0)
        _check(self.L.metasd_state_seq(self._h, seq, model, C.byref(l), C.byref(kv), C.byref(r)))
        return int(l.value), int(kv.value), int(r.value)

    def accept_fallbacks(self) -> int:
        n = C.c_int64(0)
        _check(self.L.metasd_accept_fallbacks(self._h, C.byref(n)))
        return int(n.value)

    # ---- convenience: one full round (select -> draft -> verify -> accept -> update)
    def round(self, gamma: int, k: int | None = None):
        kk = self.bandit_select()
        if k is not None:
            kk = k
        self.draft(kk, gamma)
        self.verify(gamma)
        n, tok, mask, bd = self.accept(gamma)
        self.bandit_update(kk, n, gamma, bd)
        return kk, n, tok, mask, bd


# ---- stand-alone kernels on caller-supplied logits

def accept_logits(P: torch.Tensor, Q: torch.Tensor, d: torch.Tensor, T: float, seed: int, rnd: int = 0, seq0: int = 0,
                  out=None, stream=None) -> dict:
    """P [rows, gamma+1, V], Q [rows, gamma, V] fp32, d [rows, gamma] int32 (all CUDA, contiguous)."""
    _require_gpu()
    rows, gamma, V = Q.shape
    assert P.shape == (rows, gamma + 1, V) and d.shape == (rows, gamma)
    assert P.is_cuda and Q.is_cuda and d.is_cuda and P.is_contiguous() and Q.is_contiguous() and d.is_contiguous()
    assert P.dtype == torch.float32 and Q.dtype == torch.float32 and d.dtype == torch.int32
    if out is None:
        dev = P.device
        out = dict(n_acc=torch.empty(rows, dtype=torch.int32, device=dev), token=torch.empty(rows, dtype=torch.int32, device=dev),
                   mask=torch.empty(rows, dtype=torch.int32, device=dev), bd=torch.empty((rows, gamma), dtype=torch.float64, device=dev),
                   scratch=torch.zeros(rows * (gamma + 1) * 336, dtype=torch.uint8, device=dev))   # zero-filled once, reusable
    _check(load_library().metasd_accept_logits(P.data_ptr(), Q.data_ptr(), d.data_ptr(), rows, gamma, V, T, seed, rnd, seq0,
                                               out["n_acc"].data_ptr(), out["token"].data_ptr(), out["mask"].data_ptr(),
                                               out["bd"].data_ptr(), out["scratch"].data_ptr(), _stream_ptr(stream)))
    return out


ACCEPT_NOALLOC_MAX_ITEMS = 4096


def accept_logits_noalloc(P: torch.Tensor, Q: torch.Tensor, d: torch.Tensor, T: float, seed: int, rnd: int, seq0: int, out: dict,
                          stream=None) -> dict:
    """metasd_accept_logits_noalloc: the caller passes inputs and the output tensors (out: n_acc, token, mask int32 [rows],
    bd float64 [rows, gamma]); the binding allocates nothing either."""
    _require_gpu()
    rows, gamma, V = Q.shape
    assert P.shape == (rows, gamma + 1, V) and d.shape == (rows, gamma)
    assert P.is_cuda and Q.is_cuda and d.is_cuda and P.is_contiguous() and Q.is_contiguous() and d.is_contiguous()
    assert P.dtype == torch.float32 and Q.dtype == torch.float32 and d.dtype == torch.int32
    _check(load_library().metasd_accept_logits_noalloc(P.data_ptr(), Q.data_ptr(), d.data_ptr(), rows, gamma, V, T, seed, rnd, seq0,
                                                       out["n_acc"].data_ptr(), out["token"].data_ptr(), out["mask"].data_ptr(),
                                                       out["bd"].data_ptr(), _stream_ptr(stream)))
    return out


def sample_logits(logits: torch.Tensor, T: float, seed: int, rnd: int = 0, pos: int = 0, seq0: int = 0, stream=None):
    _require_gpu()
    rows, V = logits.shape
    assert logits.is_cuda and logits.is_contiguous() and logits.dtype == torch.float32
    tok = torch.empty(rows, dtype=torch.int32, device=logits.device)
    _check(load_library().metasd_sample_logits(logits.data_ptr(), rows, V, T, seed, rnd, pos, seq0, tok.data_ptr(), _stream_ptr(stream)))
    return tok


STREAM_READ_SINK_WORDS = 8192


def stream_read(src: torch.Tensor, sink: torch.Tensor) -> None:
    """One plain streaming read of `src` (CUDA, contiguous) on the current stream; `sink`: int32 tensor of at least
    STREAM_READ_SINK_WORDS elements.  Asynchronous: time it with events."""
    _require_gpu()
    assert src.is_cuda and src.is_contiguous() and sink.is_cuda and sink.is_contiguous()
    assert sink.numel() * sink.element_size() >= 4 * STREAM_READ_SINK_WORDS
    _check(load_library().metasd_stream_read(src.data_ptr(), src.numel() * src.element_size(), sink.data_ptr(), _stream_ptr()))


def philox_words(seed: int, c0_start: int, n: int, c1: int, c2: int, c3: int, device="cuda:0") -> torch.Tensor:
    _require_gpu()
    out = torch.empty((n, 4), dtype=torch.int32, device=device)
    _check(load_library().metasd_philox_words(seed, c0_start, n, c1, c2, c3, out.data_ptr(), _stream_ptr()))
    return out


# ---- requests whose K and V lie in 4-bit pages (metasd.h): every array is a CUDA tensor of the caller's, all on one device

_DTYPES = {torch.float32: 0, torch.bfloat16: 1}


# The host's part of a small call is what bounds it, so what these wrappers ask for is asked for the short way: the current stream's handle by
# device index (torch.cuda.current_stream() builds an object for it, 2.8 us of a call that takes 8 in all), outputs like a tensor that is at hand
# (1.3 - 1.6 us, torch.empty 1.9).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda device: torch.cuda.current_stream(device).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _on(first: torch.Tensor, ints) -> int:
    """The stream to launch on: the current one of the tensors' device, which has to be the current device.  ints: contiguous int32 there."""
    dev = first.get_device()
    if dev < 0:
        raise ValueError("tensors on a GPU are needed; there is no CPU fallback")
    for t in ints:
        if t.dtype is not torch.int32 or t.get_device() != dev or not t.is_contiguous():
            raise ValueError(f"contiguous int32 on {first.device} expected, got {t.dtype} {tuple(t.shape)} on {t.device}")
    if dev != _current_device():
        raise ValueError(f"the tensors are on {first.device}, which is not the current device")
    return _raw_stream(dev)


def _rows3(name: str, x: torch.Tensor, rows: int, heads, hd: int, dtype, dev: int) -> int:
    """Elements between the rows of x: [rows, heads, hd] or [rows, heads * hd], heads next to each other.  heads None: any number of them."""
    shape, stride = x.shape, x.stride()
    if len(shape) == 2:
        wide, ok = shape[1], stride[1] == 1
    elif len(shape) == 3:
        wide, ok = shape[1] * hd, shape[2] == hd and stride[2] == 1 and (stride[1] == hd or shape[1] == 1)
    else:
        wide, ok = 0, False
    if not ok or shape[0] != rows or wide == 0 or (wide % hd if heads is None else wide != heads * hd) or x.dtype is not dtype or x.get_device() != dev:
        raise ValueError(f"{name}: {rows} rows of {'' if heads is None else heads} heads of {hd}, {dtype} on cuda:{dev}, heads next to each other; got {tuple(shape)} {x.dtype}")
    return stride[0] if rows > 1 else wide


def _pages(pool: torch.Tensor, page: int, n_kv_heads: int, head_dim: int) -> _Pages:
    """pool: uint8 [n_pages, bytes of a page], pages any stride apart."""
    shape, stride = pool.shape, pool.stride()
    if pool.dtype is not torch.uint8 or len(shape) != 2 or stride[1] != 1 or shape[1] < n_kv_heads * (page // 16) * 17 * head_dim:
        raise ValueError(f"pool: uint8 [n_pages, page_bytes] with contiguous pages expected, got {pool.dtype} {tuple(shape)}")
    return _Pages(n_kv_heads, head_dim, page, shape[0], pool.data_ptr(), stride[0] if shape[0] > 1 else shape[1])


class Rope:
    """How heads are rotated (metasd_rope): style "half" or "pairs", scaling "none", "linear", "wave" or "index"."""
    __slots__ = ("c",)

    def __init__(self, style: str = "half", rot_dim: int = 0, theta: float = 10000.0, scaling: str = "none", factor: float = 1.0, low: float = 1.0,
                 high: float = 4.0, orig_ctx: int = 4096, gain: float = 1.0):
        self.c = _RopeSpec({"half": 0, "pairs": 1}[style], rot_dim, {"none": 0, "linear": 1, "wave": 2, "index": 3}[scaling], orig_ctx, theta, factor, low, high, gain)


def page_bytes(n_kv_heads: int, head_dim: int, page: int) -> int:
    n = C.c_size_t(0)
    _check(load_library().metasd_page_bytes(n_kv_heads, head_dim, page, C.byref(n)))
    return int(n.value)


def page_plan(table: torch.Tensor, held: torch.Tensor, ring: torch.Tensor, state: torch.Tensor, lens: torch.Tensor, n_new: torch.Tensor, page: int,
              rows: int, out=None) -> dict:
    """metasd_page_plan: table [batch, width], held [batch], ring [n_pages] and state [4] are updated in place.  Returns slots and pos [rows],
    start [batch + 1], served [batch] (out: the same dict, reused)."""
    st = _on(table, (table, held, ring, state, lens, n_new))
    B, width = table.shape
    if held.numel() != B or lens.numel() != B or n_new.numel() != B or state.numel() < 4:
        raise ValueError("page_plan: held, lens and n_new have one entry per request, state four")
    if out is None:
        buf = table.new_empty(2 * rows + 2 * B + 1)
        slots, pos, start, served = torch.split_with_sizes(buf, (rows, rows, B + 1, B))
        out = dict(slots=slots, pos=pos, start=start, served=served)
    else:
        _on(table, (out["slots"], out["pos"], out["start"], out["served"]))
        if out["slots"].numel() < rows or out["pos"].numel() < rows or out["start"].numel() < B + 1 or out["served"].numel() < B:
            raise ValueError("page_plan: out is too small")
    _check(load_library().metasd_page_plan(table.data_ptr(), B, width, held.data_ptr(), ring.data_ptr(), ring.numel(), state.data_ptr(), lens.data_ptr(), n_new.data_ptr(),
                                           page, rows, out["slots"].data_ptr(), out["pos"].data_ptr(), out["start"].data_ptr(), out["served"].data_ptr(), st))
    return out


def rope_append(q, k, v, pos: torch.Tensor, slots, pool, page: int, n_kv_heads: int, head_dim: int, rope: Rope, out=None):
    """metasd_rope_append: q [rows, n_heads (,) head_dim] rotated (returned, [rows, n_heads, head_dim]); k rotated and v appended to the pool at
    `slots`.  q may be None, or k, v, slots and pool."""
    lead = q if q is not None else k
    if lead is None or (k is not None and (v is None or slots is None or pool is None)):
        raise ValueError("rope_append: q, or k with v, slots and pool, or both")
    st = _on(lead, (pos,) if k is None else (pos, slots))
    rows, dtype, dev = lead.shape[0], lead.dtype, lead.get_device()
    if rows == 0:                                       # nothing to do
        return out if out is not None or q is None else q.new_empty((0, q.shape[1] if q.dim() == 3 else q.shape[1] // head_dim, head_dim))
    if pos.numel() != rows or (k is not None and slots.numel() != rows):
        raise ValueError("rope_append: one position and one slot per row")
    H = ldq = ldo = ldk = ldv = 0
    if q is not None:
        ldq = _rows3("q", q, rows, None, head_dim, dtype, dev)
        H = q.numel() // (rows * head_dim)
        if out is None:
            out, ldo = q.new_empty((rows, H, head_dim)), H * head_dim
        else:
            ldo = _rows3("out", out, rows, H, head_dim, dtype, dev)
    if k is not None:
        ldk, ldv = _rows3("k", k, rows, n_kv_heads, head_dim, dtype, dev), _rows3("v", v, rows, n_kv_heads, head_dim, dtype, dev)
        if pool.get_device() != dev:
            raise ValueError(f"pool is on {pool.device}")
        pages = _pages(pool, page, n_kv_heads, head_dim)
    else:
        pages = _Pages(n_kv_heads, head_dim, page, 0, None, 0)
    qp, op = (None, None) if q is None else (q.data_ptr(), out.data_ptr())
    kp, vp, sp = (None, None, None) if k is None else (k.data_ptr(), v.data_ptr(), slots.data_ptr())
    _check(load_library().metasd_rope_append(C.byref(rope.c), C.byref(pages), _DTYPES.get(dtype, -1), rows, H, qp, ldq, op, ldo, kp, ldk, vp, ldv, pos.data_ptr(), sp, st))
    return out


def kv_rows(pool: torch.Tensor, slots: torch.Tensor, page: int, n_kv_heads: int, head_dim: int, dtype=torch.float32):
    """metasd_kv_rows: the values held at the slots, k and v [rows, n_kv_heads, head_dim]."""
    st = _on(pool, (slots,))
    pages = _pages(pool, page, n_kv_heads, head_dim)
    rows = slots.numel()
    k = torch.empty((rows, n_kv_heads, head_dim), dtype=dtype, device=pool.device)
    v = torch.empty_like(k)
    if rows == 0:
        return k, v
    _check(load_library().metasd_kv_rows(C.byref(pages), slots.data_ptr(), rows, _DTYPES.get(dtype, -1), k.data_ptr(), v.data_ptr(), st))
    return k, v


@functools.lru_cache(maxsize=256)
def _attn_scratch(batch, H, KH, hd, dtype, max_new, max_len, device) -> int:
    n = C.c_size_t(0)
    _check(load_library().metasd_attn_pages_scratch(batch, H, KH, hd, dtype, max_new, max_len, C.byref(n)))
    return int(n.value)


def attn_pages(q: torch.Tensor, pool: torch.Tensor, table: torch.Tensor, start: torch.Tensor, lens: torch.Tensor, page: int, n_kv_heads: int, scale: float,
               max_new: int, max_len: int, out=None) -> torch.Tensor:
    """metasd_attn_pages: q [rows, n_heads, head_dim]; request b's rows are start[b] .. start[b + 1] - 1, its lens[b] positions in the pages
    table[b].  Rows of a new `out` behind the last request are not written."""
    st = _on(q, (table, start, lens))
    rows, H, hd = q.shape
    B, width = table.shape
    dtype, dev = q.dtype, q.get_device()
    if start.numel() != B + 1 or lens.numel() != B or pool.get_device() != dev:
        raise ValueError("attn_pages: start has batch + 1 entries, lens batch, the pool is on the same device")
    ldo = H * hd
    if out is None:
        out = torch.empty_like(q) if q.is_contiguous() else q.new_empty((rows, H, hd))
    elif rows:
        ldo = _rows3("out", out, rows, H, hd, dtype, dev)
    if rows == 0:
        return out
    dt, ldq = _DTYPES.get(dtype, -1), _rows3("q", q, rows, H, hd, dtype, dev)
    pages = _pages(pool, page, n_kv_heads, hd)
    n = _attn_scratch(B, H, n_kv_heads, hd, dt, max_new, max_len, dev)
    scratch = torch.empty(n, dtype=torch.uint8, device=q.device) if n else None
    _check(load_library().metasd_attn_pages(C.byref(pages), dt, rows, H, q.data_ptr(), ldq, out.data_ptr(), ldo, table.data_ptr(), B, width, start.data_ptr(), lens.data_ptr(),
                                            max_new, max_len, scale, scratch.data_ptr() if n else None, n, st))
    return out


def accept_probs(P: torch.Tensor, Q, d: torch.Tensor, n_draft, u: torch.Tensor, w: torch.Tensor, out=None) -> dict:
    """metasd_accept_probs: P [rows, gamma + 1, V] and Q [rows, gamma, V] (or None) fp32 probabilities, d [rows, gamma] int32, n_draft [rows] int32
    (or None), u [rows, gamma] and w [rows] fp32.  Returns n_acc [rows] and tokens [rows, gamma + 1] int32."""
    st = _on(P, (d,) if n_draft is None else (d, n_draft))
    rows, g1, V = P.shape
    if d.shape != (rows, g1 - 1) or u.shape != d.shape or w.shape != (rows,) or (n_draft is not None and n_draft.shape != (rows,)) or (Q is not None and Q.shape != (rows, g1 - 1, V)):
        raise ValueError("accept_probs: P [rows, gamma + 1, V], Q [rows, gamma, V], d and u [rows, gamma], w and n_draft [rows]")
    dev = P.get_device()
    for t in (P, u, w) if Q is None else (P, Q, u, w):
        if t.dtype is not torch.float32 or t.get_device() != dev or (t.stride(-1) != 1 and t.shape[-1] > 1):
            raise ValueError("accept_probs: fp32 on one device, the last dimension contiguous")
    if not (u.is_contiguous() and w.is_contiguous()):
        raise ValueError("accept_probs: u and w contiguous")
    if out is None:
        n_acc, tokens = d.new_empty(rows), d.new_empty((rows, g1))
        out = dict(n_acc=n_acc, tokens=tokens)
    else:
        n_acc, tokens = out["n_acc"], out["tokens"]
        _on(P, (n_acc, tokens))
        if n_acc.numel() < rows or tokens.numel() < rows * g1:
            raise ValueError("accept_probs: out is too small")
    if rows == 0:
        return out
    ps, qs = P.stride(), (0, 0) if Q is None else Q.stride()
    _check(load_library().metasd_accept_probs(P.data_ptr(), ps[0], ps[1], None if Q is None else Q.data_ptr(), qs[0], qs[1], d.data_ptr(),
                                              None if n_draft is None else n_draft.data_ptr(), u.data_ptr(), w.data_ptr(), rows, g1 - 1, V, n_acc.data_ptr(),
                                              tokens.data_ptr(), st))
    return out
