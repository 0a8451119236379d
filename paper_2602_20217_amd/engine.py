"""Device-side model and call helpers over the C ABI.

PyTorch supplies device memory and the stream; every computation runs in
libknapspec's HIP kernels.  ``DeviceModel`` uploads row-major weights, packs
them into the kernels' layout with ``ks_pack_matrix`` / ``ks_pack_gate_up``,
allocates the KV cache and workspace, and exposes the decode-step calls.
"""
from __future__ import annotations

import ctypes as C
import math

import numpy as np
import torch

from . import _lib as K

_PER_LAYER = ("wq", "wk", "wv", "wo", "w_gate", "w_up", "w_down")


def _ptr(t: torch.Tensor) -> int:
    return t.data_ptr()


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


def _bf16_bits(a: np.ndarray) -> np.ndarray:
    u = np.ascontiguousarray(a, dtype=np.float32).view(np.uint32)
    if np.any(u & 0xFFFF):
        raise ValueError("bf16 model weights must hold exactly representable bf16 values")
    return (u >> 16).astype(np.uint16)


def select_params(c, quant_mode="paper_min", bins=0, tau=0.5, prune_half=True, D=10,
                  t_head=0.0):
    return K.SelectParams(float(c[0]), float(c[1]), float(c[2]),
                          K.KS_QUANT_BINS if quant_mode == "bins" else K.KS_QUANT_PAPER_MIN,
                          int(bins), float(tau), 1 if prune_half else 0, int(D), float(t_head))


class DeviceModel:
    """One decoder on one GPU behind a ks_ctx.

    cfg needs attributes L, d, hq, hkv, hd, ffn, vocab, eps, rope_theta, qk_norm,
    dtype ("f32" or "bf16").  Call ``upload(kind, layer, array)`` for every weight
    (kinds embed, lm_head, wq, wk, wv, wo, w_gate, w_up, w_down; row-major [out, in]
    float32 arrays, bf16-valued for bf16 models), then ``finalize()``.

    cache: "flat" (the model's type, contiguous), or pages of 64 tokens of "bf16" or
    of "e4m3" (8 bits, a scale for every 16 tokens and head: half the bytes of bf16);
    ``use_paged`` gives the context other pages.
    """

    def __init__(self, cfg, n_max: int, gamma_max: int = 8, m_rounds: int = 5,
                 cap_max: int = 256, prefill_chunk: int = 256, device: str = "cuda:0",
                 cache: str = "flat"):
        _need(cache in ("flat", "bf16", "e4m3"), "cache must be 'flat', 'bf16' or 'e4m3'")
        self.cfg = cfg
        self.dev = torch.device(device)
        self.bf = cfg.dtype == "bf16"
        self.desc = K.ModelDesc(cfg.L, cfg.d, cfg.hq, cfg.hkv, cfg.hd, cfg.ffn, cfg.vocab,
                                n_max, 1 if cfg.qk_norm else 0,
                                K.KS_BF16 if self.bf else K.KS_F32, float(cfg.eps),
                                float(cfg.rope_theta))
        self.lim = K.Limits(gamma_max, m_rounds, cap_max, prefill_chunk)
        kvb = K.ks_kv_cache_bytes(C.byref(self.desc))
        wsb = K.ks_workspace_bytes(C.byref(self.desc), C.byref(self.lim))
        if kvb == 0 or wsb == 0:
            raise K.KsError(K.KS_EINVAL, K.last_error())
        self._cache_kind = cache
        self.kv = torch.zeros(kvb if cache == "flat" else 0, dtype=torch.uint8, device=self.dev)
        self.ws = torch.zeros(wsb, dtype=torch.uint8, device=self.dev)
        wdt = torch.int16 if self.bf else torch.float32
        L, d = cfg.L, cfg.d
        nq = (cfg.hq + 2 * cfg.hkv) * cfg.hd
        e = lambda *s: torch.empty(*s, dtype=wdt, device=self.dev)
        self.w = {
            "embed": e(cfg.vocab, d), "lm_head": e(cfg.vocab, d),
            "wqkv": [e(nq, d) for _ in range(L)], "wo": [e(d, cfg.hq * cfg.hd) for _ in range(L)],
            "w_gate_up": [e(2 * cfg.ffn, d) for _ in range(L)],
            "w_down": [e(d, cfg.ffn) for _ in range(L)],
        }
        ones = lambda n: torch.ones(n, dtype=torch.float32, device=self.dev)
        self.gains = {"final_norm": ones(d), "attn_norm": [ones(d) for _ in range(L)],
                      "mlp_norm": [ones(d) for _ in range(L)],
                      "q_norm": [ones(cfg.hd) for _ in range(L)],
                      "k_norm": [ones(cfg.hd) for _ in range(L)]}
        self._pending = {}
        self._done = set()
        self.ctx = None

    # ------------------------------------------------------------ weights
    def _to_dev(self, a: np.ndarray) -> torch.Tensor:
        if self.bf:
            return torch.from_numpy(_bf16_bits(a).view(np.int16)).to(self.dev)
        return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(self.dev)

    def _pack(self, src: torch.Tensor, dst: torch.Tensor):
        N, Kd = src.shape
        K.ks_pack_matrix(_ptr(src), _ptr(dst), N, Kd, self.desc.dtype, _stream())

    def upload(self, kind: str, layer: int, a: np.ndarray):
        if kind == "embed":
            self.w["embed"].copy_(self._to_dev(a))
        elif kind == "lm_head":
            self._pack(self._to_dev(a), self.w["lm_head"])
        elif kind in ("wq", "wk", "wv"):
            p = self._pending.setdefault(("qkv", layer), {})
            p[kind] = a
            if len(p) == 3:
                cat = self._to_dev(np.concatenate([p["wq"], p["wk"], p["wv"]], axis=0))
                c = self.cfg
                K.ks_pack_qkv(_ptr(cat), _ptr(self.w["wqkv"][layer]), c.hq, c.hkv, c.hd, c.d,
                              self.desc.dtype, _stream())
                torch.cuda.current_stream().synchronize()
                del self._pending[("qkv", layer)]
        elif kind == "wo":
            self._pack(self._to_dev(a), self.w["wo"][layer])
        elif kind in ("w_gate", "w_up"):
            p = self._pending.setdefault(("gu", layer), {})
            p[kind] = self._to_dev(a)
            if len(p) == 2:
                K.ks_pack_gate_up(_ptr(p["w_gate"]), _ptr(p["w_up"]),
                                  _ptr(self.w["w_gate_up"][layer]), self.cfg.ffn, self.cfg.d,
                                  self.desc.dtype, _stream())
                torch.cuda.current_stream().synchronize()
                del self._pending[("gu", layer)]
        elif kind == "w_down":
            self._pack(self._to_dev(a), self.w["w_down"][layer])
        else:
            raise KeyError(kind)
        self._done.add((kind, layer))

    def upload_all(self, weights: dict):
        for (kind, layer), a in weights.items():
            self.upload(kind, layer, a)
        return self.finalize()

    def finalize(self):
        need = 2 + 7 * self.cfg.L
        if len(self._done) != need or self._pending:
            raise RuntimeError(f"uploaded {len(self._done)} of {need} weight tensors")
        torch.cuda.current_stream().synchronize()
        L = self.cfg.L
        arr = lambda ts: (C.c_void_p * L)(*[_ptr(t) for t in ts])
        self._arrays = {k: arr(self.w[k]) for k in ("wqkv", "wo", "w_gate_up", "w_down")}
        self._arrays.update({k: arr(self.gains[k]) for k in
                             ("attn_norm", "mlp_norm", "q_norm", "k_norm")})
        A = self._arrays
        cast = lambda x: C.cast(x, C.POINTER(C.c_void_p))
        self.weights = K.Weights(_ptr(self.w["embed"]), _ptr(self.w["lm_head"]),
                                 _ptr(self.gains["final_norm"]), cast(A["attn_norm"]),
                                 cast(A["wqkv"]), cast(A["wo"]), cast(A["q_norm"]),
                                 cast(A["k_norm"]), cast(A["mlp_norm"]), cast(A["w_gate_up"]),
                                 cast(A["w_down"]))
        ctx = C.c_void_p()
        K.ks_create(C.byref(self.desc), C.byref(self.lim), C.byref(self.weights),
                    _ptr(self.kv) or None, self.kv.numel(), _ptr(self.ws), self.ws.numel(),
                    _stream(), C.byref(ctx))
        self.ctx = ctx
        if self._cache_kind != "flat":
            n = (self.desc.n_max + 63) // 64
            self.use_paged([PagedCache(n, 64, self.cfg.hkv, self.cfg.hd, self._cache_kind,
                                       device=self.dev) for _ in range(self.cfg.L)],
                           torch.arange(n, dtype=torch.int32, device=self.dev))
        torch.cuda.current_stream().synchronize()
        return self

    def resized(self, n_max: int) -> "DeviceModel":
        """A second context over the same uploaded weights, with its own KV cache
        of n_max positions and workspace (the decode attention splits follow the
        cache size, so a deployment sizes the cache to its context)."""
        if self.ctx is None:
            raise RuntimeError("finalize() the weights first")
        other = DeviceModel.__new__(DeviceModel)
        other.cfg, other.dev, other.bf = self.cfg, self.dev, self.bf
        d = self.desc
        other.desc = K.ModelDesc(d.L, d.d, d.hq, d.hkv, d.hd, d.ffn, d.vocab, n_max, d.qk_norm,
                                 d.dtype, d.eps, d.rope_theta)
        other.lim = self.lim
        kvb = K.ks_kv_cache_bytes(C.byref(other.desc))
        wsb = K.ks_workspace_bytes(C.byref(other.desc), C.byref(other.lim))
        if kvb == 0 or wsb == 0:
            raise K.KsError(K.KS_EINVAL, K.last_error())
        other._cache_kind = self._cache_kind
        other.kv = torch.zeros(kvb if self._cache_kind == "flat" else 0, dtype=torch.uint8,
                               device=self.dev)
        other.ws = torch.zeros(wsb, dtype=torch.uint8, device=self.dev)
        other.w, other.gains = self.w, self.gains
        other._pending, other._done = {}, set(self._done)
        other.ctx = None
        return other.finalize()

    def close(self):
        if self.ctx is not None:
            K.ks_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ------------------------------------------------------------ cache views
    def kv_layer(self, layer: int):
        """(K, V) views [hkv, n_max, hd] of one layer's cache (bf16 or float32)."""
        c = self.cfg
        es = 2 if self.bf else 4
        n = c.hkv * self.desc.n_max * c.hd * es
        base = 2 * layer * n
        dt = torch.bfloat16 if self.bf else torch.float32
        kk = self.kv[base:base + n].view(dt).view(c.hkv, self.desc.n_max, c.hd)
        vv = self.kv[base + n:base + 2 * n].view(dt).view(c.hkv, self.desc.n_max, c.hd)
        return kk, vv

    def use_paged(self, layers, table: torch.Tensor):
        """Keys and values in pages from now on (see ks_use_paged): layers, one
        PagedCache each, and the int32 table of the sequence's pages, n_max positions
        at least.  layers = None: back to the flat cache."""
        if layers is None:
            K.ks_use_paged(self.ctx, None, None, 0)
            self.pages = self.page_table = None
            return
        if len(layers) != self.cfg.L or any(c.device != self.dev for c in layers):
            raise ValueError("one PagedCache per layer, on the model's device")
        if (table.dim() != 1 or table.dtype != torch.int32 or not table.is_contiguous()
                or table.device != self.dev):
            raise ValueError("table must be a dense int32 vector on the model's device")
        arr = (K.PagedCache * len(layers))(*[c.desc for c in layers])
        K.ks_use_paged(self.ctx, arr, _ptr(table), table.numel())
        self.pages, self.page_table = list(layers), table  # kept alive

    # ------------------------------------------------------------ decode calls
    def prefill(self, tokens) -> int:
        t = np.ascontiguousarray(tokens, dtype=np.int32)
        out = C.c_int32()
        K.ks_prefill(self.ctx, t.ctypes.data, len(t), C.byref(out))
        return out.value

    def set_context(self, n_cached: int, last_token: int):
        K.ks_set_context(self.ctx, int(n_cached), int(last_token))

    def draft_step(self, exec_mask):
        m = np.ascontiguousarray(np.asarray(exec_mask, dtype=bool).astype(np.uint8))
        tok, p = C.c_int32(), C.c_float()
        K.ks_draft_step(self.ctx, m.ctypes.data, C.byref(tok), C.byref(p))
        return tok.value, p.value

    def verify(self, tokens):
        t = np.ascontiguousarray(tokens, dtype=np.int32)
        pred = np.zeros(len(t), dtype=np.int32)
        a = C.c_int()
        K.ks_verify(self.ctx, t.ctypes.data, len(t) - 1, pred.ctypes.data, C.byref(a))
        return pred, a.value

    def select(self, params: K.SelectParams, debug_cells: int = 0):
        out = K.Selection()
        dbg = None
        if debug_cells:
            n = 2 * self.cfg.L + 1
            self._dbg = {
                "bits": np.zeros((n, debug_cells), dtype=np.uint8),
                "reach": np.zeros((n, debug_cells), dtype=np.uint8),
                "sig_e": np.zeros((n, debug_cells), dtype=np.float64),
                "sig_s": np.zeros((n, debug_cells), dtype=np.float64),
                "n_match": np.zeros(debug_cells, dtype=np.int32),
            }
            g = self._dbg
            dbg = K.SelectionDebug(debug_cells,
                                   g["bits"].ctypes.data_as(C.POINTER(C.c_uint8)),
                                   g["reach"].ctypes.data_as(C.POINTER(C.c_uint8)),
                                   g["sig_e"].ctypes.data_as(C.POINTER(C.c_double)),
                                   g["sig_s"].ctypes.data_as(C.POINTER(C.c_double)),
                                   g["n_match"].ctypes.data_as(C.POINTER(C.c_int)))
        K.ks_knapsack_select(self.ctx, C.byref(params), C.byref(out),
                             C.byref(dbg) if dbg is not None else None)
        return (out, self._dbg) if debug_cells else out

    def set_draft_policy(self, tau_conf: float = 0.0, gamma_source: str = "fixed"):
        """Dynamic drafting exit below tau_conf (0 disables) and the draft cap of
        each round: the call's gamma ("fixed") or min(gamma*, gamma) ("selected")."""
        src = {"fixed": K.KS_GAMMA_FIXED, "selected": K.KS_GAMMA_SELECTED}[gamma_source]
        K.ks_set_draft_policy(self.ctx, C.byref(K.DraftPolicy(tau_conf, src)))

    def set_sampling(self, temperature: float = 0.0, top_k: int = 50, top_p: float = 0.95,
                     seed: int = 0):
        """Speculative sampling with the T / top-k / top-p filter and Philox
        stream `seed`; temperature <= 0 returns to greedy decoding."""
        K.ks_set_sampling(self.ctx, C.byref(K.Sampling(temperature, top_k, top_p, seed)))

    def generate(self, prompt, n_new: int, gamma: int, reselect_every: int = 32,
                 params: K.SelectParams | None = None, max_sel_log: int = 256):
        p = np.ascontiguousarray(prompt, dtype=np.int32)
        out = np.zeros(n_new, dtype=np.int32)
        st = K.GenStats()
        log = (K.Selection * max_sel_log)()
        K.ks_generate(self.ctx, p.ctypes.data, len(p), n_new, gamma, reselect_every,
                      C.byref(params) if params is not None else None, out.ctypes.data,
                      C.byref(st), log, max_sel_log)
        sels = [log[i] for i in range(min(st.n_selections, max_sel_log))]
        return out, st, sels

    def decode(self, n_new: int, gamma: int, reselect_every: int = 32,
               params: K.SelectParams | None = None, max_sel_log: int = 256):
        """Generation loop from the current state (no prefill)."""
        out = np.zeros(n_new, dtype=np.int32)
        st = K.GenStats()
        log = (K.Selection * max_sel_log)()
        K.ks_decode(self.ctx, n_new, gamma, reselect_every,
                    C.byref(params) if params is not None else None, out.ctypes.data,
                    C.byref(st), log, max_sel_log)
        sels = [log[i] for i in range(min(st.n_selections, max_sel_log))]
        return out, st, sels

    def profile_decode(self, exec_mask=None, steps: int = 8, per_kernel: bool = True) -> dict:
        """Mean per-launch duration (ms) of every kernel class of a decode step."""
        m = None
        if exec_mask is not None:
            m = np.ascontiguousarray(np.asarray(exec_mask, dtype=bool).astype(np.uint8))
        pr = K.KernelProfile()
        K.ks_profile_decode(self.ctx, m.ctypes.data if m is not None else None, steps,
                            1 if per_kernel else 0, C.byref(pr))
        return {"ms": {n: pr.ms[i] for i, n in enumerate(K.KS_KC_NAMES)},
                "launches": {n: pr.launches[i] for i, n in enumerate(K.KS_KC_NAMES)},
                "ms_step": pr.ms_step, "steps": pr.steps}

    def sublayer_apply(self, i: int, x: torch.Tensor, pos, mode: int = 0, out=None):
        pos = np.ascontiguousarray(pos, dtype=np.int32)
        out = x if out is None else out
        K.ks_sublayer_apply(self.ctx, i, _ptr(x), _ptr(out), pos.ctypes.data, len(pos), mode)
        return out

    def head_rows(self, x: torch.Tensor, want_logits: bool = True):
        R = x.shape[0]
        logits = (torch.empty(R, self.cfg.vocab, dtype=torch.float32, device=self.dev)
                  if want_logits else None)
        am = torch.empty(R, dtype=torch.int32, device=self.dev)
        top1 = torch.empty(R, dtype=torch.float32, device=self.dev)
        K.ks_head_rows(self.ctx, _ptr(x), R, _ptr(logits) if want_logits else None, _ptr(am),
                       _ptr(top1))
        return logits, am, top1


# ------------------------------------------------------- raw-pointer calls
def hidden_cos(X: torch.Tensor, Y: torch.Tensor) -> torch.Tensor:
    """mean row cosine of every [r, d] group of X [G, r, d] against Y [r, d]."""
    G, r, d = X.shape
    out = torch.empty(G, dtype=torch.float32, device=X.device)
    K.ks_hidden_cos(_ptr(X), _ptr(Y), G, r, d, _ptr(out), _stream())
    return out


def sample_filter(logits: torch.Tensor, temperature: float, top_k: int, top_p: float,
                  seed: int = 0, pos0: int | None = None, purpose: int = 2):
    """Filter tables (ids, probs, counts), unfiltered top-1 probability and, when
    pos0 is given, the draw of row r at position pos0 + r."""
    R, V = logits.shape
    dev = logits.device
    s = K.Sampling(temperature, top_k, top_p, seed)
    ws_b = K.ks_sample_workspace_bytes(R, V, top_k)  # 0: the call reports the bad argument
    ws = torch.empty(max(ws_b, 256), dtype=torch.uint8, device=dev)
    ids = torch.empty(R, K.KS_SAMPLE_KMAX, dtype=torch.int32, device=dev)
    probs = torch.empty(R, K.KS_SAMPLE_KMAX, dtype=torch.float32, device=dev)
    cnt = torch.empty(R, dtype=torch.int32, device=dev)
    top1 = torch.empty(R, dtype=torch.float32, device=dev)
    tok = torch.empty(R, dtype=torch.int32, device=dev) if pos0 is not None else None
    K.ks_sample_filter(_ptr(logits), R, V, logits.stride(0), C.byref(s), pos0 or 0, purpose,
                       _ptr(ids), _ptr(probs), _ptr(cnt), _ptr(top1),
                       _ptr(tok) if tok is not None else None, _ptr(ws), ws_b, _stream())
    return ids, probs, cnt, top1, tok


def spec_accept(p_ids, p_probs, p_cnt, q_ids, q_probs, q_cnt, drafts: torch.Tensor, seed: int,
                pos0: int):
    """Acceptance chain of one round on device tables: (accepted drafts, token)."""
    g = drafts.numel()
    out = torch.empty(2, dtype=torch.int32, device=p_ids.device)
    K.ks_spec_accept(_ptr(p_ids), _ptr(p_probs), _ptr(p_cnt), _ptr(q_ids), _ptr(q_probs),
                     _ptr(q_cnt), _ptr(drafts), g, seed, pos0, _ptr(out), _stream())
    a, t = out.cpu().tolist()
    return a, t


def sample_uniforms(seed: int, pos: torch.Tensor, purpose: int) -> torch.Tensor:
    out = torch.empty(pos.numel(), dtype=torch.float32, device=pos.device)
    K.ks_sample_uniforms(seed, _ptr(pos), pos.numel(), purpose, _ptr(out), _stream())
    return out


def knapsack_quantize(t: np.ndarray, s: np.ndarray, bins: int):
    t = np.ascontiguousarray(t, dtype=np.float64)
    s = np.ascontiguousarray(s, dtype=np.float64)
    B, n = t.shape
    w = np.zeros((B, n), dtype=np.int32)
    q = np.zeros((B, n), dtype=np.int32)
    K.ks_knapsack_quantize(t.ctypes.data, s.ctypes.data, B, n, bins, w.ctypes.data, q.ctypes.data)
    return w, q


def knapsack_batch(w: torch.Tensor, q: torch.Tensor, C_cap: int, max_skip: int):
    B, n = w.shape
    best = torch.empty(B, C_cap + 1, dtype=torch.int32, device=w.device)
    bits = torch.empty(B, n, C_cap // 64 + 1, dtype=torch.int64, device=w.device)
    K.ks_knapsack_batch(_ptr(w), _ptr(q), B, n, C_cap, max_skip, _ptr(best), _ptr(bits), _stream())
    return best, bits


def knapsack_backtrack(bits: torch.Tensor, w: torch.Tensor, C_cap: int, j: torch.Tensor):
    B, n = w.shape
    skip = torch.empty(B, n, dtype=torch.uint8, device=w.device)
    err = torch.empty(B, dtype=torch.int32, device=w.device)
    K.ks_knapsack_backtrack(_ptr(bits), _ptr(w), B, n, C_cap, _ptr(j), _ptr(skip), _ptr(err),
                            _stream())
    return skip, err


def knapsack_batch_select(best, bits, w, s, C_cap: int, D: int = 10):
    B, n = w.shape
    dev = w.device
    js = torch.empty(B, dtype=torch.int32, device=dev)
    gs = torch.empty(B, dtype=torch.int32, device=dev)
    tpt = torch.empty(B, dtype=torch.float64, device=dev)
    skip = torch.empty(B, n, dtype=torch.uint8, device=dev)
    K.ks_knapsack_batch_select(_ptr(best), _ptr(bits), _ptr(w), _ptr(s), B, n, C_cap, D, _ptr(js),
                               _ptr(gs), _ptr(tpt), _ptr(skip), _stream())
    return js, gs, tpt, skip


# ------------------------------------------- draws and the paged cache
def _need(ok: bool, msg: str):
    if not ok:
        raise ValueError(msg)


def _here(at: int, f, *args):
    """Calls f with args and the current stream of GPU at, it being current.  (These calls
    take a few microseconds on the GPU, and so their checks look at devices by index and
    build their messages only when they fail.)"""
    s = torch._C._cuda_getCurrentRawStream(at)  # current_stream() builds an object: 2.8 us
    if at == torch._C._cuda_getDevice():
        f(*args, s)
    else:
        with torch.cuda.device(at):
            f(*args, s)


def _need_workspace(w: torch.Tensor, at: int):
    _need(w.dtype is torch.uint8 and w.is_contiguous() and w.get_device() == at,
          "workspace must be dense uint8 on the same device")


_DT = {torch.float32: K.KS_F32, torch.bfloat16: K.KS_BF16}


def _rows3(t: torch.Tensor, heads: int, hd: int, name: str) -> int:
    """Row stride (elements) of t [rows, heads, hd], dense inside a row."""
    shape = t.shape
    if len(shape) == 3 and shape[1] == heads and shape[2] == hd:
        n, (ld, sh, sd) = shape[0], t.stride()
        if n == 0 or sd == 1 and (heads == 1 or sh == hd):
            return ld if n > 1 else max(ld, heads * hd)
    raise ValueError(f"{name} must be [rows, {heads}, {hd}], dense rows")


def sample_draw_workspace(rows: int, vocab: int, device="cuda") -> torch.Tensor:
    """Workspace of sample_draw calls of at most these sizes; calls that may run at the
    same time (on other streams, in other captured graphs) need one each."""
    n = K.ks_sample_draw_workspace_bytes(rows, vocab)  # 0: the call reports the bad argument
    return torch.empty(max(n, 256), dtype=torch.uint8, device=device)


def sample_draw(logits: torch.Tensor, u: torch.Tensor, temperature=None, top_k=None, top_p=None,
                min_p=None, tokens=None, logprob=None, kept=None, workspace=None) -> torch.Tensor:
    """One token per row of logits [rows, vocab] (float32 or bfloat16) from the given
    uniforms u [rows], with every row's own settings (tensors [rows], None: 1 or off):
    see ks_sample_draw.  Fills tokens (returned), logprob and kept where given."""
    _need(logits.dim() == 2 and u is not None, "logits must be [rows, vocab] and u given")
    shape, at = logits.shape, logits.get_device()
    R, V = shape
    row = shape[:1]
    ld, step = logits.stride()
    _need(logits.dtype in _DT and step == 1 and at >= 0,
          "logits must be float32 or bfloat16 [rows, vocab] on a GPU, dense rows")
    if tokens is None:
        tokens = torch.empty(R, dtype=torch.int32, device=logits.device)
    f32, i32 = torch.float32, torch.int32
    ptr = []
    for t, dt in ((temperature, f32), (top_k, i32), (top_p, f32), (min_p, f32), (u, f32),
                  (tokens, i32), (logprob, f32), (kept, i32)):
        if t is None:
            ptr.append(None)
            continue
        if (t.dtype is not dt or t.shape != row or not t.is_contiguous()
                or t.get_device() != at):
            raise ValueError(f"settings and results must be dense [{R}] on the logits' device: "
                             "int32 top_k, tokens and kept, float32 the others")
        ptr.append(t.data_ptr())
    if workspace is None:
        workspace = sample_draw_workspace(R, V, logits.device)
    _need_workspace(workspace, at)
    s = K.DrawParams(*ptr[:5])
    _here(at, K.ks_sample_draw, logits.data_ptr(), _DT[logits.dtype], R, V, ld if R > 1 else V,
          C.byref(s), *ptr[5:], workspace.data_ptr(), workspace.numel())
    return tokens


class PagedCache:
    """One layer's pages of keys and values (see ks_paged_cache): kind "e4m3" (8-bit
    floats, a scale for every `block` tokens and head) or "bf16".

    k is [n_pages, hkv, page, hd], v [n_pages, hkv, page // 16, hd, 16], the scales
    [n_pages, hkv, page // block] float32.  ``over`` wraps tensors of those shapes.
    """

    def __init__(self, n_pages: int, page: int, hkv: int, hd: int, kind: str = "e4m3",
                 block: int = 16, device="cuda"):
        _need(kind in ("e4m3", "bf16"), "kind must be 'e4m3' or 'bf16'")
        _need(page >= 16 and page % 16 == 0, "page must be a multiple of 16")
        dt = torch.float8_e4m3fn if kind == "e4m3" else torch.bfloat16
        z = lambda dt, *s: torch.zeros(*s, dtype=dt, device=device)
        self._set(z(dt, n_pages, hkv, page, hd), z(dt, n_pages, hkv, page // 16, hd, 16),
                  *([z(torch.float32, n_pages, hkv, page // block) for _ in range(2)]
                    if kind == "e4m3" else [None, None]))

    @classmethod
    def over(cls, k: torch.Tensor, v: torch.Tensor, k_scale: torch.Tensor | None = None,
             v_scale: torch.Tensor | None = None) -> "PagedCache":
        c = cls.__new__(cls)
        c._set(k, v, k_scale, v_scale)
        return c

    def _set(self, k, v, k_scale, v_scale):
        _need(k.dim() == 4 and k.dtype in (torch.bfloat16, torch.float8_e4m3fn, torch.uint8),
              "k must be [n_pages, hkv, page, hd] of bfloat16, float8_e4m3fn or uint8")
        n, hkv, page, hd = k.shape
        _need(v.shape == (n, hkv, page // 16, hd, 16) and v.dtype == k.dtype,
              "v must be [n_pages, hkv, page // 16, hd, 16] of k's type")
        e4 = k.dtype != torch.bfloat16
        block = 16
        _need((k_scale is not None) == e4 and (v_scale is not None) == e4,
              "8-bit caches have scales, bf16 ones none")
        if e4:
            nb = k_scale.shape[-1]
            _need(nb >= 1 and page % nb == 0, "a page holds a whole number of blocks")
            block = page // nb
            for s in (k_scale, v_scale):
                _need(s.shape == (n, hkv, nb) and s.dtype == torch.float32,
                      "scales must be float32 [n_pages, hkv, page // block]")
        ts = [t for t in (k, v, k_scale, v_scale) if t is not None]
        _need(all(t.is_contiguous() and t.device == k.device for t in ts),
              "cache tensors must be contiguous and on one device")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.device, self.at = k.device, k.get_device()
        self.page, self.block, self.hkv, self.hd = page, block, hkv, hd
        self.desc = K.PagedCache(_ptr(k), _ptr(v), _ptr(k_scale) if e4 else None,
                                 _ptr(v_scale) if e4 else None, n, page, block, hkv, hd,
                                 K.KS_E4M3 if e4 else K.KS_BF16)
        self.ref = C.byref(self.desc)


def _paged_rows(cache: PagedCache, table, row_start, pos0, rows, max_rows, max_len, err):
    B, width = table.shape if table.dim() == 2 else (-1, 0)
    ld, step = table.stride() if table.dim() == 2 else (0, 0)
    i32, at = torch.int32, cache.at
    _need(B >= 0 and pos0.shape == (B,) and table.dtype is i32 and step == 1
          and table.get_device() == at,
          "table must be int32 [B, pages], dense rows, on the cache's device")
    _need(row_start.shape == (B + 1,) and row_start.dtype is i32 and row_start.is_contiguous()
          and pos0.dtype is i32 and pos0.is_contiguous() and pos0.get_device() == at
          and row_start.get_device() == at,
          "row_start must be int32 [B + 1] and pos0 int32 [B], on the cache's device")
    if err is not None:
        _need(err.shape == (B,) and err.dtype is i32 and err.is_contiguous()
              and err.get_device() == at, "err must be int32 [B] on the cache's device")
    most = width * cache.page
    return K.PagedRows(B, rows, row_start.data_ptr(), pos0.data_ptr(), table.data_ptr(),
                       ld if B > 1 else width, rows if max_rows is None else max_rows,
                       most if max_len is None else min(max_len, most),
                       None if err is None else err.data_ptr())


def paged_append(cache: PagedCache, table, row_start, pos0, k, v, q=None, rope=None, q_out=None,
                 max_rows=None, err=None):
    """Stores the rows' keys (rotated by rope [positions, hd/2, 2]) and values and
    returns the rotated queries (in q_out, by default a new tensor; None without q).
    See ks_paged_append; row strides are free, so slices of a fused projection do."""
    hkv, hd, rows, at, dt = cache.hkv, cache.hd, k.shape[0], cache.at, k.dtype
    ldk, ldv = _rows3(k, hkv, hd, "k"), _rows3(v, hkv, hd, "v")
    _need(dt in _DT and v.dtype is dt and v.shape[0] == rows
          and k.get_device() == at and v.get_device() == at,
          "k and v must be float32 or bfloat16, of the same rows, on the cache's device")
    hq = ldq = ldo = 0
    pq = po = pr = None
    if q is not None:
        hq = q.shape[1]
        ldq = _rows3(q, hq, hd, "q")
        if q_out is None:
            q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        ldo = _rows3(q_out, hq, hd, "q_out")
        _need(q.dtype is dt and q_out.dtype is dt and q.shape[0] == rows
              and q_out.shape[0] == rows and q.get_device() == at
              and q_out.get_device() == at, "q and q_out must match k")
        pq, po = q.data_ptr(), q_out.data_ptr()
    n = 0
    if rope is not None:
        _need(rope.dim() == 3 and rope.shape[1:] == (hd // 2, 2) and rope.dtype is torch.float32
              and rope.is_contiguous() and rope.get_device() == at,
              "rope must be float32 [positions, hd / 2, 2] on the cache's device")
        pr, n = rope.data_ptr(), rope.shape[0]
    r = _paged_rows(cache, table, row_start, pos0, rows, max_rows, None, err)
    _here(at, K.ks_paged_append, cache.ref, C.byref(r), pq, ldq, k.data_ptr(), ldk, v.data_ptr(),
          ldv, po, ldo, hq, _DT[dt], pr, n)
    return q_out if q is not None else None


def paged_attention_workspace(cache: PagedCache, B: int, rows: int, hq: int, max_rows: int,
                              max_len: int) -> torch.Tensor:
    """Workspace of paged_attention calls with at most these bounds; calls that may run
    at the same time (on other streams, in other captured graphs) need one each."""
    n = K.ks_paged_attention_workspace_bytes(cache.ref, B, rows, hq, max_rows, max_len)
    return torch.empty(max(n, 256), dtype=torch.uint8, device=cache.device)


def paged_attention(cache: PagedCache, table, row_start, pos0, q, scale: float | None = None,
                    out=None, lse=None, max_rows=None, max_len=None, workspace=None, err=None):
    """Causal attention of the rows q [rows, hq, hd] over their sequences' pages (see
    ks_paged_attention).  max_rows and max_len bound the rows and positions of a
    sequence; they default to what the shapes allow, and tight ones are faster."""
    rows, hq, at, dt = q.shape[0], q.shape[1], cache.at, q.dtype
    ldq = _rows3(q, hq, cache.hd, "q")
    if out is None:
        out = torch.empty(q.shape, dtype=dt, device=q.device)
    ldo = _rows3(out, hq, cache.hd, "out")
    _need(dt in _DT and out.dtype is dt and out.shape[0] == rows
          and q.get_device() == at and out.get_device() == at,
          "q and out must be float32 or bfloat16, of the same rows, on the cache's device")
    if lse is not None:
        _need(lse.shape == (rows, hq) and lse.dtype is torch.float32 and lse.is_contiguous()
              and lse.get_device() == at, "lse must be float32 [rows, hq]")
    r = _paged_rows(cache, table, row_start, pos0, rows, max_rows, max_len, err)
    if workspace is None:
        workspace = paged_attention_workspace(cache, r.B, rows, hq, r.max_rows, r.max_len)
    _need_workspace(workspace, at)
    _here(at, K.ks_paged_attention, cache.ref, C.byref(r), q.data_ptr(), ldq, out.data_ptr(), ldo,
          hq, _DT[dt], cache.hd ** -0.5 if scale is None else scale,
          None if lse is None else lse.data_ptr(), workspace.data_ptr(), workspace.numel())
    return out
