"""Convenience layer over the C ABI: allocates the caller-owned device buffers
(KV pools, workspace, outputs) with torch and forwards every call to libpced.

Nothing here computes any part of the decode step.
"""
from __future__ import annotations

from typing import Optional, Sequence

import numpy as np

from . import _lib


_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


class Adjust:
    """A batch's logits adjustments (pced_adjust) with the device tensors they are in.

    history [n] int32 tokens of all queries and history_off [B + 1] int32; repetition,
    presence, frequency [B] float32; bias_token int32 and bias_value float32 [m] with
    bias_off [B + 1] int32; mask [B][words] int32, whose rows may be wider than
    ceil(V / 32) words or apart. All optional."""

    DTYPES = dict(history="int32", history_off="int32", repetition="float32", presence="float32", frequency="float32",
                  bias_token="int32", bias_value="float32", bias_off="int32", mask="int32")

    def __init__(self, n_queries, vocab, device, **tensors):
        torch = _torch()
        unknown = set(tensors) - set(self.DTYPES)
        if unknown:
            raise ValueError(f"unknown adjustments {sorted(unknown)}")
        self.n_queries, self.vocab, self.device = n_queries, vocab, device
        self.tensors = {k: t for k, t in tensors.items() if t is not None}
        for name, t in self.tensors.items():
            if t.dtype != getattr(torch, self.DTYPES[name]):
                raise ValueError(f"{name}: {t.dtype}, not {self.DTYPES[name]}")
            if t.device != device:
                raise ValueError(f"{name}: on {t.device}, the session is on {device}")
            if name == "mask":
                if t.dim() != 2 or t.shape[0] < n_queries or t.stride(1) != 1 or t.shape[1] < -(-vocab // 32):
                    raise ValueError("mask: [queries][>= ceil(vocab / 32)] words, a row's words next to each other")
                continue
            if t.dim() != 1 or not t.is_contiguous():
                raise ValueError(f"{name}: one dimension, contiguous")
            want = {"history_off": n_queries + 1, "bias_off": n_queries + 1, "repetition": n_queries,
                    "presence": n_queries, "frequency": n_queries}.get(name, 0)
            if t.numel() < want:
                raise ValueError(f"{name}: {t.numel()} entries, not {want}")
        for name, others in (("history", ("history_off",)), ("bias_token", ("bias_off", "bias_value"))):
            if name in self.tensors and any(o not in self.tensors for o in others):
                raise ValueError(f"{name} without {' or '.join(others)}")
        size = lambda n: self.tensors[n].numel() if n in self.tensors else 0  # noqa: E731
        if "bias_token" in self.tensors and size("bias_value") < size("bias_token"):
            raise ValueError("bias_value is shorter than bias_token")
        # (a list without entries has no memory to point at: it adjusts nothing)
        ptr = {k: t.data_ptr() for k, t in self.tensors.items() if t.numel() > 0}
        mask = self.tensors.get("mask")
        row = 0 if mask is None else mask.stride(0) if mask.shape[0] > 1 else mask.shape[1]
        if mask is not None and row < -(-vocab // 32):
            raise ValueError("mask: the rows overlap")
        self.struct = _lib.pced_adjust(mask_row=row, n_history=size("history"), n_bias=size("bias_token"), **ptr)


class Sampling:
    """A batch's sampling settings (pced_sampling) with the device tensors they are in: temperature [B] float32,
    and optionally top_k [B] int32, top_p and min_p [B] float32."""

    DTYPES = dict(temperature="float32", top_k="int32", top_p="float32", min_p="float32")

    def __init__(self, n_queries, device, **tensors):
        torch = _torch()
        unknown = set(tensors) - set(self.DTYPES)
        if unknown:
            raise ValueError(f"unknown settings {sorted(unknown)}")
        self.n_queries, self.device = n_queries, device
        self.tensors = {k: t for k, t in tensors.items() if t is not None}
        if "temperature" not in self.tensors:
            raise ValueError("no temperature")
        for name, t in self.tensors.items():
            if t.dtype != getattr(torch, self.DTYPES[name]) or t.shape != (n_queries,) or not t.is_contiguous():
                raise ValueError(f"{name}: {self.DTYPES[name]} [{n_queries}], contiguous")
            if t.device != device:
                raise ValueError(f"{name}: on {t.device}, the session is on {device}")
        self.struct = _lib.pced_sampling(**{k: t.data_ptr() for k, t in self.tensors.items()})


class PcedSession:
    """A context plus its two KV pools for one model geometry and capacity.

    ``kv8`` ("e4m3" or "int8", bf16 sessions): the caches are held in 8 bits instead, in the
    buffers k_codes, v_codes, scales, k_open and v_open (see pced_cache8). load, append, advance,
    attend, read_cache, lengths and the calls on logits then work as they do over pools (attend
    without ``select``); append takes up to ``max_new`` tokens at once."""

    kv8 = None

    def __init__(self, *, n_layers, n_q_heads, n_kv_heads, head_dim, vocab, dtype, max_queries,
                 max_seqs, max_pages, max_pages_per_seq, norm="rms", device="cuda", poison=False,
                 max_attn_chunks=0, aggregation="max", beta_scalar=False, ffn_dim=0, rope_theta=500000, kv8=None,
                 max_new=1):
        torch = _torch()
        if kv8 is not None and (kv8 not in _lib.CODES or dtype != "bf16" or max_new < 1):
            raise ValueError(f"kv8 is one of {sorted(_lib.CODES)}, in bf16 sessions, with max_new >= 1")
        self.kv8, self.max_new = kv8, max_new
        self.dtype = dtype
        self.geom = dict(n_layers=n_layers, n_q_heads=n_q_heads, n_kv_heads=n_kv_heads,
                         head_dim=head_dim, vocab=vocab)
        self.ffn_dim = ffn_dim
        self.cfg = _lib.make_config(n_layers=n_layers, n_q_heads=n_q_heads, n_kv_heads=n_kv_heads,
                                    head_dim=head_dim, vocab=vocab, dtype=dtype, max_queries=max_queries,
                                    max_seqs=max_seqs, max_pages=max_pages,
                                    max_pages_per_seq=max_pages_per_seq, norm=norm,
                                    max_attn_chunks=max_attn_chunks, aggregation=aggregation,
                                    beta_scalar=beta_scalar, ffn_dim=ffn_dim, rope_theta=rope_theta)
        self.ctx = _lib.Context(self.cfg, device=device)
        room = lambda n: torch.empty(n, dtype=torch.uint8, device=device)  # noqa: E731
        if kv8 is None:
            pool = _lib.pced_pool_bytes(self.cfg)
            self.k_pool, self.v_pool = held = room(pool), room(pool)
        else:
            codes, opened = _lib.pced_codes_bytes(self.cfg), _lib.pced_open_bytes(self.cfg, max_new)
            self.k_codes, self.v_codes, self.scales, self.k_open, self.v_open = held = (
                room(codes), room(codes), room(_lib.pced_scales_bytes(self.cfg)), room(opened), room(opened))
        if poison:  # all-ones bytes: NaN in bf16 and f32, to expose reads of unwritten memory
            for t in (*held, self.ctx.workspace):
                t.fill_(255)
        if kv8 is not None:
            self.scales, self.k_open, self.v_open = (t.view(torch.bfloat16) for t in held[2:])
        self.device = held[0].device  # ("cuda": the one that is current now, for later allocations too)
        self._device_index = held[0].get_device()
        self._dtypes = (torch.bfloat16, torch.int16, torch.uint16) if dtype == "bf16" else (torch.float32,)
        self._rows, self._ropes, self._out_like = _lib.pced_rows(), {}, {}
        self.n_experts: list = []
        self.S = 0
        self.B = 0
        self.NE = 0

    def pack_lm_head(self, w):
        """Packed copy (device) of row-major [V][hidden] LM-head weights."""
        torch = _torch()
        out = torch.empty(_lib.pced_lm_head_bytes(self.cfg), dtype=torch.uint8, device=self.device)
        _lib.pced_pack_lm_head(self.cfg, w, out)
        return out

    def pack_model(self, layer_tensors, embed, final_norm):
        """Packed decoder-stack weights (device). ``layer_tensors(l)`` returns the 9
        bf16 device tensors of layer l in pced_pack_model_layer order."""
        torch = _torch()
        out = torch.empty(_lib.pced_model_bytes(self.cfg), dtype=torch.uint8, device=self.device)
        for l in range(self.geom["n_layers"]):
            ts = layer_tensors(l)
            _lib.pced_pack_model_layer(self.cfg, l, ts, out)
            torch.cuda.current_stream().synchronize()  # the sources may be dropped after the copy
            del ts
        _lib.pced_pack_model_globals(self.cfg, embed, final_norm, out)
        torch.cuda.current_stream().synchronize()
        return out

    def model_step(self, model, lm_head, in_tokens, want=("logits", "winner", "top1", "top2", "beta_used")):
        torch = _torch()
        tokens = torch.empty(self.B, dtype=torch.int32, device=self.device)
        extra = self.out_buffers(want) if want else None
        self.ctx.pced_model_step(model, lm_head, in_tokens, tokens, extra)
        out = dict(extra or {})
        out["tokens"] = tokens
        return out

    # ------------------------------------------------------------------ load
    def load(self, n_experts: Sequence[int], cache_len: Sequence[int], src_k, src_v, relevance,
             gamma=2.5, beta=None, page_table=None, reserve_tokens=0):
        self.n_experts = list(n_experts)
        self.B = len(self.n_experts)
        self.S = int(sum(n + 1 for n in self.n_experts))
        self.NE = int(sum(self.n_experts))
        batch = dict(gamma=gamma, beta=beta, page_table=page_table, reserve_tokens=reserve_tokens)
        if self.kv8 is None:
            self.ctx.pced_load_caches(n_experts, cache_len, src_k, src_v, self.k_pool, self.v_pool, relevance, **batch)
        else:
            self.ctx.pced_load_codes(n_experts, cache_len, src_k, src_v, self.kv8, self.max_new, self.k_codes, self.v_codes,
                                     self.scales, self.k_open, self.v_open, relevance, **batch)
        # (shapes of fuse_adjusted's outputs: empty_like takes a third less time than a shape and a type)
        self._out_like = self.out_buffers(("winner", "top1", "top2", "beta_used"))

    # ----------------------------------------------------------------- steps
    def out_buffers(self, want=("logits", "winner", "top1", "top2", "beta_used")):
        torch = _torch()
        g = self.geom
        f32, i32 = torch.float32, torch.int32
        shapes = {
            "attn_out": ((self.S, g["n_layers"], g["n_q_heads"], g["head_dim"]), f32),
            "logits": ((self.S, g["vocab"]), f32),
            "winner": ((self.B,), i32),
            "top1": ((self.B,), f32),
            "top2": ((self.B,), f32),
            "beta_used": ((self.NE,), f32),
            "hidden": ((self.S, g["n_q_heads"] * g["head_dim"]), f32),
        }
        if self.ffn_dim:
            L, H, D = g["n_layers"], g["n_q_heads"] * g["head_dim"], g["head_dim"]
            qkv = (g["n_q_heads"] + 2 * g["n_kv_heads"]) * D
            shapes["resid_trace"] = ((L, 2, self.S, H), f32)
            shapes["qkv_trace"] = ((L, self.S, qkv), torch.int16)
            shapes["act_trace"] = ((L, self.S, self.ffn_dim), torch.int16)
        return {k: torch.empty(shapes[k][0], dtype=shapes[k][1], device=self.device) for k in want}

    def step(self, q, k_new, v_new, lm_head, want=("logits", "winner", "top1", "top2", "beta_used")):
        torch = _torch()
        tokens = torch.empty(self.B, dtype=torch.int32, device=self.device)
        extra = self.out_buffers(want) if want else None
        self.ctx.pced_step(q, k_new, v_new, lm_head, tokens, extra)
        out = dict(extra or {})
        out["tokens"] = tokens
        return out

    def generate(self, n_steps, seed, first_token, lm_head, want=()):
        torch = _torch()
        tokens = torch.empty((self.B, n_steps), dtype=torch.int32, device=self.device)
        extra = self.out_buffers(want) if want else None
        self.ctx.pced_generate(n_steps, seed, first_token, lm_head, tokens, extra)
        out = dict(extra or {})
        out["tokens"] = tokens
        return out

    # ------------------------------------------------------ layer-wise calls
    def _storage(self, t, name):
        """A tensor of the session's storage type (bf16 values or their bits, or float32)."""
        if t.dtype not in self._dtypes:
            raise ValueError(f"{name}: {t.dtype} in a session of {self.dtype}")
        return self._here(t, name)

    def _on_device(self):
        """The calls go to the current device's stream, which has to be the session's."""
        if _lib.current_device() != self._device_index:
            raise ValueError(f"the session is on {self._where()}, which is not the current device")

    def _where(self):
        return (self.k_pool if self.kv8 is None else self.k_codes).device

    def _here(self, t, name):
        if t.get_device() != self._device_index:
            raise ValueError(f"{name}: on {t.device}, the session is on {self._where()}")
        return t

    def _row_stride(self, t, name, n_tokens, n_layers, heads):
        """Elements from one row of [S * n_tokens][n_layers][heads][D] to the next."""
        d = self.geom["head_dim"]
        shape = (self.S * n_tokens, n_layers, heads, d)
        if t.shape != shape:
            raise ValueError(f"{name}: {tuple(t.shape)}, not {shape}")
        if t.dtype not in self._dtypes or t.get_device() != self._device_index:
            self._storage(t, name)  # (names the fault)
        if t.is_contiguous():
            return n_layers * heads * d
        st = t.stride()
        if (d > 1 and st[3] != 1) or (heads > 1 and st[2] != d) or (n_layers > 1 and st[1] != heads * d):
            raise ValueError(f"{name}: a row's elements must follow each other")
        if shape[0] == 1:
            return n_layers * heads * d
        if st[0] < n_layers * heads * d:  # (a broadcast row has distance 0, which the library takes for rows without gaps)
            raise ValueError(f"{name}: the rows overlap")
        return st[0]

    def _rope(self, rope):
        """(theta, rot_dim, halves) as the library takes it."""
        if rope is None:
            return None
        r = self._ropes.get(rope)
        if r is None:
            theta, rot, halves = rope
            r = self._ropes[rope] = _lib.pced_rope(theta=theta, rot_dim=rot, halves=int(bool(halves)))
        return r

    def append(self, q, k, v, n_tokens=1, rope=None, layer=0, n_layers=None, q_out=None):
        """pced_append of layers [layer, layer + n_layers) (default: to the last): rows
        [S * n_tokens][n_layers][heads][D], which may be apart (views of one projection's
        output); q None: K / V only. ``rope``: (theta, rot_dim, halves) or None. Returns the
        rotated q rows (``q_out`` or a new tensor)."""
        self._on_device()
        g = self.geom
        if n_layers is None:
            n_layers = g["n_layers"] - layer
        rows = self._rows
        rows.k_row = self._row_stride(k, "k", n_tokens, n_layers, g["n_kv_heads"])
        rows.v_row = self._row_stride(v, "v", n_tokens, n_layers, g["n_kv_heads"])
        rows.k, rows.v, rows.q, rows.q_row = k.data_ptr(), v.data_ptr(), None, 0
        if q is not None:
            rows.q_row = self._row_stride(q, "q", n_tokens, n_layers, g["n_q_heads"])
            rows.q = q.data_ptr()
            if q_out is None:
                torch = _torch()
                q_out = torch.empty_like(q) if q.is_contiguous() else torch.empty(q.shape, dtype=q.dtype, device=q.device)
            elif self._storage(q_out, "q_out").shape != q.shape or not q_out.is_contiguous():
                raise ValueError("q_out: q's shape, contiguous")
        call = self.ctx.pced_append if self.kv8 is None else self.ctx.pced_append_codes
        call(layer, n_layers, n_tokens, rows, self._rope(rope), q_out)
        return q_out

    def advance(self, n_tokens=1):
        self.ctx.pced_advance(n_tokens)

    def bind_summary(self):
        """A new buffer for the page summaries, bound to the context."""
        torch = _torch()
        self.summary = torch.empty(_lib.pced_summary_bytes(self.cfg), dtype=torch.uint8, device=self.device)
        self.ctx.pced_bind_summary(self.summary)

    def summarize(self):
        self._on_device()
        self.ctx.pced_summarize()

    def attend(self, q, n_tokens=1, select=None, layer=0, n_layers=None, want=(), x_out=None):
        """pced_attend: q as append returned it; ``select``: (n_pages, n_first, n_last) or None
        for all pages. Returns {"x": [S * n_tokens][n_layers][Hq * D]}, and with "pages" in
        ``want`` the pages [S * n_tokens][n_layers][Hkv][n_pages]."""
        self._on_device()
        torch, g = _torch(), self.geom
        if n_layers is None:
            n_layers = g["n_layers"] - layer
        for name in want:
            if name != "pages":
                raise ValueError(f"unknown output {name}")
        rows, width = self.S * n_tokens, g["n_q_heads"] * g["head_dim"]
        if self._row_stride(q, "q", n_tokens, n_layers, g["n_q_heads"]) != n_layers * width:
            raise ValueError("q: rows must follow each other")
        if x_out is None:
            x_out = q.new_empty((rows, n_layers, width))
        elif self._storage(x_out, "x_out").shape != (rows, n_layers, width) or not x_out.is_contiguous():
            raise ValueError("x_out: [S * n_tokens][n_layers][Hq * D], contiguous")
        out, sel, pages = {"x": x_out}, None, None
        if self.kv8 is not None:
            if select is not None or want:
                raise ValueError("a cache in 8 bits is attended to whole: no select, no pages")
            self.ctx.pced_attend_codes(layer, n_layers, n_tokens, q, x_out)
            return out
        if select is not None:
            sel = _lib.pced_select(*select)
            if want:
                out["pages"] = pages = torch.empty((rows, n_layers, g["n_kv_heads"], max(0, sel.n_pages)),
                                                   dtype=torch.int32, device=q.device)
        elif want:
            raise ValueError("pages without select")
        self.ctx.pced_attend(layer, n_layers, n_tokens, q, sel, x_out, pages)
        return out

    # ------------------------------------------------------- adjusted logits
    def adjust(self, **tensors):
        """The loaded batch's adjustments (see Adjust) for adjust_logits and fuse_adjusted."""
        return Adjust(self.B, self.geom["vocab"], self.device, **tensors)

    def _logits(self, t, name):
        if t.dtype != _torch().float32 or t.shape != (self.S, self.geom["vocab"]) or not t.is_contiguous():
            raise ValueError(f"{name}: float32 [{self.S}][{self.geom['vocab']}], contiguous")
        return self._here(t, name)

    def _adjust(self, adjust):
        if adjust.n_queries != self.B or adjust.vocab != self.geom["vocab"]:
            raise ValueError("the adjustments are another batch's")
        if adjust.device != self.device:
            raise ValueError(f"the adjustments are on {adjust.device}, the session is on {self.device}")
        return adjust.struct

    def adjust_logits(self, logits, adjust, out=None):
        """pced_adjust_logits of [S][V] logits; ``out`` may be logits itself."""
        self._on_device()
        self._logits(logits, "logits")
        out = _torch().empty_like(logits) if out is None else self._logits(out, "out")
        self.ctx.pced_adjust_logits(logits, self._adjust(adjust), out)
        return out

    def fuse_adjusted(self, logits, adjust, refresh_beta=False, want=("winner", "top1", "top2", "beta_used")):
        """pced_fuse_adjusted: the tokens chosen over adjusted logits, and the wanted outputs."""
        self._on_device()
        like = _torch().empty_like
        self._logits(logits, "logits")
        out = {"tokens": like(self._out_like["winner"])}
        for name in want:
            if name not in self._out_like:
                raise ValueError(f"unknown output {name}")
            out[name] = like(self._out_like[name])
        self.ctx.pced_fuse_adjusted(logits, refresh_beta, self._adjust(adjust), out["tokens"], out)
        return out

    # --------------------------------------------------------------- sampling
    def sampling(self, **tensors):
        """The loaded batch's sampling settings (see Sampling) for sample."""
        return Sampling(self.B, self.device, **tensors)

    def sample(self, logits, sampling, uniform, adjust=None, refresh_beta=False,
               want=("winner", "score", "logprob", "kept", "beta_used")):
        """pced_sample: a token per query, drawn with uniform [B] (float32) from [S][V] logits, adjusted if ``adjust``
        is given, and the wanted outputs."""
        self._on_device()
        torch = _torch()
        self._logits(logits, "logits")
        if sampling.n_queries != self.B:
            raise ValueError("the settings are another batch's")
        if sampling.device != self.device:
            raise ValueError(f"the settings are on {sampling.device}, the session is on {self.device}")
        if uniform.dtype != torch.float32 or uniform.shape != (self.B,) or not uniform.is_contiguous():
            raise ValueError(f"uniform: float32 [{self.B}], contiguous")
        self._here(uniform, "uniform")
        out = {"tokens": torch.empty_like(self._out_like["winner"])}
        for name in want:
            like = self._SAMPLE_LIKE.get(name)
            if like is None:
                raise ValueError(f"unknown output {name}")
            out[name] = torch.empty_like(self._out_like[like])
        extra = {name: out[name] for name in want}
        self.ctx.pced_sample(logits, refresh_beta, None if adjust is None else self._adjust(adjust), sampling.struct,
                             uniform, out["tokens"], extra)
        return out

    _SAMPLE_LIKE = dict(winner="winner", score="top1", logprob="top1", kept="winner", beta_used="beta_used")

    def lengths(self):
        return self.ctx.pced_get_lengths(self.S)

    def read_cache(self, seq, layer, start, count):
        """(k, v) rows [count][Hkv][D] of one sequence and layer, read out of the
        pool (int16 bf16 bits or float32), on the session's device."""
        torch = _torch()
        g = self.geom
        dt = torch.int16 if self.dtype == "bf16" else torch.float32
        k = torch.empty((count, g["n_kv_heads"], g["head_dim"]), dtype=dt, device=self.device)
        v = torch.empty_like(k)
        call = self.ctx.pced_read_cache if self.kv8 is None else self.ctx.pced_read_codes
        call(seq, layer, start, count, k, v)
        return k, v


def session_for_workload(wl, device="cuda", extra_tokens: Optional[int] = None, norm="rms",
                         load_now=True, max_queries=None, poison=False, max_attn_chunks=0, aggregation="max",
                         beta_scalar=False, ffn_dim=0, rope_theta=500000):
    """Build a session sized for a synthetic workload (duck-typed: any object with
    the attributes of ``pced_inputs.workloads.Workload``) and load its caches,
    materialised on ``device``."""
    g = wl.geom
    extra = wl.steps if extra_tokens is None else extra_tokens
    need = wl.pages_needed(extra)
    maxpps = int(need.max())
    sess = PcedSession(n_layers=g.n_layers, n_q_heads=g.n_q_heads, n_kv_heads=g.n_kv_heads,
                       head_dim=g.head_dim, vocab=g.vocab, dtype=g.dtype,
                       max_queries=max_queries or wl.n_queries, max_seqs=wl.n_seqs,
                       max_pages=int(need.sum()), max_pages_per_seq=maxpps, norm=norm, device=device,
                       poison=poison, max_attn_chunks=max_attn_chunks, aggregation=aggregation,
                       beta_scalar=beta_scalar, ffn_dim=ffn_dim, rope_theta=rope_theta)
    sess.workload_page_table = wl.page_table(extra, maxpps)
    if load_now:
        load_workload(sess, wl)
    return sess


def load_workload(sess: PcedSession, wl, src=None):
    """(Re)load the workload's caches into the session; ``src`` optionally reuses
    already materialised (k, v) device tensors."""
    torch = _torch()
    if src is None:
        src_k = [wl.kcache_device(s, sess.device) for s in range(wl.n_seqs)]
        src_v = [wl.vcache_device(s, sess.device) for s in range(wl.n_seqs)]
    else:
        src_k, src_v = src
    sess.load(wl.n_experts, wl.cache_len.tolist(), src_k, src_v, wl.relevance.tolist(), gamma=wl.gamma,
              beta=None if wl.beta is None else np.asarray(wl.beta).tolist(),
              page_table=sess.workload_page_table)
    torch.cuda.current_stream().synchronize()
    return src_k, src_v
