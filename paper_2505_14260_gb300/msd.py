"""Thin ctypes binding of the MSD C ABI (include/msd.h).

Argument marshalling only: every step of the decode path runs in the CUDA
library. PyTorch supplies device memory and the stream. Loading fails loudly
if the library has not been built (``python -m paper_2505_14260_gb300.build``);
there is no fallback.
"""
from __future__ import annotations

import contextlib
import ctypes
import os
from ctypes import POINTER, c_char_p, c_float, c_int32, c_int64, c_void_p

import torch

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libmsd.so")

MSD_OK, MSD_ERR_INVALID, MSD_ERR_CAPACITY, MSD_ERR_OOM, MSD_ERR_CUDA, MSD_ERR_DEVICE = 0, -1, -2, -3, -4, -5
MSD_F32, MSD_BF16 = 0, 1
DRAFT_INPUTS = {"embedding": 0, "concat": 1, "feature": 2}     # MSD_DRAFT_*
STATUS_NAMES = {0: "MSD_OK", -1: "MSD_ERR_INVALID", -2: "MSD_ERR_CAPACITY", -3: "MSD_ERR_OOM",
                -4: "MSD_ERR_CUDA", -5: "MSD_ERR_DEVICE"}


class msd_config(ctypes.Structure):
    _fields_ = [("n_layers", c_int32), ("hidden", c_int32), ("n_heads", c_int32),
                ("head_dim", c_int32), ("ffn", c_int32), ("vocab", c_int32),
                ("rms_eps", c_float), ("rope_base", c_float), ("dtype", c_int32),
                ("max_batch", c_int32), ("max_seq", c_int32), ("tree_nodes", c_int32),
                ("tree_depth", c_int32), ("topk", c_int32), ("draft_input", c_int32)]


LAYER_FIELDS = ("attn_norm", "wq", "wk", "wv", "wo", "mlp_norm", "w_gate", "w_up", "w_down")


class msd_layer(ctypes.Structure):
    _fields_ = [(n, c_void_p) for n in LAYER_FIELDS]


class msd_weights(ctypes.Structure):
    _fields_ = [("embed", c_void_p), ("layers", POINTER(msd_layer)), ("final_norm", c_void_p),
                ("lm_head", c_void_p), ("draft", msd_layer), ("draft_fc", c_void_p)]


class msd_tree(ctypes.Structure):
    _fields_ = [("tokens", c_void_p), ("parent", c_void_p), ("depth", c_void_p),
                ("mask", c_void_p), ("n_nodes", c_void_p)]


class msd_draft_record(ctypes.Structure):
    _fields_ = [("logits", c_void_p), ("topk_ids", c_void_p), ("topk_logp", c_void_p)]


class msd_state_view(ctypes.Structure):
    _fields_ = [("target_kv", c_void_p), ("draft_kv", c_void_p), ("seq_len", c_void_p),
                ("n_pending", c_void_p), ("root", c_void_p), ("elem_bytes", c_int64),
                ("lo_offset", c_int64)]


class msd_profile(ctypes.Structure):
    _fields_ = [("kernel_launches", c_int64), ("gemm_launches", c_int64), ("gemm_ms", ctypes.c_double),
                ("gemm_bytes", ctypes.c_double), ("gemm_weight_bytes", ctypes.c_double),
                ("gemm_critical_ms", ctypes.c_double), ("windows", c_int64),
                ("gemm_flops", ctypes.c_double), ("gemm_mma_flops", ctypes.c_double),
                ("gemm_prefetch_bytes", ctypes.c_double)]


class msd_kernel_slot(ctypes.Structure):
    _fields_ = [("kind", c_int32), ("rows", c_int32), ("outputs", c_int32), ("inner", c_int32),
                ("launches", c_int64), ("bytes", ctypes.c_double), ("critical_ms", ctypes.c_double),
                ("span_ms", ctypes.c_double)]


class msd_gemm_shape(ctypes.Structure):
    _fields_ = [("ctas", c_int32), ("cluster", c_int32), ("smem_bytes", c_int32), ("tmem_cols", c_int32),
                ("chain", c_int32), ("chunks", c_int32), ("cut_tiles", c_int32)]


class msd_pages_config(ctypes.Structure):
    _fields_ = [("dtype", c_int32), ("n_layers", c_int32), ("n_heads", c_int32), ("n_kv_heads", c_int32),
                ("head_dim", c_int32), ("page_size", c_int32), ("n_pages", c_int32), ("max_seqs", c_int32),
                ("max_pages", c_int32), ("rot_dim", c_int32), ("rot_section", c_int32 * 3),
                ("rot_interleaved", c_int32), ("rope_base", c_float)]


class msd_pages_buffers(ctypes.Structure):
    _fields_ = [("kv", c_void_p), ("table", c_void_p), ("len", c_void_p), ("refs", c_void_p)]


class msd_batch(ctypes.Structure):
    _fields_ = [("n", c_int32), ("seqs", c_void_p), ("row_start", c_void_p), ("rows", c_int32)]


class msd_weight4(ctypes.Structure):
    _fields_ = [("codes", c_void_p), ("scales", c_void_p), ("zeros", c_void_p), ("o", c_int32), ("k", c_int32),
                ("group", c_int32)]


class msd_linear4_shape(ctypes.Structure):
    _fields_ = [("few", c_int32), ("rows", c_int32), ("outputs", c_int32), ("split", c_int32), ("staged", c_int32),
                ("direct", c_int32), ("smem_bytes", c_int32)]


class msd_filter(ctypes.Structure):
    _fields_ = [("temperature", c_void_p), ("top_k", c_void_p), ("top_p", c_void_p), ("min_p", c_void_p)]


_SIGNATURES = {
    "msd_create": (c_int32, [POINTER(msd_config), POINTER(msd_weights), POINTER(c_void_p)]),
    "msd_destroy": (c_int32, [c_void_p]),
    "msd_prefill": (c_int32, [c_void_p, c_int32, POINTER(c_int32), c_void_p, c_int32, c_void_p,
                              POINTER(c_int64), c_void_p, c_void_p]),
    "msd_draft_tree": (c_int32, [c_void_p, POINTER(msd_tree), POINTER(msd_draft_record), c_void_p]),
    "msd_verify": (c_int32, [c_void_p, POINTER(msd_tree), c_void_p, c_void_p, c_void_p]),
    "msd_accept_compact": (c_int32, [c_void_p, POINTER(msd_tree), c_void_p, c_void_p, c_void_p,
                                     c_void_p, c_void_p, c_void_p]),
    "msd_accept_sample": (c_int32, [c_void_p, POINTER(msd_tree), c_void_p, c_float, c_void_p,
                                    c_void_p, c_void_p, c_void_p, c_void_p, c_void_p]),
    "msd_step": (c_int32, [c_void_p, POINTER(msd_tree), c_void_p, c_void_p, c_void_p, c_void_p,
                           c_void_p]),
    "msd_step_sample": (c_int32, [c_void_p, POINTER(msd_tree), c_float, c_void_p, c_void_p, c_void_p,
                                  c_void_p, c_void_p, c_void_p]),
    "msd_ar_step": (c_int32, [c_void_p, c_void_p, c_void_p]),
    "msd_linear": (c_int32, [c_void_p, c_void_p, c_int32, c_int32, c_int32, c_void_p, c_int32,
                             c_void_p, c_int32, c_int32, c_void_p]),
    "msd_linear_noalloc": (c_int32, [c_void_p, c_int32, c_int32, c_int32, c_void_p, c_int32,
                                     c_void_p, c_int32, c_int32, c_void_p]),
    "msd_tree_complete": (c_int32, [c_void_p, POINTER(msd_tree), c_int32, c_void_p]),
    "msd_test_wait_timeout": (c_int32, [c_void_p, c_int64, c_void_p]),
    "msd_test_gemm_shape": (c_int32, [c_int32] * 6 + [POINTER(msd_gemm_shape)]),
    "msd_profile_enable": (c_int32, [c_void_p, c_int32]),
    "msd_profile_read": (c_int32, [c_void_p, POINTER(msd_profile)]),
    "msd_profile_slots": (c_int32, [c_void_p, POINTER(msd_kernel_slot), c_int32, POINTER(c_int32)]),
    "msd_state": (c_int32, [c_void_p, POINTER(msd_state_view)]),
    "msd_last_error": (c_char_p, [c_void_p]),
    "msd_pages_create": (c_int32, [POINTER(msd_pages_config), POINTER(msd_pages_buffers), POINTER(c_void_p)]),
    "msd_pages_destroy": (c_int32, [c_void_p]),
    "msd_pages_last_error": (c_char_p, [c_void_p]),
    "msd_pages_restore": (c_int32, [c_void_p, c_void_p]),
    "msd_pages_reserve": (c_int32, [c_void_p, POINTER(msd_batch), c_void_p]),
    "msd_pages_fork": (c_int32, [c_void_p, c_int32, c_void_p, c_void_p, c_int32, c_void_p]),
    "msd_pages_compact": (c_int32, [c_void_p, POINTER(msd_batch), c_void_p, c_int32, c_void_p, c_void_p]),
    "msd_pages_free": (c_int32, [c_void_p, c_int32, c_void_p, c_void_p]),
    "msd_rope_positions": (c_int32, [c_void_p, POINTER(msd_batch), c_void_p, c_void_p, c_int32, c_void_p, c_void_p,
                                     c_int64, c_void_p, c_void_p]),
    "msd_rope_append": (c_int32, [c_void_p, c_int32, POINTER(msd_batch), c_void_p, c_int64, c_void_p, c_int64,
                                  c_void_p, c_int64, c_int32, c_void_p, c_int64, c_void_p, c_int64, c_void_p]),
    "msd_pages_attention": (c_int32, [c_void_p, c_int32, POINTER(msd_batch), POINTER(msd_tree), c_int32, c_int32,
                                      c_int32, c_void_p, c_int64, c_void_p, c_int64, c_void_p, c_void_p]),
    "msd_linear4": (c_int32, [c_void_p, c_int64, c_int32, c_int32, POINTER(msd_weight4), c_void_p, c_int64, c_int32,
                              c_void_p]),
    "msd_test_linear4_shape": (c_int32, [c_int32, c_int32, POINTER(msd_weight4), POINTER(msd_linear4_shape)]),
    "msd_test_linear4_timeout": (c_int32, [c_void_p, c_int64, c_int32, c_int32, POINTER(msd_weight4), c_void_p, c_int64, c_int32,
                                           c_void_p]),
    "msd_quantize4": (c_int32, [c_void_p, c_int64, c_int32, POINTER(msd_weight4), c_void_p, c_int64, c_void_p]),
    "msd_sample": (c_int32, [c_void_p, c_int64, c_int32, c_int32, c_int32, POINTER(msd_filter), c_void_p, c_void_p,
                             c_void_p, c_void_p, c_int64, c_void_p]),
    "msd_accept_batch": (c_int32, [c_void_p, c_int64, c_int32, c_int32, POINTER(msd_batch), POINTER(msd_tree), c_int32,
                                   POINTER(msd_filter), c_void_p, c_int32, c_int32, c_void_p, c_void_p, c_void_p,
                                   c_void_p, c_void_p]),
}

_lib = None


def lib() -> ctypes.CDLL:
    """The loaded library; raises if it is missing (no fallback path exists)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError(f"MSD CUDA library not built: {_LIB_PATH} is missing "
                               "(run python -m paper_2505_14260_gb300.build)")
        L = ctypes.CDLL(_LIB_PATH)
        for name, (res, args) in _SIGNATURES.items():
            f = getattr(L, name)
            f.restype = res
            f.argtypes = args
        _lib = L
    return _lib


class MsdError(RuntimeError):
    def __init__(self, status: int, call: str, msg: str):
        super().__init__(f"{call} -> {STATUS_NAMES.get(status, status)}: {msg}")
        self.status = status


def _ptr(t) -> int | None:
    return None if t is None else t.data_ptr()


def _stream(stream) -> int:
    s = torch.cuda.current_stream() if stream is None else stream
    return s.cuda_stream


class _DevArray:
    """Exposes a raw device pointer to torch.as_tensor (no copy)."""

    def __init__(self, ptr: int, shape, typestr: str):
        self.__cuda_array_interface__ = {"shape": tuple(shape), "typestr": typestr,
                                         "data": (ptr, False), "version": 3}


def device_view(ptr: int, shape, dtype: torch.dtype) -> torch.Tensor:
    typestr = {torch.int32: "<i4", torch.float32: "<f4", torch.int16: "<i2"}[
        torch.int16 if dtype == torch.bfloat16 else dtype]
    t = torch.as_tensor(_DevArray(ptr, shape, typestr), device="cuda")
    return t.view(torch.bfloat16) if dtype == torch.bfloat16 else t


class Tree:
    """Caller-owned device tree arrays in the layout of include/msd.h."""

    def __init__(self, B: int, N: int, device="cuda"):
        self.B, self.N, self.W = B, N, (N + 63) // 64
        self.tokens = torch.zeros(B * N, dtype=torch.int32, device=device)
        self.parent = torch.full((B * N,), -1, dtype=torch.int32, device=device)
        self.depth = torch.zeros(B * N, dtype=torch.int32, device=device)
        self.mask = torch.zeros(B * N * self.W, dtype=torch.int64, device=device)
        self.n_nodes = torch.full((B,), N, dtype=torch.int32, device=device)

    def c(self) -> msd_tree:
        return msd_tree(_ptr(self.tokens), _ptr(self.parent), _ptr(self.depth), _ptr(self.mask),
                        _ptr(self.n_nodes))

    def set_nodes(self, b: int, tokens, parent):
        """Writes the tokens and parent links of request b (n <= N nodes, node 0
        the root; the rest padded). Depths and ancestor masks are derived by the
        library: Engine.plant (msd_tree_complete)."""
        n = len(tokens)
        if n < 1 or n > self.N or len(parent) != n:
            raise ValueError("a tree needs 1..N nodes and one parent entry per node")
        pad = self.N - n
        sl = slice(b * self.N, (b + 1) * self.N)
        dev = self.tokens.device
        self.tokens[sl] = torch.tensor(list(tokens) + [0] * pad, dtype=torch.int32, device=dev)
        self.parent[sl] = torch.tensor(list(parent) + [-1] * pad, dtype=torch.int32, device=dev)
        self.n_nodes[b] = n


class Engine:
    """One context of the C ABI plus the caller-owned buffers of a step."""

    def __init__(self, cfg: msd_config, weights: dict):
        self.cfg = cfg
        self.w = weights             # keeps the borrowed device tensors alive
        L = lib()
        self._layers = (msd_layer * cfg.n_layers)(
            *[msd_layer(*[_ptr(lw[n]) for n in LAYER_FIELDS]) for lw in weights["layers"]])
        d = weights["draft"]
        self._weights = msd_weights(_ptr(weights["embed"]), self._layers, _ptr(weights["final_norm"]),
                                    _ptr(weights["lm_head"]),
                                    msd_layer(*[_ptr(d[n]) for n in LAYER_FIELDS]),
                                    _ptr(weights["draft_fc"]))
        ctx = c_void_p()
        st = L.msd_create(ctypes.byref(cfg), ctypes.byref(self._weights), ctypes.byref(ctx))
        if st != MSD_OK:
            raise MsdError(st, "msd_create", "invalid configuration or allocation failure")
        self.ctx = ctx
        B, N, D = cfg.max_batch, cfg.tree_nodes, cfg.tree_depth
        self.tree = Tree(B, N)
        self.argmax = torch.zeros(B * N, dtype=torch.int32, device="cuda")
        self.path = torch.zeros(B * (D + 1), dtype=torch.int32, device="cuda")
        self.accept_len = torch.zeros(B, dtype=torch.int32, device="cuda")
        self.bonus = torch.zeros(B, dtype=torch.int32, device="cuda")
        self.index_map = torch.zeros(B * (D + 1), dtype=torch.int32, device="cuda")
        self.root_out = torch.zeros(B, dtype=torch.int32, device="cuda")

    def close(self):
        if getattr(self, "ctx", None) is not None and self.ctx.value:
            lib().msd_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, st: int, call: str):
        if st != MSD_OK:
            msg = lib().msd_last_error(self.ctx)
            raise MsdError(st, call, msg.decode() if msg else "")

    # -- the five calls ------------------------------------------------------
    def prefill(self, ids: torch.Tensor, lengths, vis: torch.Tensor | None, vis_off, stream=None):
        """ids: int32 [B, stride] on the device (-1 = visual slot)."""
        B = len(lengths)
        lens = (c_int32 * B)(*[int(x) for x in lengths])
        offs = (c_int64 * B)(*[int(x) for x in vis_off])
        st = lib().msd_prefill(self.ctx, B, lens, _ptr(ids), ids.shape[1], _ptr(vis), offs,
                               _ptr(self.root_out), _stream(stream))
        self._check(st, "msd_prefill")
        return self.root_out

    def draft_tree(self, record: dict | None = None, tree: Tree | None = None, stream=None):
        t = self.tree if tree is None else tree
        rec = None
        if record is not None:
            rec = msd_draft_record(_ptr(record.get("logits")), _ptr(record.get("topk_ids")),
                                   _ptr(record.get("topk_logp")))
        st = lib().msd_draft_tree(self.ctx, ctypes.byref(t.c()),
                                  ctypes.byref(rec) if rec is not None else None, _stream(stream))
        self._check(st, "msd_draft_tree")
        return t

    def verify(self, tree: Tree | None = None, logits: torch.Tensor | None = None, stream=None):
        t = self.tree if tree is None else tree
        st = lib().msd_verify(self.ctx, ctypes.byref(t.c()), _ptr(self.argmax), _ptr(logits),
                              _stream(stream))
        self._check(st, "msd_verify")
        return self.argmax

    def accept_compact(self, tree: Tree | None = None, stream=None):
        t = self.tree if tree is None else tree
        st = lib().msd_accept_compact(self.ctx, ctypes.byref(t.c()), _ptr(self.argmax),
                                      _ptr(self.path), _ptr(self.accept_len), _ptr(self.bonus),
                                      _ptr(self.index_map), _stream(stream))
        self._check(st, "msd_accept_compact")
        return self.path, self.accept_len, self.bonus

    def accept_sample(self, temperature: float, u: torch.Tensor, logits: torch.Tensor | None = None,
                      tree: Tree | None = None, stream=None):
        """Speculative sampling at temperature T > 0 + compaction (msd_accept_sample).
        u: fp32 [B, D+1, k+1] uniforms on the device; logits: the tensor given to
        verify(), or None if verify() kept them in the context."""
        t = self.tree if tree is None else tree
        st = lib().msd_accept_sample(self.ctx, ctypes.byref(t.c()), _ptr(logits), float(temperature),
                                     _ptr(u), _ptr(self.path), _ptr(self.accept_len), _ptr(self.bonus),
                                     _ptr(self.index_map), _stream(stream))
        self._check(st, "msd_accept_sample")
        return self.path, self.accept_len, self.bonus

    def step_sample(self, temperature: float, u: torch.Tensor, stream=None):
        """draft -> verify -> sample/compact at temperature T as one replayed
        CUDA graph (msd_step_sample); u is read when the step runs."""
        st = lib().msd_step_sample(self.ctx, ctypes.byref(self.tree.c()), float(temperature), _ptr(u),
                                   _ptr(self.argmax), _ptr(self.path), _ptr(self.accept_len),
                                   _ptr(self.bonus), _stream(stream))
        self._check(st, "msd_step_sample")
        return self.path, self.accept_len, self.bonus

    def step(self, stream=None):
        """draft -> verify -> accept/compact as one replayed CUDA graph (msd_step)."""
        st = lib().msd_step(self.ctx, ctypes.byref(self.tree.c()), _ptr(self.argmax),
                            _ptr(self.path), _ptr(self.accept_len), _ptr(self.bonus),
                            _stream(stream))
        self._check(st, "msd_step")
        return self.path, self.accept_len, self.bonus

    def step_calls(self, stream=None):
        """The same step as three separate calls (no graph)."""
        self.draft_tree(stream=stream)
        self.verify(stream=stream)
        return self.accept_compact(stream=stream)

    def ar_step(self, out: torch.Tensor | None = None, stream=None):
        """One plain greedy decode step (msd_ar_step): the next token of every request."""
        if out is None:
            if getattr(self, "_ar_out", None) is None:
                self._ar_out = torch.zeros(self.cfg.max_batch, dtype=torch.int32, device="cuda")
            out = self._ar_out
        st = lib().msd_ar_step(self.ctx, _ptr(out), _stream(stream))
        self._check(st, "msd_ar_step")
        return out

    def linear(self, x: torch.Tensor, w: torch.Tensor, y: torch.Tensor, accumulate=False,
               stream=None):
        """y (=|+=) x @ w.T through the library's GEMM (x, w in the model dtype)."""
        st = lib().msd_linear(self.ctx, _ptr(x), x.stride(0), x.shape[0], x.shape[1], _ptr(w),
                              w.shape[0], _ptr(y), y.stride(0), int(accumulate), _stream(stream))
        self._check(st, "msd_linear")
        return y

    def plant(self, tree: Tree, b: int, tokens, parent, stream=None):
        """A caller-planted tree for request b: tokens and parent links are
        copied, depths and ancestor masks derived on the device
        (msd_tree_complete; a parent that does not precede its node is reported
        by the next call as MSD_ERR_DEVICE)."""
        tree.set_nodes(b, tokens, parent)
        st = lib().msd_tree_complete(self.ctx, ctypes.byref(tree.c()), int(b), _stream(stream))
        self._check(st, "msd_tree_complete")
        return tree

    def test_wait_timeout(self, limit_ns: int, stream=None):
        """Test hook: a bounded wait that runs out and sets the status word."""
        st = lib().msd_test_wait_timeout(self.ctx, int(limit_ns), _stream(stream))
        self._check(st, "msd_test_wait_timeout")

    def profile_enable(self, mode=True):
        """0/False off, 1/True CUDA events around separate launches, 2 launch
        stamps inside the replayed step graphs."""
        self._check(lib().msd_profile_enable(self.ctx, int(mode)), "msd_profile_enable")

    def profile_read(self) -> dict:
        p = msd_profile()
        self._check(lib().msd_profile_read(self.ctx, ctypes.byref(p)), "msd_profile_read")
        return {n: getattr(p, n) for n, _ in msd_profile._fields_}

    def profile_slots(self, max_slots: int = 4096) -> list:
        """Per-launch sums of the stamped step graphs since the last call
        (mode 2): GEMM slots in launch order, then the attention launches."""
        buf = (msd_kernel_slot * max_slots)()
        n = c_int32(0)
        self._check(lib().msd_profile_slots(self.ctx, buf, max_slots, ctypes.byref(n)), "msd_profile_slots")
        return [{f: getattr(buf[i], f) for f, _ in msd_kernel_slot._fields_} for i in range(n.value)]

    # -- state ---------------------------------------------------------------
    def state(self) -> dict:
        v = msd_state_view()
        self._check(lib().msd_state(self.ctx, ctypes.byref(v)), "msd_state")
        c = self.cfg
        dt = torch.bfloat16 if c.dtype == MSD_BF16 else torch.float32
        B, nh, S, hd = c.max_batch, c.n_heads, c.max_seq, c.head_dim
        out = {
            "target_kv": device_view(v.target_kv, (c.n_layers, 2, B, nh, S, hd), dt),
            "draft_kv": device_view(v.draft_kv, (2, B, nh, S, hd), dt),
            "seq_len": device_view(v.seq_len, (B,), torch.int32),
            "n_pending": device_view(v.n_pending, (B,), torch.int32),
            "root": device_view(v.root, (B,), torch.int32),
            "lo_offset": int(v.lo_offset),
        }
        if v.lo_offset:     # bf16: the lo planes of the split cache entries
            eb = int(v.elem_bytes)
            out["target_kv_lo"] = device_view(v.target_kv + v.lo_offset * eb, (c.n_layers, 2, B, nh, S, hd), dt)
            out["draft_kv_lo"] = device_view(v.draft_kv + v.lo_offset * eb, (2, B, nh, S, hd), dt)
        return out


class Batch:
    """The rows of a call on a Pages pool (msd_batch): int32 device tensors seqs [n] and
    row_start [n + 1], and the total row count."""

    def __init__(self, seqs: torch.Tensor, row_start: torch.Tensor, rows: int):
        if row_start.numel() != seqs.numel() + 1:
            raise ValueError("row_start has one entry more than seqs")
        self.seqs, self.row_start, self.n, self.rows = _ints(seqs), _ints(row_start), seqs.numel(), int(rows)
        self._c = msd_batch(self.n, _ptr(seqs), _ptr(row_start), self.rows)
        self._ref = ctypes.byref(self._c)

    def c(self):
        return self._ref


def _ints(t: torch.Tensor | None):
    if t is not None and not (t.is_cuda and t.dtype == torch.int32 and t.is_contiguous()):
        raise ValueError("index arrays are contiguous int32 tensors on the GPU")
    return t


class Pages:
    """A pool of K/V pages (msd_pages): many sequences of one model's cache, which share full
    pages. State lives in the tensors kv [layers, n_pages, 2, kv_heads, page_size, head_dim],
    table [max_seqs, max_pages], lens [max_seqs] and refs [n_pages], allocated here unless
    given. A pool made on fresh tensors is empty; on given ones call restore() first. Calls
    are queued: an error that only the device can see (too few pages, bad lists) is raised by a
    later call, and what was queued behind a page operation that failed has done nothing."""

    def __init__(self, *, dtype: str, layers: int, heads: int, kv_heads: int, head_dim: int, page_size: int,
                 n_pages: int, max_seqs: int, max_pages: int, rot_dim: int | None = None, rot_sections=None,
                 rot_interleaved: bool = False, rope_base: float = 10000.0, kv=None, table=None, lens=None,
                 refs=None, device="cuda"):
        if dtype not in ("bf16", "f32"):
            raise ValueError('dtype is "bf16" or "f32"')
        rot_dim = head_dim if rot_dim is None else rot_dim
        sections = (rot_dim // 2, 0, 0) if rot_sections is None else rot_sections
        self.cfg = msd_pages_config(MSD_BF16 if dtype == "bf16" else MSD_F32, layers, heads, kv_heads, head_dim,
                                    page_size, n_pages, max_seqs, max_pages, rot_dim, (c_int32 * 3)(*sections),
                                    int(rot_interleaved), rope_base)
        self.dtype = torch.bfloat16 if dtype == "bf16" else torch.float32
        self._H, self._K, self._hd = heads, kv_heads, head_dim
        fresh = lens is None
        shape = (layers, n_pages, 2, kv_heads, page_size, head_dim)
        i32 = dict(dtype=torch.int32, device=device)
        self.kv = torch.empty(shape, dtype=self.dtype, device=device) if kv is None else kv
        self.table = torch.full((max_seqs, max_pages), -1, **i32) if table is None else table
        self.lens = torch.zeros(max_seqs, **i32) if lens is None else lens
        self.refs = torch.zeros(n_pages, **i32) if refs is None else refs
        if self.kv.dtype != self.dtype or tuple(self.kv.shape) != shape or not self.kv.is_contiguous() or not self.kv.is_cuda:
            raise ValueError(f"kv is a contiguous tensor of shape {shape} in the pool's type, on the GPU")
        for t, n in ((self.table, max_seqs * max_pages), (self.lens, max_seqs), (self.refs, n_pages)):
            if _ints(t).numel() != n:
                raise ValueError("table, lens and refs have an entry per cell, sequence and page")
        self._dev = self.kv.device.index
        buf = msd_pages_buffers(_ptr(self.kv), _ptr(self.table), _ptr(self.lens), _ptr(self.refs))
        self.ptr = c_void_p()
        st = lib().msd_pages_create(ctypes.byref(self.cfg), ctypes.byref(buf), ctypes.byref(self.ptr))
        if st != MSD_OK:
            raise MsdError(st, "msd_pages_create", "invalid configuration or allocation failure")
        if fresh:
            self.restore()

    def close(self):
        if getattr(self, "ptr", None) is not None and self.ptr.value:
            lib().msd_pages_destroy(self.ptr)
            self.ptr = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, st: int, call: str):
        if st != MSD_OK:
            raise MsdError(st, call, lib().msd_pages_last_error(self.ptr).decode())

    def _rows(self, t: torch.Tensor, heads: int, rows: int) -> int:
        """The row stride of q, k, v or out: [rows, heads, head_dim] or [rows, heads * head_dim]."""
        hd, shape, stride = self._hd, t.shape, t.stride()
        if not t.is_cuda or not (shape == (rows, heads * hd) and stride[1] == 1 or
                                 shape == (rows, heads, hd) and stride[2] == 1 and (stride[1] == hd or heads == 1)):
            raise ValueError(f"expected {rows} rows of {heads} heads of {hd} elements, one after another, on the GPU")
        return stride[0] if rows > 1 else heads * hd

    def _on(self, stream) -> int:
        """The stream of a call as a number; the current one without making a Stream object
        (which takes longer than a small launch)."""
        return torch._C._cuda_getCurrentRawStream(self._dev) if stream is None else stream.cuda_stream

    def restore(self, stream=None):
        """Takes lens and table as they are; refs and free pages follow from them."""
        self._check(lib().msd_pages_restore(self.ptr, self._on(stream)), "msd_pages_restore")

    def reserve(self, batch: Batch, stream=None):
        """Room for the batch's rows at the end of their sequences."""
        self._check(lib().msd_pages_reserve(self.ptr, batch.c(), self._on(stream)), "msd_pages_reserve")

    def fork(self, src: torch.Tensor, dst: torch.Tensor, deep: bool = False, stream=None):
        """Unused sequences dst[i] become copies of src[i]; full pages are shared unless deep."""
        if src.numel() != dst.numel():
            raise ValueError("src and dst have one entry per copy")
        self._check(lib().msd_pages_fork(self.ptr, dst.numel(), _ptr(_ints(src)), _ptr(_ints(dst)), int(deep),
                                         self._on(stream)), "msd_pages_fork")

    def compact(self, batch: Batch, keep: torch.Tensor | None, n_keep: torch.Tensor, stream=None):
        """Of the batch's rows keep keep[i, :n_keep[i]] (None: the first n_keep[i])."""
        n = batch.n
        if n_keep.numel() != n or (keep is not None and keep.shape[0] != n):
            raise ValueError("keep and n_keep have an entry per sequence")
        self._check(lib().msd_pages_compact(self.ptr, batch.c(), _ptr(_ints(keep)),
                                            0 if keep is None else keep.shape[1], _ptr(_ints(n_keep)),
                                            self._on(stream)), "msd_pages_compact")

    def free(self, seqs: torch.Tensor, stream=None):
        self._check(lib().msd_pages_free(self.ptr, seqs.numel(), _ptr(_ints(seqs)), self._on(stream)),
                    "msd_pages_free")

    def positions(self, batch: Batch, span_start, spans, pos: torch.Tensor, next_pos: torch.Tensor | None = None,
                  first: torch.Tensor | None = None, stream=None):
        """pos [3, rows] of interleaved text, images and video (msd_rope_positions)."""
        if pos.shape[0] != 3 or pos.shape[1] < batch.rows:
            raise ValueError("pos is [3, rows]")
        if span_start is not None and (span_start.numel() != batch.seqs.numel() + 1 or spans.shape[-1] != 5):
            raise ValueError("span_start has an entry per sequence and one more, spans five per span")
        for t in (next_pos, first):
            if t is not None and t.numel() != batch.seqs.numel():
                raise ValueError("next and first have an entry per sequence")
        self._check(lib().msd_rope_positions(self.ptr, batch.c(), _ptr(_ints(span_start)), _ptr(_ints(spans)),
                                             0 if spans is None else spans.shape[0], _ptr(_ints(first)),
                                             _ptr(_ints(pos)), pos.stride(0),
                                             _ptr(_ints(next_pos)), self._on(stream)), "msd_rope_positions")
        return pos

    def rope_append(self, layer: int, batch: Batch, q, k, v, pos: torch.Tensor, q_out, stream=None):
        """Rotated q into q_out, rotated k and v into the rows' slots (msd_rope_append).
        pos: [3, rows], or [1, rows] where the three axes agree."""
        n, dt, H, K = batch.rows, q.dtype, self._H, self._K
        if k.dtype != dt or v.dtype != dt or dt not in (torch.float32, torch.bfloat16) or q_out.dtype != self.dtype:
            raise ValueError("q, k and v have one type, fp32 or the cache's; q_out the cache's")
        axes, width = pos.shape
        if axes not in (1, 3) or width < n:
            raise ValueError("pos is [3, rows] or [1, rows]")
        st = lib().msd_rope_append(
            self.ptr, layer, batch.c(), q.data_ptr(), self._rows(q, H, n), k.data_ptr(), self._rows(k, K, n),
            v.data_ptr(), self._rows(v, K, n), MSD_F32 if dt == torch.float32 else MSD_BF16, _ints(pos).data_ptr(),
            width if axes == 3 else 0, q_out.data_ptr(), self._rows(q_out, H, n), self._on(stream))
        if st:
            self._check(st, "msd_rope_append")
        return q_out

    def attention(self, layer: int, batch: Batch, q, out, lse: torch.Tensor | None = None, tree: Tree | None = None,
                  window: int = 0, sinks: int = 0, stream=None):
        """The batch's rows over their sequences' pages (msd_pages_attention). lse: fp32
        [rows, heads]; tree: one per listed sequence, its rows the tree's nodes."""
        n, H = batch.rows, self._H
        if q.dtype != self.dtype or out.dtype != self.dtype:
            raise ValueError("q and out have the cache's type")
        if lse is not None and not (lse.is_cuda and lse.dtype == torch.float32 and lse.is_contiguous() and lse.numel() == n * H):
            raise ValueError("lse is a contiguous fp32 tensor [rows, heads] on the GPU")
        if tree is not None and (tree.B != batch.n or not tree.mask.is_cuda):
            raise ValueError("a tree per listed sequence, on the GPU")
        st = lib().msd_pages_attention(
            self.ptr, layer, batch.c(), None if tree is None else ctypes.byref(tree.c()), 0 if tree is None else tree.N,
            window, sinks, q.data_ptr(), self._rows(q, H, n), out.data_ptr(), self._rows(out, H, n), _ptr(lse),
            self._on(stream))
        if st:
            self._check(st, "msd_pages_attention")
        return out


_TYPES = {torch.float32: MSD_F32, torch.bfloat16: MSD_BF16}
_F32 = (torch.float32,)


def _matrix(t: torch.Tensor, what: str, types=_TYPES) -> int:
    """The row stride of a 2-D tensor on the current GPU whose rows are contiguous."""
    if t.dim() != 2 or t.dtype not in types or not t.is_cuda:
        _refuse_matrix(what, types)
    (rows, width), (ld, step) = t.shape, t.stride()
    if step != 1 and width > 1:
        _refuse_matrix(what, types)
    if t.get_device() != torch._C._cuda_getDevice():
        raise ValueError(f"{what} is not on the current GPU")
    return ld if rows > 1 else width


def _refuse_matrix(what: str, types):
    raise ValueError(f"{what}: a matrix with contiguous rows on the GPU, {' or '.join(str(d) for d in types)}")


def _vector(t: torch.Tensor | None, what: str, dtype: torch.dtype, n: int, device) -> int | None:
    """The address of n contiguous values (None stays None)."""
    if t is None:
        return None
    if t.dtype != dtype or t.device != device or t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{what}: {n} contiguous values of {dtype} on {device}")
    return t.data_ptr()


def _raw_stream(stream, device) -> int:
    return torch._C._cuda_getCurrentRawStream(device if type(device) is int else device.index) if stream is None else stream.cuda_stream


def _memory_of(stream):
    """Tensors made inside are memory that a call on `stream` (None: the current one) may write now."""
    return contextlib.nullcontext() if stream is None else torch.cuda.stream(stream)


def _call(st: int, call: str):
    if st != MSD_OK:
        raise MsdError(st, call, "bad sizes, strides or alignment" if st == MSD_ERR_INVALID else "launch failed")


class Weight4:
    """A weight matrix [out, in] in 4 bits (msd_weight4): codes uint8 [out, in / 2], scales bf16
    [out, groups] and zeros uint8 [out, groups] or None, held by the caller. Weight4.of(w) makes
    one from a bf16 or fp32 matrix."""

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, zeros: torch.Tensor | None = None, group: int = 128):
        if codes.dim() != 2 or codes.dtype != torch.uint8 or not codes.is_cuda or not codes.is_contiguous():
            raise ValueError("codes are a contiguous uint8 matrix on the GPU")
        if group not in (32, 64, 128):
            raise ValueError("group is 32, 64 or 128")
        self.o, self.k, self.group = codes.shape[0], 2 * codes.shape[1], group
        self.codes, self.scales, self.zeros, self._device = codes, scales, zeros, codes.get_device()
        n = self.o * -(-self.k // group)
        self._c = msd_weight4(codes.data_ptr(), _vector(scales, "scales", torch.bfloat16, n, codes.device),
                              _vector(zeros, "zeros", torch.uint8, n, codes.device), self.o, self.k, group)
        self._ref = ctypes.byref(self._c)

    @classmethod
    def of(cls, w: torch.Tensor, group: int = 128, zeros: bool = False, stream=None) -> "Weight4":
        """w [out, in] in 4 bits (msd_quantize4). Codes, scales and zeros are memory of the stream that the call runs
        on, as tensors made there are: another stream uses them behind that one, and as long as they are held."""
        _matrix(w, "w")
        if group not in (32, 64, 128):
            raise ValueError("group is 32, 64 or 128")
        o, k = w.shape
        n = -(-k // group)
        with _memory_of(stream):
            self = cls(torch.empty(o, k // 2, dtype=torch.uint8, device=w.device),
                       torch.empty(o, n, dtype=torch.bfloat16, device=w.device),
                       torch.empty(o, n, dtype=torch.uint8, device=w.device) if zeros else None, group)
        return self.quantize(w, stream=stream)

    def quantize(self, w: torch.Tensor, values: torch.Tensor | None = None, stream=None) -> "Weight4":
        """Codes, scales and zeros from w; values (optional, w's type): what they stand for."""
        ld, ldv = _matrix(w, "w"), 0
        if w.shape != (self.o, self.k):
            raise ValueError(f"w is [{self.o}, {self.k}]")
        if values is not None:
            ldv = _matrix(values, "values")
            if values.shape != w.shape or values.dtype != w.dtype:
                raise ValueError("values has w's shape and type")
        self._on(w)
        _call(lib().msd_quantize4(w.data_ptr(), ld, _TYPES[w.dtype], self._ref, _ptr(values), ldv,
                                  _raw_stream(stream, w.device)), "msd_quantize4")
        return self

    def linear(self, x: torch.Tensor, y: torch.Tensor, accumulate: bool = False, stream=None) -> torch.Tensor:
        """y (=|+=) x w^T (msd_linear4): x [m, in] bf16 or fp32, y [m, out] fp32."""
        ldx, ldy, m, device = _matrix(x, "x"), _matrix(y, "y", _F32), len(x), x.get_device()
        if x.shape[1] != self.k or y.shape != (m, self.o):
            raise ValueError(f"x is [m, {self.k}] and y [m, {self.o}]")
        if device != self._device:
            raise ValueError("the weight is on another GPU")
        st = lib().msd_linear4(x.data_ptr(), ldx, _TYPES[x.dtype], m, self._ref, y.data_ptr(), ldy, int(accumulate),
                               _raw_stream(stream, device))
        if st:
            _call(st, "msd_linear4")
        return y

    def _on(self, t: torch.Tensor):
        if t.device != self.codes.device:
            raise ValueError("the weight is on another GPU")


class Filter:
    """Settings of rows of logits (msd_filter), a value per row (sample) or per sequence
    (accept): fp32 temperature, top_p and min_p, int32 top_k, each None where it is off."""

    def __init__(self, temperature: torch.Tensor | None = None, top_k: torch.Tensor | None = None,
                 top_p: torch.Tensor | None = None, min_p: torch.Tensor | None = None):
        given = [t for t in (temperature, top_k, top_p, min_p) if t is not None]
        self.n = given[0].numel() if given else None
        self.device = given[0].device if given else None
        if given and not given[0].is_cuda:
            raise ValueError("settings are tensors on the GPU")
        f32 = lambda t, what: _vector(t, what, torch.float32, self.n, self.device)  # noqa: E731
        self._c = msd_filter(f32(temperature, "temperature"), _vector(top_k, "top_k", torch.int32, self.n, self.device),
                             f32(top_p, "top_p"), f32(min_p, "min_p"))
        self._held = given
        self._ref = ctypes.byref(self._c)

    def _for(self, n: int, device):
        if self.n is not None and (self.n != n or self.device != device):
            raise ValueError(f"settings have {n} values each, on the logits' GPU")
        return self._ref


def sample(logits: torch.Tensor, u: torch.Tensor, settings: Filter | None, tokens: torch.Tensor,
           logp: torch.Tensor | None = None, probs: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """A token for each row of logits [rows, vocab] (fp32 or bf16) from the uniforms u [rows]
    (msd_sample). tokens: int32 [rows]; logp: fp32 [rows]; probs: fp32 [rows, vocab]."""
    ld, dev, (rows, vocab) = _matrix(logits, "logits"), logits.device, logits.shape
    ldp = 0
    if probs is not None:
        ldp = _matrix(probs, "probs", _F32)
        if probs.shape != logits.shape:
            raise ValueError("probs has the logits' shape")
    st = lib().msd_sample(logits.data_ptr(), ld, _TYPES[logits.dtype], rows, vocab,
                          None if settings is None else settings._for(rows, dev),
                          _vector(u, "u", torch.float32, rows, dev), _vector(tokens, "tokens", torch.int32, rows, dev),
                          _vector(logp, "logp", torch.float32, rows, dev), _ptr(probs), ldp, _raw_stream(stream, dev))
    if st:
        _call(st, "msd_sample")
    return tokens


def accept(logits: torch.Tensor, batch: Batch, tree: Tree, u: torch.Tensor, settings: Filter | None, path: torch.Tensor,
           accept_len: torch.Tensor, bonus: torch.Tensor, stream=None):
    """Speculative sampling over a batch's drafted trees (msd_accept_batch). logits [rows, vocab]:
    the batch's rows are the trees' nodes; u [n, depth + 1, children + 1]; path [n, depth + 1],
    accept_len [n] and bonus [n] int32. path and accept_len + 1 go to Pages.compact."""
    ld, dev, n, rows = _matrix(logits, "logits"), logits.device, batch.n, batch.rows
    if logits.shape[0] != rows or tree.B != n:
        raise ValueError("a row of logits per row of the batch, a tree per sequence")
    if u.dim() != 3 or u.shape[0] != n or path.shape != (n, u.shape[1]):
        raise ValueError("u is [n, depth + 1, children + 1], path [n, depth + 1]")
    for t in (batch.seqs, batch.row_start):
        if t.device != dev:
            raise ValueError("batch, tree and logits are on one GPU")
    for what, t, size in (("tokens", tree.tokens, n * tree.N), ("parent", tree.parent, n * tree.N), ("n_nodes", tree.n_nodes, n)):
        _vector(t, f"the tree's {what}", torch.int32, size, dev)
    with _memory_of(stream):
        scratch = torch.empty(2 * rows, dtype=torch.int32, device=dev)
    st = lib().msd_accept_batch(
        logits.data_ptr(), ld, _TYPES[logits.dtype], logits.shape[1], batch.c(), ctypes.byref(tree.c()), tree.N,
        None if settings is None else settings._for(n, dev), _vector(u, "u", torch.float32, u.numel(), dev),
        u.shape[1] - 1, u.shape[2] - 1, scratch.data_ptr(), _vector(path, "path", torch.int32, path.numel(), dev),
        _vector(accept_len, "accept_len", torch.int32, n, dev), _vector(bonus, "bonus", torch.int32, n, dev),
        _raw_stream(stream, dev))
    if st:
        _call(st, "msd_accept_batch")
    return path, accept_len, bonus


def make_config(wl, max_seq: int, batch: int | None = None) -> msd_config:
    """msd_config of a synth.Workload."""
    return msd_config(n_layers=wl.n_layers, hidden=wl.hidden, n_heads=wl.n_heads,
                      head_dim=wl.head_dim, ffn=wl.ffn, vocab=wl.vocab, rms_eps=wl.rms_eps,
                      rope_base=wl.rope_base,
                      dtype=MSD_BF16 if wl.dtype == "bf16" else MSD_F32,
                      max_batch=wl.batch if batch is None else batch, max_seq=max_seq,
                      tree_nodes=wl.tree_nodes, tree_depth=wl.tree_depth, topk=wl.topk,
                      draft_input=DRAFT_INPUTS[wl.draft_input])


def upload_prompts(prompts, device="cuda"):
    """Packs synth prompts into the msd_prefill layout: ids [B, stride] int32,
    lengths, concatenated visual rows and their per-request offsets."""
    B = len(prompts)
    stride = max(p.length for p in prompts)
    ids = torch.full((B, stride), 0, dtype=torch.int32)
    vis_rows, offs, off = [], [], 0
    for b, p in enumerate(prompts):
        ids[b, :p.length] = torch.from_numpy(p.ids)
        offs.append(off)
        vis_rows.append(p.vis)
        off += p.vis.shape[0]
    vis = torch.cat(vis_rows, 0).to(device) if off > 0 else None
    return ids.to(device), [p.length for p in prompts], vis, offs
