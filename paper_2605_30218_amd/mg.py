"""ctypes binding of libmg.so (include/mg.h, include/mg_ops.h).

Argument marshalling only: every step of the hot path runs in the library's HIP
kernels.  torch supplies device memory and the stream; tensors are passed as raw
device pointers.  load() raises when the library is missing: there is no fallback.
"""
from __future__ import annotations

import collections
import ctypes as C
import os

import numpy as np
import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libmg.so")

MG_OK = 0
MG_ERR_WORKSPACE = -3
# repair actions (include/mg.h)
REPAIR_ON_MISMATCH, REPAIR_TOKEN_ONLY, REPAIR_COPY_ALWAYS = 0, 1, 2
KIND_FAST_GEMM, KIND_FAST_ATTN, KIND_CANON_GEMV, KIND_CANON_ATTN, KIND_GATE = range(5)
WPL = 12

_STATUS = {0: "ok", -1: "invalid argument", -2: "unsupported model shape", -3: "workspace or KV pool too small",
           -4: "HIP runtime error", -5: "invalid state"}


class MgError(RuntimeError):
    def __init__(self, call, status):
        super().__init__(f"{call} failed: {_STATUS.get(status, status)} ({status})")
        self.status = status


class MgModelCfg(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_layers", "d_model", "n_q_heads", "n_kv_heads", "head_dim", "d_ffn",
                                         "vocab", "qkv_bias")] + \
               [("rope_theta", C.c_float), ("rms_eps", C.c_float)] + \
               [(n, C.c_int32) for n in ("page_size", "max_batch", "max_pages_per_row", "n_pages", "max_prefill")]


class MgKv8Cache(C.Structure):
    _fields_ = [("codes", C.c_void_p), ("scales", C.c_void_p), ("n_pages", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32)]


class MgKv8AttnArgs(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_rows", "n_tokens", "n_q_heads", "max_new", "max_len",
                                         "max_pages_per_row", "window")] + \
               [("scale", C.c_float), ("softcap", C.c_float), ("q", C.c_void_p), ("q_stride", C.c_int64),
                ("out", C.c_void_p), ("out_stride", C.c_int64), ("page_table", C.c_void_p), ("lens", C.c_void_p),
                ("cu_new", C.c_void_p)]


# name -> (restype, argtypes); the set of C-ABI symbols the binding uses
P, I, F, I64, SZ = C.c_void_p, C.c_int, C.c_float, C.c_int64, C.c_size_t
SIGNATURES = {
    "mg_weight_count": (I, [P]),
    "mg_kv_pool_bytes": (SZ, [P]),
    "mg_kv_col_elems": (SZ, [P]),
    "mg_workspace_bytes": (SZ, [P]),
    "mg_status_string": (C.c_char_p, [I]),
    "mg_create": (I, [P, P, P, SZ, P, SZ, P]),
    "mg_destroy": (I, [P]),
    "mg_decode_step": (I, [P, I, P, P, P, P, P]),
    "mg_margin_gate": (I, [P, I, P, P, F, P, P, P, P, P, P, P]),
    "mg_margin_gate_noalloc": (I, [I, I, P, P, F, P, P, P, P, P, P]),
    "mg_verify_rows": (I, [P, I, P, P, P, P, P, P, P, P, P]),
    "mg_repair_kv_column": (I, [P, I, P, P, P, P, P, P, P, P, P, P]),
    "mg_repair_kv_column_action": (I, [P, I, P, P, P, P, P, P, P, P, P, I, P]),
    "mg_verify_rows_mfma": (I, [P, I, P, P, P, P, P, P, P, P]),
    "mg_prefill": (I, [P, I, P, P, P, P, P]),
    "mg_advance": (I, [P, I, P, P, P, P]),
    "mg_kv8_code_bytes": (SZ, [I, I, I]),
    "mg_kv8_scale_bytes": (SZ, [I, I, I]),
    "mg_batch_plan": (I, [I, I, P, P, P, P, I, P, P, P, P, P, P, P, P, P]),
    "mg_kv8_append": (I, [P, I, P, I64, P, I64, P, P]),
    "mg_kv8_read": (I, [P, I, P, P, I64, P, I64, P]),
    "mg_kv8_attention_workspace_bytes": (SZ, [P, P]),
    "mg_kv8_attention": (I, [P, P, P, SZ, P]),
    "mg_profile_begin": (I, [P, I, I]),
    "mg_profile_end": (I, [P, I, P, P, P, P]),
    "mg_op_copy": (I, [I64, P, P, P]),
    "mg_op_read_stream_sink_words": (I, []),
    "mg_op_read_stream": (I, [I64, P, P, P]),
    "mg_op_probe_bf16": (I, [I64, P, P, P]),
    "mg_op_probe_exp": (I, [I64, P, P, P]),
    "mg_op_probe_divsqrt": (I, [I64, P, P, P, P, P]),
    "mg_op_probe_mfma_fma": (I, [I, P, P, P, P, P]),
    "mg_op_probe_mfma4_fma": (I, [I, P, P, P, P, P]),
    "mg_op_linear_workspace_bytes": (SZ, [I, I, I]),
    "mg_op_linear": (I, [I, I, I, I, P, P, P, P, P, SZ, P]),
    "mg_op_fast_gemm_config": (I, [I, I, I, I, P, P]),
    "mg_op_canon_gemv_config": (I, [I, I, I, I, I, P, P, P, P, P]),
    "mg_op_rmsnorm": (I, [I, I, P, P, F, P, P]),
    "mg_op_decode_step_taps": (I, [P, I, P, P, P, P, P, P]),
}

_lib = None


def load():
    """Open libmg.so (built in-tree by build_lib.py).  Raises if it is not there."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2605_30218_amd.build_lib` "
                               "(or __graft_entry__.build()); there is no fallback path")
        lib = C.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            f = getattr(lib, name)
            f.restype = res
            f.argtypes = args
        _lib = lib
    return _lib


def host_count_slot():
    """A few int32 of coherent, mapped pinned host memory (hipHostMalloc), for a count that
    a kernel stores with system scope and the host polls.  Returns (device pointer, numpy
    view of the int32s).  The memory is held until the process ends."""
    hip = C.CDLL("libamdhip64.so")
    host = C.c_void_p()
    flags = 0x40000000 | 0x2  # hipHostMallocCoherent | hipHostMallocMapped
    if hip.hipHostMalloc(C.byref(host), C.c_size_t(64), C.c_uint(flags)) != 0 or not host.value:
        raise RuntimeError("hipHostMalloc of the gate count slot failed")
    dev = C.c_void_p()
    if hip.hipHostGetDevicePointer(C.byref(dev), host, C.c_uint(0)) != 0 or not dev.value:
        raise RuntimeError("hipHostGetDevicePointer of the gate count slot failed")
    view = np.ctypeslib.as_array((C.c_int32 * 16).from_address(host.value))
    return dev.value, view


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _stream(stream=None):
    if stream is None:
        stream = torch.cuda.current_stream()
    return stream.cuda_stream


def _check(call, rc):
    if rc != MG_OK:
        raise MgError(call, rc)


def make_cfg(shape, max_batch, max_pages_per_row, n_pages, max_prefill=0) -> MgModelCfg:
    return MgModelCfg(shape.n_layers, shape.d_model, shape.n_q_heads, shape.n_kv_heads, shape.head_dim,
                      shape.d_ffn, shape.vocab, int(shape.qkv_bias), float(shape.rope_theta), float(shape.rms_eps),
                      shape.page_size, max_batch, max_pages_per_row, n_pages, max_prefill)


class Engine:
    """A libmg context over caller-owned device memory: weights (list of int16 tensors holding bf16
    bits, None for absent biases), the paged KV pool and the workspace."""

    def __init__(self, shape, weights, max_batch, max_pages_per_row, n_pages, max_prefill=0, device="cuda"):
        self.lib = load()
        self.shape = shape
        self.cfg = make_cfg(shape, max_batch, max_pages_per_row, n_pages, max_prefill)
        self.device = torch.device(device)
        nw = self.lib.mg_weight_count(C.byref(self.cfg))
        assert len(weights) == nw, (len(weights), nw)
        self.weights = [None if w is None else w.to(self.device) for w in weights]
        self._wtab = (C.c_void_p * nw)(*[None if w is None else w.data_ptr() for w in self.weights])
        kv_bytes = self.lib.mg_kv_pool_bytes(C.byref(self.cfg))
        ws_bytes = self.lib.mg_workspace_bytes(C.byref(self.cfg))
        if ws_bytes == 0:
            raise MgError("mg_workspace_bytes", -2)
        self.kv_pool = torch.zeros(kv_bytes // 2, dtype=torch.int16, device=self.device)
        self.workspace = torch.zeros(ws_bytes, dtype=torch.uint8, device=self.device)
        self.col_elems = self.lib.mg_kv_col_elems(C.byref(self.cfg))
        ctx = C.c_void_p()
        _check("mg_create", self.lib.mg_create(C.byref(self.cfg), self._wtab, self.kv_pool.data_ptr(), kv_bytes,
                                               self.workspace.data_ptr(), ws_bytes, C.byref(ctx)))
        self.ctx = ctx

    def close(self):
        if getattr(self, "ctx", None):
            self.lib.mg_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def kv_view(self):
        s, c = self.shape, self.cfg
        return self.kv_pool.view(s.n_layers, c.n_pages, 2, s.n_kv_heads, s.page_size, s.head_dim)

    # the C-ABI calls, same names without the mg_ prefix
    def decode_step(self, B, tokens, positions, page_table, logits, stream=None):
        _check("mg_decode_step", self.lib.mg_decode_step(self.ctx, B, _ptr(tokens), _ptr(positions),
                                                         _ptr(page_table), _ptr(logits), _stream(stream)))

    def decode_step_taps(self, B, tokens, positions, page_table, logits, x_taps, stream=None):
        """mg_op_decode_step_taps: the fast step plus the residual stream at every layer boundary
        (x_taps int16 [(n_layers + 1), B, d_model] holding bf16 bits)."""
        _check("mg_op_decode_step_taps", self.lib.mg_op_decode_step_taps(
            self.ctx, B, _ptr(tokens), _ptr(positions), _ptr(page_table), _ptr(logits), _ptr(x_taps),
            _stream(stream)))

    def margin_gate(self, B, logits, protected_mask, tau, top1, margin, gate, gated_rows, n_gated,
                    n_gated_host=None, stream=None):
        """n_gated_host: optional pinned CPU int32 tensor that receives the count too."""
        _check("mg_margin_gate", self.lib.mg_margin_gate(self.ctx, B, _ptr(logits), _ptr(protected_mask), float(tau),
                                                         _ptr(top1), _ptr(margin), _ptr(gate), _ptr(gated_rows),
                                                         _ptr(n_gated), _ptr(n_gated_host), _stream(stream)))

    def verify_rows(self, n, rows, n_dev, tokens, positions, page_table, v_logits, v_tok, v_kvcol, stream=None):
        _check("mg_verify_rows", self.lib.mg_verify_rows(self.ctx, n, _ptr(rows), _ptr(n_dev), _ptr(tokens),
                                                         _ptr(positions), _ptr(page_table), _ptr(v_logits),
                                                         _ptr(v_tok), _ptr(v_kvcol), _stream(stream)))

    def repair_kv_column(self, n, rows, n_dev, positions, page_table, top1, v_tok, v_kvcol, emitted, n_repaired,
                         stream=None):
        _check("mg_repair_kv_column", self.lib.mg_repair_kv_column(
            self.ctx, n, _ptr(rows), _ptr(n_dev), _ptr(positions), _ptr(page_table), _ptr(top1), _ptr(v_tok),
            _ptr(v_kvcol), _ptr(emitted), _ptr(n_repaired), _stream(stream)))

    def verify_rows_mfma(self, n, rows, tokens, positions, page_table, v_logits, v_tok, v_kvcol, stream=None):
        _check("mg_verify_rows_mfma", self.lib.mg_verify_rows_mfma(
            self.ctx, n, _ptr(rows), _ptr(tokens), _ptr(positions), _ptr(page_table), _ptr(v_logits), _ptr(v_tok),
            _ptr(v_kvcol), _stream(stream)))

    def repair_kv_column_action(self, n, rows, n_dev, positions, page_table, top1, v_tok, v_kvcol, emitted,
                                n_repaired, action, stream=None):
        _check("mg_repair_kv_column_action", self.lib.mg_repair_kv_column_action(
            self.ctx, n, _ptr(rows), _ptr(n_dev), _ptr(positions), _ptr(page_table), _ptr(top1), _ptr(v_tok),
            _ptr(v_kvcol), _ptr(emitted), _ptr(n_repaired), int(action), _stream(stream)))

    def prefill(self, n_items, tokens, positions, item_rows, page_table, stream=None):
        _check("mg_prefill", self.lib.mg_prefill(self.ctx, n_items, _ptr(tokens), _ptr(positions), _ptr(item_rows),
                                                 _ptr(page_table), _stream(stream)))

    def advance(self, B, emitted, tokens, positions, stream=None):
        _check("mg_advance", self.lib.mg_advance(self.ctx, B, _ptr(emitted), _ptr(tokens), _ptr(positions),
                                                 _stream(stream)))

    def profile_begin(self, kind, max_launches):
        _check("mg_profile_begin", self.lib.mg_profile_begin(self.ctx, kind, max_launches))

    def profile_end(self, kind):
        n, ms, b, f = C.c_int(), C.c_double(), C.c_double(), C.c_double()
        _check("mg_profile_end", self.lib.mg_profile_end(self.ctx, kind, C.byref(n), C.byref(ms), C.byref(b),
                                                         C.byref(f)))
        return n.value, ms.value, b.value, f.value


def margin_gate_noalloc(B, V, logits, protected_mask, tau, top1, margin, gate, gated_rows, n_gated, stream=None):
    """mg_margin_gate_noalloc: the margin gate with no context and no allocation (its scratch is a
    static device array of the library)."""
    _check("mg_margin_gate_noalloc", load().mg_margin_gate_noalloc(
        int(B), int(V), _ptr(logits), _ptr(protected_mask), float(tau), _ptr(top1), _ptr(margin), _ptr(gate),
        _ptr(gated_rows), _ptr(n_gated), _stream(stream)))


# ---------------------------------------------------------------- batch plan and 8-bit K/V cache

# A decode step makes these calls once a layer, and their kernels take some microseconds: the checks are
# plain comparisons, messages are made only when one fails, and the device is switched only when
# the tensors are on another than the current one.  As with torch's own operators, tensors that a call makes
# belong to the stream it runs on: a program that then uses them on another one waits, and records them there.

BatchPlan = collections.namedtuple("BatchPlan", "cu_new lens admitted positions rows slots n_left")
_BF16 = (torch.bfloat16, torch.int16)
_I32 = 1 << 31
_raw_stream = torch._C._cuda_getCurrentRawStream if hasattr(torch._C, "_cuda_getCurrentRawStream") else None

_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _refuse(name, t, want):
    what = f"{t.dtype} {tuple(t.shape)} strides {t.stride()} on {t.device}" if isinstance(t, torch.Tensor) else repr(t)
    raise ValueError(f"{name}: {want} is needed, got {what}")


def _ints(name, t, device, numel=None):
    """The address of an int32 tensor of the call's device, contiguous, with the given number of values."""
    if t.dtype is not torch.int32 or t.device != device or not t.is_contiguous() or \
            (numel is not None and t.numel() != numel):
        _refuse(name, t, f"a contiguous int32 tensor of {'any' if numel is None else numel} values on {device}")
    return t.data_ptr()


def _call(name, device, stream, fn, *args):
    """fn(*args, stream) on the tensors' device, on the given stream or the device's current one."""
    if device.type != "cuda":
        raise ValueError(f"{name}: tensors on the GPU are needed, got {device}")
    if stream is not None and stream.device != device:
        raise ValueError(f"{name}: a stream of {device} is needed, got one of {stream.device}")
    if device.index != _current_device():
        with torch.cuda.device(device):
            return _call(name, device, stream, fn, *args)
    if stream is not None:
        s = stream.cuda_stream
    elif _raw_stream is not None:
        s = _raw_stream(device.index)
    else:
        s = torch.cuda.current_stream(device).cuda_stream
    rc = fn(*args, s)
    if rc != MG_OK:
        raise MgError(name, rc)


def _new(shape, dtype, device, stream):
    """A tensor of torch's allocator that the call's stream may write: of that stream's own memory, which
    neither earlier work of the current one still reads nor later work takes too soon."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def batch_plan(ctx_len, n_new, free_pages, n_free, page_table, max_tokens, out=None, stream=None):
    """mg_batch_plan: pages, slots and per-token lists of a batch from its requests' lengths.  All
    tensors int32 on one GPU: ctx_len, n_new [B], free_pages [any], n_free [1] (the count in use, at
    most free_pages' length), page_table [B, max_pages] (updated in place).  out: a BatchPlan to write into, whose tensors the
    caller keeps (a captured step), or None for new ones."""
    dev, M = ctx_len.device, int(max_tokens)
    if page_table.dim() != 2:
        _refuse("page_table", page_table, "[B, max_pages]")
    if not 0 <= M <= 1 << 30:
        _refuse("max_tokens", M, "0 .. 2^30")
    B, maxp = page_table.shape
    count = _ints("n_free", n_free, dev, 1)
    args = (_ints("ctx_len", ctx_len, dev, B), _ints("n_new", n_new, dev, B),
            _ints("free_pages", free_pages, dev) or count,  # (an empty list has no address, and none is read)
            count, M, _ints("page_table", page_table, dev))
    if out is None:
        buf = _new(3 * M + 3 * B + 2, torch.int32, dev, stream)
        cu, lens, adm, pos, row, slot, left = torch.unsafe_split_with_sizes(buf, (B + 1, B, B, M, M, M, 1))
        out = BatchPlan(cu, lens, adm, pos, row, slot, left)
        at = buf.data_ptr()
        lists = 3 * B + 1
        ptrs = [at + 4 * k for k in (0, B + 1, 2 * B + 1, lists, lists + M, lists + 2 * M, lists + 3 * M)]
    else:
        ptrs = [_ints(n, t, dev, k) for n, t, k in zip(BatchPlan._fields, out, (B + 1, B, B, M, M, M, 1))]
    _call("mg_batch_plan", dev, stream, load().mg_batch_plan, B, maxp, *args, *ptrs)
    return out


def _kv8(codes, scales):
    """The MgKv8Cache of a layer's codes [n_pages, Hkv, 2, 16 hd] and scales [n_pages, Hkv, 2]."""
    shape = codes.shape
    if codes.dtype is not torch.uint8 or len(shape) != 4 or shape[2] != 2 or shape[3] % 16 or not codes.is_contiguous():
        _refuse("codes", codes, "contiguous uint8 [n_pages, Hkv, 2, 16 hd]")
    if scales.dtype is not torch.uint8 or scales.shape != shape[:3] or not scales.is_contiguous() or \
            scales.device != codes.device:
        _refuse("scales", scales, f"contiguous uint8 [n_pages, Hkv, 2] for codes {tuple(shape)} on {codes.device}")
    return MgKv8Cache(codes.data_ptr(), scales.data_ptr(), shape[0], shape[1], shape[3] // 16)


def kv8_empty(n_pages, n_kv_heads, head_dim, device="cuda"):
    """An empty 8-bit cache of one layer: (codes, scales)."""
    if load().mg_kv8_code_bytes(n_pages, n_kv_heads, head_dim) == 0:
        raise MgError("mg_kv8_code_bytes", -2)
    return (torch.zeros((n_pages, n_kv_heads, 2, 16 * head_dim), dtype=torch.uint8, device=device),
            torch.zeros((n_pages, n_kv_heads, 2), dtype=torch.uint8, device=device))


def _rows16(name, t, n, heads, hd, device):
    """(address, stride) of bf16 rows [n, heads, hd] (or their bits as int16), each row contiguous."""
    if t.dtype not in _BF16 or t.device != device or t.shape != (n, heads, hd):
        _refuse(name, t, f"bf16 [{n}, {heads}, {hd}] on {device}")
    st = t.stride()
    if n and (st[2] != 1 or (heads > 1 and st[1] != hd)):
        _refuse(name, t, "rows [heads, head_dim] without gaps")
    return t.data_ptr(), (st[0] if n > 1 else heads * hd)


def kv8_append(codes, scales, k, v, slots, stream=None):
    """mg_kv8_append: K (after RoPE) and V rows [n, Hkv, hd] quantised into the cache at slots [n]."""
    c = _kv8(codes, scales)
    dev, n = codes.device, slots.numel()
    kp, ks = _rows16("k", k, n, c.n_kv_heads, c.head_dim, dev)
    vp, vs = _rows16("v", v, n, c.n_kv_heads, c.head_dim, dev)
    _call("mg_kv8_append", dev, stream, load().mg_kv8_append, C.byref(c), n, kp, ks, vp, vs, _ints("slots", slots, dev))


def kv8_read(codes, scales, slots, k_out=None, v_out=None, stream=None):
    """mg_kv8_read: the values of slots [n] as bf16 rows (k, v), each [n, Hkv, hd].  Rows of slots
    outside the cache are not written: in a new tensor they hold anything."""
    c = _kv8(codes, scales)
    dev, shape = codes.device, (slots.numel(), c.n_kv_heads, c.head_dim)
    n, heads, hd = shape
    if k_out is None:
        k_out = _new(shape, torch.bfloat16, dev, stream)
        kp, ks = k_out.data_ptr(), heads * hd
    else:
        kp, ks = _rows16("k_out", k_out, n, heads, hd, dev)
    if v_out is None:
        v_out = _new(shape, torch.bfloat16, dev, stream)
        vp, vs = v_out.data_ptr(), heads * hd
    else:
        vp, vs = _rows16("v_out", v_out, n, heads, hd, dev)
    _call("mg_kv8_read", dev, stream, load().mg_kv8_read, C.byref(c), n, _ints("slots", slots, dev), kp, ks, vp, vs)
    return k_out, v_out


def _attn_args(c, q, page_table, lens, cu_new, max_new, max_len, scale, window, softcap, out, dev):
    """The MgKv8AttnArgs of a call; out None: not known yet."""
    if q.dim() != 3 or q.shape[2] != c.head_dim:
        _refuse("q", q, f"[T, Hq, {c.head_dim}]")
    if page_table.dim() != 2:
        _refuse("page_table", page_table, "[B, max_pages]")
    T, Hq, hd = q.shape
    B, maxp = page_table.shape
    if max_new is None:  # without token offsets every row has one
        max_new = 1 if cu_new is None else max(T, 1)
    # (ctypes takes what passes 32 bits without a word)
    if not (-_I32 <= max_new < _I32 and -_I32 <= max_len < _I32 and -_I32 <= window < _I32):
        for name, n in (("max_new", max_new), ("max_len", max_len), ("window", window)):
            if not -_I32 <= n < _I32:
                _refuse(name, n, "an int32")
    if scale and abs(scale) < 1e-30 or softcap and abs(softcap) < 1e-30:
        _refuse("scale, softcap", (scale, softcap), "0 or 1e-15 .. 1e15")
    qp, qs = _rows16("q", q, T, Hq, hd, dev)
    op, os_ = (None, Hq * hd) if out is None else _rows16("out", out, T, Hq, hd, dev)
    return MgKv8AttnArgs(B, T, Hq, max_new, max_len, maxp, window, 0.0 if scale is None else scale, softcap, qp, qs, op,
                         os_, _ints("page_table", page_table, dev), _ints("lens", lens, dev, B),
                         None if cu_new is None else _ints("cu_new", cu_new, dev, B + 1))


def kv8_attention_workspace_bytes(codes, scales, q, page_table, lens, cu_new=None, max_new=None, max_len=0, window=0):
    """mg_kv8_attention_workspace_bytes of the call with these arguments (no device work): for a program
    that keeps a workspace, as one that captures its step does."""
    c = _kv8(codes, scales)
    a = _attn_args(c, q, page_table, lens, cu_new, max_new, max_len, None, window, 0.0, q, codes.device)
    with torch.cuda.device(codes.device):
        return load().mg_kv8_attention_workspace_bytes(C.byref(c), C.byref(a))


def kv8_attention(codes, scales, q, page_table, lens, cu_new=None, max_new=None, max_len=0, scale=None, window=0,
                  softcap=0.0, out=None, workspace=None, stream=None):
    """mg_kv8_attention: q [T, Hq, hd] attends over the cache's positions of its rows -> out [T, Hq, hd]
    bf16.  Tokens behind the last row's are not written: in a new tensor they hold anything.
    max_new: at least the most tokens of any row; None: all of q's with cu_new, else one.  A program that knows
    a smaller number gives it: the launch, and with it the time and a probability's bits, follow it.
    workspace: a contiguous uint8 tensor of kv8_attention_workspace_bytes that no other call in flight
    uses, or None to take one per call."""
    c = _kv8(codes, scales)
    dev = codes.device
    a = _attn_args(c, q, page_table, lens, cu_new, max_new, max_len, scale, window, softcap, out, dev)
    if out is None:
        out = _new(q.shape, q.dtype, dev, stream)
        a.out = out.data_ptr()
    args = "mg_kv8_attention", dev, stream, load().mg_kv8_attention, C.byref(c), C.byref(a)
    if workspace is not None:
        if workspace.dtype is not torch.uint8 or workspace.device != dev or not workspace.is_contiguous():
            _refuse("workspace", workspace, f"contiguous uint8 on {dev}")
        _call(*args, workspace.data_ptr(), workspace.numel())
        return out
    try:  # short calls need none, and asking first would take a tenth of their time
        _call(*args, None, 0)
    except MgError as e:
        if e.status != MG_ERR_WORKSPACE:
            raise
        with torch.cuda.device(dev):
            n = load().mg_kv8_attention_workspace_bytes(*args[4:])
        workspace = _new(n, torch.uint8, dev, stream)
        _call(*args, workspace.data_ptr(), n)
    return out


# ---------------------------------------------------------------- op-level calls (tests)

def op_copy(src, dst):
    _check("mg_op_copy", load().mg_op_copy(src.numel() * src.element_size(), src.data_ptr(), dst.data_ptr(),
                                           _stream()))


def op_read_stream(src, sink):
    """mg_op_read_stream: read every byte of src once (the HBM read-rate reference)."""
    _check("mg_op_read_stream", load().mg_op_read_stream(src.numel() * src.element_size(), src.data_ptr(),
                                                         sink.data_ptr(), _stream()))


def read_stream_sink_words():
    return int(load().mg_op_read_stream_sink_words())


def op_probe_bf16(x):
    out = torch.empty(x.shape, dtype=torch.int16, device=x.device)
    _check("mg_op_probe_bf16", load().mg_op_probe_bf16(x.numel(), x.data_ptr(), out.data_ptr(), _stream()))
    return out


def op_probe_exp(x):
    out = torch.empty_like(x)
    _check("mg_op_probe_exp", load().mg_op_probe_exp(x.numel(), x.data_ptr(), out.data_ptr(), _stream()))
    return out


def op_probe_divsqrt(a, b):
    q, r = torch.empty_like(a), torch.empty_like(a)
    _check("mg_op_probe_divsqrt", load().mg_op_probe_divsqrt(a.numel(), a.data_ptr(), b.data_ptr(), q.data_ptr(),
                                                             r.data_ptr(), _stream()))
    return q, r


def op_probe_mfma_fma(a, b, c):
    d = torch.empty_like(c)
    _check("mg_op_probe_mfma_fma", load().mg_op_probe_mfma_fma(a.shape[0], a.data_ptr(), b.data_ptr(), c.data_ptr(),
                                                               d.data_ptr(), _stream()))
    return d


def op_probe_mfma4_fma(a, b, c):
    d = torch.empty_like(c)
    _check("mg_op_probe_mfma4_fma", load().mg_op_probe_mfma4_fma(a.shape[0], a.data_ptr(), b.data_ptr(), c.data_ptr(),
                                                                 d.data_ptr(), _stream()))
    return d


def op_linear(canon, X, W):
    n, K = X.shape
    N = W.shape[0]
    Y = torch.empty((n, N), dtype=torch.float32, device=X.device)
    lib = load()
    wsb = lib.mg_op_linear_workspace_bytes(n, N, K)
    ws = torch.empty(max(wsb, 1), dtype=torch.uint8, device=X.device)
    _check("mg_op_linear", lib.mg_op_linear(int(canon), n, N, K, X.data_ptr(), W.data_ptr(), None, Y.data_ptr(),
                                            ws.data_ptr(), wsb, _stream()))
    return Y


def fast_gemm_config(n, N, K, n_cu=256):
    """(split-K factor, waves per block) of the fast GEMM launch for n rows of an N x K
    projection on a device of n_cu compute units (host logic, no device call)."""
    S, w = C.c_int(0), C.c_int(0)
    _check("mg_op_fast_gemm_config", load().mg_op_fast_gemm_config(n, N, K, n_cu, C.byref(S), C.byref(w)))
    return S.value, w.value


def canon_gemv_config(n, N, K, swiglu=False, n_cu=256):
    """(kernel, rows per tile, 4-row quads, waves per feature group, ring depth) of the
    verifier's canonical GEMV for n rows of an N x K projection (kernel 2: the vector-fma
    kernel, the rest 0; 3: the matrix-core kernel) on a device of n_cu compute units (host
    logic, no device call)."""
    out = [C.c_int(0) for _ in range(5)]
    _check("mg_op_canon_gemv_config",
           load().mg_op_canon_gemv_config(n, N, K, int(bool(swiglu)), n_cu, *[C.byref(o) for o in out]))
    return tuple(o.value for o in out)


def op_rmsnorm(x, gamma, eps):
    n, d = x.shape
    y = torch.empty_like(x)
    _check("mg_op_rmsnorm", load().mg_op_rmsnorm(n, d, x.data_ptr(), gamma.data_ptr(), float(eps), y.data_ptr(),
                                                 _stream()))
    return y
