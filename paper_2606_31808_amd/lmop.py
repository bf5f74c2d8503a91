"""Python binding of liblmop (include/lmop.h): argument marshalling only.

Every computation runs in the library's HIP kernels; this module converts
numpy / torch arguments to the C structs and back.  The functions keep the C
names (lmop_create, lmop_load_weights, lmop_set_prefix, lmop_eval_rows, ...);
`Context` bundles them for convenience.  If the built library is missing,
importing the binding raises: there is no fallback.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
from typing import Optional, Sequence

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "_lib", "liblmop.so")

LMOP_OK, LMOP_ERR_INVALID_ARG, LMOP_ERR_STATE, LMOP_ERR_OOM, LMOP_ERR_DEVICE, \
    LMOP_ERR_UNSUPPORTED = 0, -1, -2, -3, -4, -5
LMOP_BOOL, LMOP_ENUM, LMOP_INT, LMOP_AUTOMATON = 0, 1, 2, 3
LMOP_W_INT4_G32, LMOP_W_FP8_E4M3, LMOP_W_FP8_BLOCK = 0, 1, 2
_WEIGHT_FORMATS = {"int4_g32": LMOP_W_INT4_G32, "fp8_e4m3": LMOP_W_FP8_E4M3,
                   "fp8_block": LMOP_W_FP8_BLOCK}
LMOP_NO_DEDUP = 1
LMOP_HEAD_RESTRICTED = 2

EXPORTED = (
    "lmop_create", "lmop_destroy", "lmop_last_error", "lmop_status_string", "lmop_load_weights",
    "lmop_set_prefix", "lmop_set_prefixes", "lmop_release_prefix", "lmop_prefix_length", "lmop_eval_rows",
    "lmop_dedup_rows", "lmop_set_profiling", "lmop_get_kernel_stats", "lmop_set_workspace",
    "lmop_get_memory", "lmop_eval_rows_noalloc", "lmop_plan_rows", "lmop_quantize", "lmop_matmul",
    "lmop_qk_norm_rope", "lmop_load_qk_norms",
)
LMOP_F16, LMOP_BF16, LMOP_F32 = 0, 1, 2
LMOP_FP8_GROUP = 128
LMOP_V_ROWS, LMOP_V_COLUMNS = 0, 1
# size of the static device array lmop_eval_rows_noalloc carves its scratch from
LMOP_NOALLOC_SCRATCH_BYTES = 256 << 20


class lmop_config(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("d_model", C.c_int32), ("n_heads", C.c_int32),
                ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("d_ff", C.c_int32),
                ("vocab", C.c_int32), ("group_size", C.c_int32), ("rms_eps", C.c_float),
                ("rope_theta", C.c_float), ("max_seq", C.c_int32)]


class lmop_qmat(C.Structure):
    _fields_ = [("qweight", C.c_void_p), ("scales", C.c_void_p), ("n", C.c_int32),
                ("k", C.c_int32)]


class lmop_layer(C.Structure):
    _fields_ = [("attn_norm", C.c_void_p), ("mlp_norm", C.c_void_p), ("wq", lmop_qmat),
                ("wk", lmop_qmat), ("wv", lmop_qmat), ("wo", lmop_qmat), ("w_gate", lmop_qmat),
                ("w_up", lmop_qmat), ("w_down", lmop_qmat)]


class lmop_weights(C.Structure):
    _fields_ = [("tok_embedding", C.c_void_p), ("lm_head", C.c_void_p),
                ("final_norm", C.c_void_p), ("layers", C.POINTER(lmop_layer)),
                ("n_layers", C.c_int32), ("on_device", C.c_int32), ("format", C.c_int32)]


class lmop_automaton(C.Structure):
    _fields_ = [("n_states", C.c_int32), ("edge_offset", C.POINTER(C.c_int32)),
                ("edge_token", C.POINTER(C.c_int32)), ("edge_next", C.POINTER(C.c_int32)),
                ("accepting", C.POINTER(C.c_uint8))]


class lmop_type(C.Structure):
    _fields_ = [("kind", C.c_int32), ("tokens", C.POINTER(C.c_int32)), ("n_tokens", C.c_int32),
                ("eos_token", C.c_int32), ("max_tokens", C.c_int32),
                ("automaton", C.POINTER(lmop_automaton))]


class lmop_result(C.Structure):
    _fields_ = [("value", C.c_int64), ("logprob", C.c_float), ("logprob_full", C.c_float),
                ("n_tokens", C.c_int32), ("tokens", C.c_int32 * 8)]


class lmop_eval_opts(C.Structure):
    _fields_ = [("flags", C.c_uint32), ("max_batch_tokens", C.c_int32),
                ("debug_logits", C.POINTER(C.c_float)), ("limit", C.c_int32),
                ("limit_value", C.c_int64), ("row_mask", C.POINTER(C.c_uint8))]


class lmop_memory_stats(C.Structure):
    _fields_ = [("device_bytes", C.c_uint64), ("device_peak", C.c_uint64),
                ("workspace_bytes", C.c_uint64), ("workspace_peak", C.c_uint64)]


class lmop_eval_plan(C.Structure):
    _fields_ = [("unique_rows", C.c_int32), ("batches", C.c_int32), ("batch_tokens", C.c_int32),
                ("max_batch_tokens", C.c_int32), ("decode_groups", C.c_int32),
                ("pad_", C.c_int32), ("scratch_bytes", C.c_uint64), ("own_kv_bytes", C.c_uint64),
                ("min_workspace_bytes", C.c_uint64)]


class lmop_kernel_stat(C.Structure):
    _fields_ = [("name", C.c_char * 48), ("launches", C.c_int64), ("timed_launches", C.c_int64),
                ("total_ms", C.c_double), ("flops", C.c_double), ("bytes", C.c_double)]


class lmop_quantize_args(C.Structure):
    _fields_ = [("x", C.c_void_p), ("gate", C.c_void_p), ("q", C.c_void_p), ("scale", C.c_void_p),
                ("ldx", C.c_int64), ("ldg", C.c_int64), ("ldq", C.c_int64), ("lds", C.c_int64),
                ("rows", C.c_int32), ("cols", C.c_int32), ("dtype", C.c_int32)]


class lmop_matmul_args(C.Structure):
    _fields_ = [("a", C.c_void_p), ("a_scale", C.c_void_p), ("b", C.c_void_p),
                ("b_scale", C.c_void_p), ("add", C.c_void_p), ("c", C.c_void_p),
                ("lda", C.c_int64), ("ldb", C.c_int64), ("ldas", C.c_int64), ("ldbs", C.c_int64),
                ("ldadd", C.c_int64), ("ldc", C.c_int64), ("m", C.c_int32), ("n", C.c_int32),
                ("k", C.c_int32), ("dtype", C.c_int32), ("fast", C.c_int32)]


class lmop_qk_norm_rope_args(C.Structure):
    _fields_ = [("q", C.c_void_p), ("k", C.c_void_p), ("v", C.c_void_p), ("q_gain", C.c_void_p),
                ("k_gain", C.c_void_p), ("pos", C.c_void_p), ("slot", C.c_void_p),
                ("q_out", C.c_void_p), ("k_out", C.c_void_p), ("v_out", C.c_void_p),
                ("ldq", C.c_int64), ("ldk", C.c_int64), ("ldv", C.c_int64), ("ldqo", C.c_int64),
                ("ldko", C.c_int64), ("ldvo", C.c_int64), ("n_tokens", C.c_int32),
                ("n_slots", C.c_int32), ("v_layout", C.c_int32), ("dtype", C.c_int32)]


RESULT_DTYPE = np.dtype([("value", "<i8"), ("logprob", "<f4"), ("logprob_full", "<f4"),
                         ("n_tokens", "<i4"), ("tokens", "<i4", (8,)), ("_pad", "<i4")])
assert C.sizeof(lmop_result) == RESULT_DTYPE.itemsize


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built; run `python -m paper_2606_31808_amd.build`")
    # torch (imported above) ships its own HIP runtime under the same soname.
    # Loading it first makes the library bind to that one runtime: the streams
    # and device pointers torch hands over are only valid there, and a second
    # runtime loaded beside it finds no devices.
    lib = C.CDLL(LIB_PATH)
    vp, i32, st = C.c_void_p, C.c_int32, C.c_int
    sig = {
        "lmop_create": (st, [C.POINTER(lmop_config), i32, vp, C.POINTER(vp)]),
        "lmop_destroy": (None, [vp]),
        "lmop_last_error": (C.c_char_p, [vp]),
        "lmop_status_string": (C.c_char_p, [st]),
        "lmop_load_weights": (st, [vp, C.POINTER(lmop_weights)]),
        "lmop_set_prefix": (st, [vp, vp, C.POINTER(C.c_int32), i32, C.POINTER(vp)]),
        "lmop_set_prefixes": (st, [vp, vp, C.POINTER(C.c_int32), C.POINTER(C.c_int64), i32,
                                   C.POINTER(vp)]),
        "lmop_release_prefix": (st, [vp, vp]),
        "lmop_prefix_length": (i32, [vp]),
        "lmop_eval_rows": (st, [vp, vp, C.POINTER(vp), C.POINTER(C.c_int32),
                                C.POINTER(C.c_int64), i32, C.POINTER(lmop_type), vp,
                                C.POINTER(lmop_eval_opts)]),
        "lmop_eval_rows_noalloc": (st, [vp, vp, C.POINTER(vp), C.POINTER(C.c_int32),
                                        C.POINTER(C.c_int64), i32, C.POINTER(lmop_type), vp,
                                        C.POINTER(lmop_eval_opts)]),
        "lmop_plan_rows": (st, [vp, vp, C.POINTER(vp), C.POINTER(C.c_int32),
                                C.POINTER(C.c_int64), i32, C.POINTER(lmop_type),
                                C.POINTER(lmop_eval_opts), C.POINTER(lmop_eval_plan)]),
        "lmop_set_workspace": (st, [vp, vp, C.c_size_t]),
        "lmop_get_memory": (st, [vp, C.POINTER(lmop_memory_stats)]),
        "lmop_dedup_rows": (st, [C.POINTER(C.c_int32), C.POINTER(C.c_int64), i32,
                                 C.POINTER(C.c_int64), C.POINTER(C.c_int32),
                                 C.POINTER(C.c_int32)]),
        "lmop_set_profiling": (st, [vp, i32]),
        "lmop_get_kernel_stats": (st, [vp, C.POINTER(lmop_kernel_stat), i32,
                                       C.POINTER(C.c_int32)]),
        "lmop_load_qk_norms": (st, [vp, vp, vp, i32]),
        "lmop_quantize": (st, [vp, vp]),
        "lmop_matmul": (st, [vp, vp]),
        "lmop_qk_norm_rope": (st, [vp, vp]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    return lib


_lib = _load()


class LmopError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{_lib.lmop_status_string(status).decode()} ({status}): {message}")
        self.status = status


def _check(status: int, ctx) -> None:
    if status != LMOP_OK:
        msg = _lib.lmop_last_error(ctx)
        raise LmopError(status, msg.decode() if msg else "")


def _i32(a) -> np.ndarray:
    return np.ascontiguousarray(np.asarray(a, dtype=np.int32))


def _i64(a) -> np.ndarray:
    return np.ascontiguousarray(np.asarray(a, dtype=np.int64))


def _ptr(a: np.ndarray, ct):
    return a.ctypes.data_as(C.POINTER(ct))


# ---------------------------------------------------------------- C-named calls
class _Ctx(C.c_void_p):
    """A ctx, and the shape of its query and key norms (n_layers, head_dim)."""
    norms = None


def lmop_create(cfg: lmop_config, device: int = 0, stream: Optional[int] = None):
    out = _Ctx()
    st = _lib.lmop_create(C.byref(cfg), device, C.c_void_p(stream or 0), C.byref(out))
    _check(st, None)
    out.norms = cfg.n_layers, cfg.head_dim
    return out


def lmop_destroy(ctx) -> None:
    _lib.lmop_destroy(ctx)


def _tensor_ptr(t, keep):
    """Device or host address of a contiguous torch tensor / numpy array."""
    if hasattr(t, "data_ptr"):
        t = t.contiguous()
        keep.append(t)
        return t.data_ptr(), t.device.type != "cpu"
    a = np.ascontiguousarray(t)
    keep.append(a)
    return a.ctypes.data, False


def _qk_norms(weights, ctx):
    """The layers' query and key norms, [n_layers, head_dim] each; None without."""
    norms = [(getattr(l, "q_norm", None), getattr(l, "k_norm", None)) for l in weights.layers]
    if all(n is None for pair in norms for n in pair):
        return None
    if any(n is None for pair in norms for n in pair):
        raise ValueError("query and key norms: in every layer, or in none")
    norms = [[torch.as_tensor(n).detach().cpu().float() for n in pair] for pair in norms]
    for n in (n for pair in norms for n in pair):
        if tuple(n.shape) != (ctx.norms[1],):
            raise ValueError(f"a query or key norm of shape {tuple(n.shape)}, expected ({ctx.norms[1]},)")
    return [torch.stack([pair[i] for pair in norms]) for i in (0, 1)]


def lmop_load_weights(ctx, weights) -> None:
    """weights: object with tok_embedding, lm_head (fp16 [V][d]), final_norm, layers[...]
    (attn_norm, mlp_norm, wq .. w_down each with qweight/scales/n/k and a format name
    `fmt`, "int4_g32" (default), "fp8_e4m3" or "fp8_block"), all on one device.  Layers
    with q_norm and k_norm (fp32 [head_dim]) have these loaded too."""
    norms = _qk_norms(weights, ctx)  # refused before anything is loaded
    keep = []
    where = set()

    def p(t):
        a, dev = _tensor_ptr(t, keep)
        where.add(dev)
        return a

    def qm(m):
        return lmop_qmat(p(m.qweight), p(m.scales), int(m.n), int(m.k))

    L = len(weights.layers)
    arr = (lmop_layer * max(L, 1))()
    for i, l in enumerate(weights.layers):
        arr[i] = lmop_layer(p(l.attn_norm), p(l.mlp_norm), qm(l.wq), qm(l.wk), qm(l.wv), qm(l.wo),
                            qm(l.w_gate), qm(l.w_up), qm(l.w_down))
    fmts = {getattr(getattr(l, nm), "fmt", "int4_g32") for l in weights.layers
            for nm in ("wq", "wk", "wv", "wo", "w_gate", "w_up", "w_down")}
    if len(fmts) > 1:
        raise ValueError("all linear maps must have one weight format")
    fmt = _WEIGHT_FORMATS[fmts.pop() if fmts else "int4_g32"]
    w = lmop_weights(p(weights.tok_embedding), p(weights.lm_head), p(weights.final_norm),
                     C.cast(arr, C.POINTER(lmop_layer)), L, 0, fmt)
    if len(where) != 1:
        raise ValueError("weights must all be on the host or all on the device")
    w.on_device = 1 if where.pop() else 0
    _check(_lib.lmop_load_weights(ctx, C.byref(w)), ctx)
    if norms is not None:
        lmop_load_qk_norms(ctx, *norms)


def lmop_load_qk_norms(ctx, q_gain=None, k_gain=None) -> None:
    """Query and key norms, [n_layers, head_dim] (both None: no norms); ctx is one of
    lmop_create."""
    # few values, from the host: a copy or conversion on torch's current stream is
    # not ordered with the ctx's
    keep = [None if g is None else torch.as_tensor(g).detach().cpu().float().contiguous()
            for g in (q_gain, k_gain)]
    for g in keep:
        if g is not None and tuple(g.shape) != ctx.norms:
            raise ValueError(f"norms of shape {tuple(g.shape)}, expected {ctx.norms}")
    _check(_lib.lmop_load_qk_norms(ctx, *(None if g is None else g.data_ptr() for g in keep), 0),
           ctx)


def lmop_set_prefix(ctx, tokens, parent=None):
    t = _i32(tokens)
    out = C.c_void_p()
    _check(_lib.lmop_set_prefix(ctx, parent, _ptr(t, C.c_int32), len(t), C.byref(out)), ctx)
    return out


def lmop_set_prefixes(ctx, token_lists, parent=None):
    lists = [_i32(t) for t in token_lists]
    n = len(lists)
    offs = np.zeros(n + 1, dtype=np.int64)
    offs[1:] = np.cumsum([len(t) for t in lists])
    t = np.concatenate(lists) if n else np.zeros(0, dtype=np.int32)
    t = np.ascontiguousarray(t, dtype=np.int32)
    out = (C.c_void_p * max(n, 1))()
    _check(_lib.lmop_set_prefixes(ctx, parent, _ptr(t, C.c_int32), _ptr(offs, C.c_int64), n,
                                  out), ctx)
    return [C.c_void_p(out[i]) for i in range(n)]


def lmop_release_prefix(ctx, prefix) -> None:
    _check(_lib.lmop_release_prefix(ctx, prefix), ctx)


def lmop_prefix_length(prefix) -> int:
    return int(_lib.lmop_prefix_length(prefix))


def lmop_eval_rows(ctx, tokens, offsets, kind: int, allowed: Sequence[int], eos: int = -1,
                   max_tokens: int = 1, prefix=None, row_prefix=None, flags: int = 0,
                   max_batch_tokens: int = 0, debug_logits: bool = False, vocab: int = 0,
                   limit: int = 0, limit_value: int = 1, row_mask=None, no_alloc: bool = False):
    """Returns a structured numpy array of lmop_result (value, logprob, logprob_full,
    n_tokens, tokens) and, with debug_logits, fp32 logits [n_rows][steps][vocab].
    For LMOP_AUTOMATON, `allowed` is an object with n_states, edge_offset,
    edge_token, edge_next and accepting arrays.  no_alloc calls
    lmop_eval_rows_noalloc (scratch in the library's static array) instead."""
    toks, offs, n, ty, opts, rp, keep = _call_args(tokens, offsets, kind, allowed, eos, max_tokens,
                                                   row_prefix, flags, max_batch_tokens, limit,
                                                   limit_value, row_mask)
    out = np.zeros(max(n, 0), dtype=RESULT_DTYPE)
    steps = max_tokens if kind in (LMOP_INT, LMOP_AUTOMATON) else 1
    dbg = None
    if debug_logits:
        if vocab <= 0:
            raise ValueError("debug_logits needs vocab")
        dbg = np.empty((n, steps, vocab), dtype=np.float32)
        opts.debug_logits = _ptr(dbg, C.c_float)
    fn = _lib.lmop_eval_rows_noalloc if no_alloc else _lib.lmop_eval_rows
    _check(fn(ctx, prefix, rp, _ptr(toks, C.c_int32), _ptr(offs, C.c_int64), n, C.byref(ty),
              out.ctypes.data, C.byref(opts)), ctx)
    del keep
    return out, dbg


def lmop_plan_rows(ctx, tokens, offsets, kind: int, allowed: Sequence[int], eos: int = -1,
                   max_tokens: int = 1, prefix=None, row_prefix=None, flags: int = 0,
                   max_batch_tokens: int = 0, limit: int = 0, limit_value: int = 1,
                   row_mask=None, debug_logits: bool = False) -> dict:
    """lmop_plan_rows: the plan lmop_eval_rows would use for these arguments
    (a dict of lmop_eval_plan's fields); runs nothing on the device.
    debug_logits plans the logit dump's scratch (the library writes nothing)."""
    toks, offs, n, ty, opts, rp, keep = _call_args(tokens, offsets, kind, allowed, eos, max_tokens,
                                                   row_prefix, flags, max_batch_tokens, limit,
                                                   limit_value, row_mask)
    if debug_logits:
        dummy = np.zeros(1, dtype=np.float32)
        keep.append(dummy)
        opts.debug_logits = _ptr(dummy, C.c_float)
    pl = lmop_eval_plan()
    _check(_lib.lmop_plan_rows(ctx, prefix, rp, _ptr(toks, C.c_int32), _ptr(offs, C.c_int64), n,
                               C.byref(ty), C.byref(opts), C.byref(pl)), ctx)
    del keep
    return {k: int(getattr(pl, k)) for k, _ in lmop_eval_plan._fields_ if k != "pad_"}


def _call_args(tokens, offsets, kind, allowed, eos, max_tokens, row_prefix, flags,
               max_batch_tokens, limit, limit_value, row_mask):
    """The marshalled arguments shared by lmop_eval_rows and lmop_plan_rows:
    token and offset arrays, row count, lmop_type, lmop_eval_opts, the row
    prefix array, and the arrays those structs point into (kept alive by the
    caller until the call returns)."""
    toks = _i32(tokens)
    offs = _i64(offsets)
    n = len(offs) - 1
    keep = []
    if kind == LMOP_AUTOMATON:
        eo, et, en = _i32(allowed.edge_offset), _i32(allowed.edge_token), _i32(allowed.edge_next)
        ac = np.ascontiguousarray(np.asarray(allowed.accepting, dtype=np.uint8))
        keep = [eo, et, en, ac]
        aut = lmop_automaton(int(allowed.n_states), _ptr(eo, C.c_int32), _ptr(et, C.c_int32),
                             _ptr(en, C.c_int32), _ptr(ac, C.c_uint8))
        ty = lmop_type(kind, None, 0, int(eos), int(max_tokens), C.pointer(aut))
    else:
        al = _i32(allowed)
        keep = [al]
        ty = lmop_type(kind, _ptr(al, C.c_int32), len(al), int(eos), int(max_tokens), None)
    keep.append(ty)
    opts = lmop_eval_opts(flags, max_batch_tokens, None, int(limit), int(limit_value), None)
    if row_mask is not None:
        mk = np.ascontiguousarray(np.asarray(row_mask, dtype=bool).astype(np.uint8))
        if len(mk) != n:
            raise ValueError("row_mask needs one entry per row")
        keep.append(mk)
        opts.row_mask = _ptr(mk, C.c_uint8)
    rp = None
    if row_prefix is not None:
        rp = (C.c_void_p * max(n, 1))(*[r.value if isinstance(r, C.c_void_p) else r
                                        for r in row_prefix])
    return toks, offs, n, ty, opts, rp, keep


def lmop_dedup_rows(tokens, offsets, keys=None):
    toks = _i32(tokens)
    offs = _i64(offsets)
    n = len(offs) - 1
    rep = np.zeros(max(n, 0), dtype=np.int32)
    nu = C.c_int32()
    kp = None
    if keys is not None:
        k = _i64(keys)
        kp = _ptr(k, C.c_int64)
    st = _lib.lmop_dedup_rows(_ptr(toks, C.c_int32), _ptr(offs, C.c_int64), n, kp,
                              _ptr(rep, C.c_int32), C.byref(nu))
    if st != LMOP_OK:
        raise LmopError(st, "invalid CSR arguments")
    return rep, int(nu.value)


def lmop_eval_rows_noalloc(ctx, tokens, offsets, kind: int, allowed, **kw):
    """lmop_eval_rows_noalloc: lmop_eval_rows with no device allocation."""
    return lmop_eval_rows(ctx, tokens, offsets, kind, allowed, no_alloc=True, **kw)


def lmop_set_workspace(ctx, ptr: int, nbytes: int) -> None:
    """Scratch carved from the caller's device memory [ptr, ptr + nbytes)
    (e.g. a torch tensor's data_ptr()); (0, 0) returns to library scratch."""
    _check(_lib.lmop_set_workspace(ctx, C.c_void_p(ptr or None), C.c_size_t(nbytes)), ctx)


def lmop_get_memory(ctx) -> dict:
    m = lmop_memory_stats()
    _check(_lib.lmop_get_memory(ctx, C.byref(m)), ctx)
    return {k: int(getattr(m, k)) for k, _ in lmop_memory_stats._fields_}


def lmop_set_profiling(ctx, period) -> None:
    """period: False/0 off, True/1 time every launch, N time every N-th launch
    of each kernel."""
    _check(_lib.lmop_set_profiling(ctx, int(period)), ctx)


def lmop_get_kernel_stats(ctx):
    n = C.c_int32()
    _check(_lib.lmop_get_kernel_stats(ctx, None, 0, C.byref(n)), ctx)
    arr = (lmop_kernel_stat * max(n.value, 1))()
    _check(_lib.lmop_get_kernel_stats(ctx, arr, n.value, C.byref(n)), ctx)
    return {arr[i].name.decode(): dict(launches=arr[i].launches, timed=arr[i].timed_launches,
                                       ms=arr[i].total_ms, flops=arr[i].flops, bytes=arr[i].bytes)
            for i in range(n.value)}


# ---------------------------------------------------------------- operators
# Tensors here are torch tensors: inputs of rows with adjacent elements at any
# row stride, outputs given or allocated by the Context methods below.  A call
# on one token takes the GPU 2 to 4 us, so these functions are kept short: the
# argument structs are packed with `struct`, which takes a quarter of the time
# of filling a ctypes structure (whose fields are checked against the formats
# below when the module loads).
_DTYPES = {torch.float16: LMOP_F16, torch.bfloat16: LMOP_BF16, torch.float32: LMOP_F32}
_CODES = {torch.float8_e4m3fn: 0, torch.uint8: 0}
_F32 = {torch.float32: LMOP_F32}
_PACK = {}
for _name, _fmt, _struct in (("quantize", "4P4q3i4x", lmop_quantize_args),
                             ("matmul", "6P6q5i4x", lmop_matmul_args),
                             ("qk_norm_rope", "10P6q4i", lmop_qk_norm_rope_args)):
    assert struct.calcsize(_fmt) == C.sizeof(_struct)
    _PACK[_name] = struct.Struct(_fmt).pack


def _bad(t, what: str, rows: int, cols: int, dtypes, dev: int):
    """Raises what is wrong with a tensor."""
    if t.get_device() != dev:
        raise ValueError(f"{what} is on {t.device}, the ctx on device {dev}")
    if tuple(t.shape) != (rows, cols):
        raise ValueError(f"{what}: shape {tuple(t.shape)}, expected ({rows}, {cols})")
    if t.dtype not in dtypes:
        raise ValueError(f"{what}: dtype {t.dtype}")
    raise ValueError(f"{what}: the elements of a row are not adjacent")


def _ld(t, what: str, rows: int, cols: int, dtypes, dev: int, least: int = 0) -> int:
    """The row stride of a [rows][cols] tensor; a single row's does not matter and
    counts as its length, or `least`."""
    if t.get_device() != dev or t.shape != (rows, cols) or t.dtype not in dtypes:
        _bad(t, what, rows, cols, dtypes, dev)
    ld, inner = t.stride()
    if inner != 1 and cols > 1:
        _bad(t, what, rows, cols, dtypes, dev)
    return ld if rows > 1 else max(least, cols)


def _ld_codes(t, what: str, rows: int, cols: int, dev: int) -> int:
    """_ld of FP8 codes, whose rows are read to the next multiple of 16 bytes."""
    most = (cols + 15) & -16
    ld = _ld(t, what, rows, cols, _CODES, dev, most)
    if most != cols and rows > 0 and (t.storage_offset() + (rows - 1) * ld + most >
                                      t.untyped_storage().nbytes()):
        raise ValueError(f"{what}: the last row's storage ends before {most} bytes")
    return ld


def _current_stream(dev: int) -> int:
    return torch.cuda.current_stream(dev).cuda_stream


# the same without an object around it, where torch offers it: 0.07 us, not 1.1
_current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", _current_stream)


def _vec(t, what: str, n: int, dtype, dev: int) -> int:
    if t is None:
        return 0
    if (t.get_device() != dev or t.shape != (n,) or t.dtype != dtype or
            (n > 1 and t.stride(0) != 1)):
        raise ValueError(f"{what}: expected {n} adjacent elements of {dtype} on device {dev}")
    return t.data_ptr()


def lmop_quantize(ctx, x, q, scale, gate=None) -> None:
    """E4M3 codes q and scales of x, or of silu(gate) * x."""
    rows, cols = x.shape
    dt, dev = x.dtype, x.get_device()
    ldx = _ld(x, "x", rows, cols, _DTYPES, dev)
    pg = ldg = 0
    if gate is not None:
        ldg = _ld(gate, "gate", rows, cols, (dt,), dev)
        pg = gate.data_ptr()
    st = _lib.lmop_quantize(ctx, _PACK["quantize"](
        x.data_ptr(), pg, q.data_ptr(), scale.data_ptr(), ldx, ldg,
        _ld_codes(q, "q", rows, cols, dev), _ld(scale, "scale", rows, (cols + 127) >> 7, _F32, dev),
        rows, cols, _DTYPES[dt]))
    if st:
        _check(st, ctx)


def lmop_matmul(ctx, a, a_scale, b, b_scale, c, add=None, fast: bool = False) -> None:
    """c = a b^T (+ add) of E4M3 codes: scales per row and 128 features of a, per
    128 x 128 block of b.  fast: float32 results on the 8-bit instruction."""
    (m, k), n, dev = a.shape, b.shape[0], a.get_device()
    groups = (k + 127) >> 7
    pd = ldadd = 0
    if add is not None:
        ldadd = _ld(add, "add", m, n, _F32, dev)
        pd = add.data_ptr()
    ldc = _ld(c, "c", m, n, _DTYPES, dev)
    st = _lib.lmop_matmul(ctx, _PACK["matmul"](
        a.data_ptr(), a_scale.data_ptr(), b.data_ptr(), b_scale.data_ptr(), pd, c.data_ptr(),
        _ld_codes(a, "a", m, k, dev), _ld_codes(b, "b", n, k, dev),
        _ld(a_scale, "a_scale", m, groups, _F32, dev),
        _ld(b_scale, "b_scale", (n + 127) >> 7, groups, _F32, dev), ldadd, ldc, m, n, k,
        _DTYPES[c.dtype], fast))
    if st:
        _check(st, ctx)


def lmop_qk_norm_rope(ctx, heads, n_tokens, q=None, k=None, v=None, pos=None, q_gain=None,
                      k_gain=None, slot=None, q_out=None, k_out=None, v_out=None,
                      v_columns: bool = False) -> None:
    """Per-head RMSNorm, RoPE and cache write of n_tokens tokens; heads is the
    ctx's (n_heads, n_kv_heads, head_dim)."""
    first = q if q is not None else k if k is not None else v
    if first is None:
        raise ValueError("q, k and v are all None")
    nq, nkv, hd = heads
    nq *= hd
    nkv *= hd
    dev, dt = first.get_device(), first.dtype
    if dt not in _DTYPES or dt is torch.float32:
        raise ValueError(f"dtype {dt}: float16 or bfloat16")
    own = (dt,)
    n_slots = 0
    if v is not None:
        n_slots = v_out.shape[1 if v_columns else 0]
    if k is not None:
        if v is not None and n_slots != k_out.shape[0]:
            raise ValueError(f"k_out has {k_out.shape[0]} slots, v_out {n_slots}")
        n_slots = k_out.shape[0]
    pq = pk = pv = pqo = pko = pvo = ldq = ldk = ldv = ldqo = ldko = ldvo = 0
    if q is not None:
        ldq, ldqo = _ld(q, "q", n_tokens, nq, own, dev), _ld(q_out, "q_out", n_tokens, nq, own, dev)
        pq, pqo = q.data_ptr(), q_out.data_ptr()
    if k is not None:
        ldk, ldko = _ld(k, "k", n_tokens, nkv, own, dev), _ld(k_out, "k_out", n_slots, nkv, own, dev)
        pk, pko = k.data_ptr(), k_out.data_ptr()
    if v is not None:
        ldv = _ld(v, "v", n_tokens, nkv, own, dev)
        ldvo = (_ld(v_out, "v_out", nkv, n_slots, own, dev) if v_columns
                else _ld(v_out, "v_out", n_slots, nkv, own, dev))
        pv, pvo = v.data_ptr(), v_out.data_ptr()
    st = _lib.lmop_qk_norm_rope(ctx, _PACK["qk_norm_rope"](
        pq, pk, pv, _vec(q_gain, "q_gain", hd, torch.float32, dev),
        _vec(k_gain, "k_gain", hd, torch.float32, dev), _vec(pos, "pos", n_tokens, torch.int32, dev),
        _vec(slot, "slot", n_tokens, torch.int32, dev), pqo, pko, pvo, ldq, ldk, ldv, ldqo, ldko,
        ldvo, n_tokens, n_slots, LMOP_V_COLUMNS if v_columns else LMOP_V_ROWS, _DTYPES[dt]))
    if st:
        _check(st, ctx)


# ---------------------------------------------------------------- convenience
def config_from_shape(shape, max_seq: int = 0) -> lmop_config:
    return lmop_config(shape.n_layers, shape.d_model, shape.n_heads, shape.n_kv_heads,
                       shape.head_dim, shape.d_ff, shape.vocab, shape.group_size,
                       shape.rms_eps, shape.rope_theta, max_seq)


# ctxs that nothing referred to any more while a stream was being captured, where
# freeing one would end the capture: freed with the next ctx made or closed
_dropped = []


def _free_dropped():
    while _dropped:
        lmop_destroy(_dropped.pop())


class Context:
    """One lmop ctx on a HIP device (device=-1: host-only, validation only).  It has to outlive
    the graphs that captured its operators."""

    def __init__(self, shape, device: int = 0, stream: Optional[int] = None, max_seq: int = 0,
                 n_layers: Optional[int] = None):
        cfg = config_from_shape(shape, max_seq)
        if n_layers is not None:
            cfg.n_layers = n_layers
        self.vocab = shape.vocab
        self.heads = (cfg.n_heads, cfg.n_kv_heads, cfg.head_dim)
        self.n_layers = cfg.n_layers
        # where the operators' tensors live (-1: the host), and the torch stream
        # they are ordered on
        self.device = max(int(device), -1)
        self.stream = int(stream or 0)
        _free_dropped()
        self.ctx = lmop_create(cfg, device, stream)

    def close(self):
        _free_dropped()
        if self.ctx:
            lmop_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            # a garbage collection may come in the middle of a capture
            if self.ctx and self.device >= 0 and torch.cuda.is_current_stream_capturing():
                _dropped.append(self.ctx)
                self.ctx = None
            else:
                self.close()
        except Exception:
            pass

    def load_weights(self, weights):
        lmop_load_weights(self.ctx, weights)

    def load_qk_norms(self, q_gain=None, k_gain=None):
        lmop_load_qk_norms(self.ctx, q_gain, k_gain)

    def set_prefix(self, tokens, parent=None):
        return lmop_set_prefix(self.ctx, tokens, parent)

    def set_prefixes(self, token_lists, parent=None):
        return lmop_set_prefixes(self.ctx, token_lists, parent)

    def release_prefix(self, p):
        lmop_release_prefix(self.ctx, p)

    def eval_rows(self, tokens, offsets, kind, allowed, eos=-1, max_tokens=1, prefix=None,
                  row_prefix=None, no_dedup=False, max_batch_tokens=0, debug_logits=False,
                  head_restricted=False, limit=0, limit_value=1, row_mask=None, no_alloc=False):
        flags = (LMOP_NO_DEDUP if no_dedup else 0) | (LMOP_HEAD_RESTRICTED if head_restricted else 0)
        return lmop_eval_rows(self.ctx, tokens, offsets, kind, allowed, eos, max_tokens, prefix,
                              row_prefix, flags, max_batch_tokens, debug_logits, self.vocab,
                              limit, limit_value, row_mask, no_alloc)

    def plan_rows(self, tokens, offsets, kind, allowed, eos=-1, max_tokens=1, prefix=None,
                  row_prefix=None, no_dedup=False, max_batch_tokens=0, head_restricted=False,
                  limit=0, limit_value=1, row_mask=None, debug_logits=False) -> dict:
        flags = (LMOP_NO_DEDUP if no_dedup else 0) | (LMOP_HEAD_RESTRICTED if head_restricted else 0)
        return lmop_plan_rows(self.ctx, tokens, offsets, kind, allowed, eos, max_tokens, prefix,
                              row_prefix, flags, max_batch_tokens, limit, limit_value, row_mask,
                              debug_logits)

    def set_workspace(self, ptr: int, nbytes: int):
        lmop_set_workspace(self.ctx, ptr, nbytes)

    def memory(self) -> dict:
        return lmop_get_memory(self.ctx)

    def set_profiling(self, period):
        lmop_set_profiling(self.ctx, period)

    def kernel_stats(self):
        return lmop_get_kernel_stats(self.ctx)

    # -- operators: they queue work on the ctx's stream (made without one: on the
    # null stream) and return
    def _here(self, t):
        """t has to be on the ctx's device, and torch's current stream has to be the one
        that the operators run on: the ctx's, or without one the null stream."""
        dev = self.device
        if t.get_device() != dev or (dev < 0 and not t.is_cpu):
            raise ValueError(f"a tensor is on {t.device}, the ctx on device {dev}")
        if dev >= 0 and _current_stream(dev) != self.stream:
            raise ValueError("torch's current stream is not the ctx's stream: make the Context "
                             "with stream=..., or call under torch.cuda.stream(...)")

    def quantize(self, x, gate=None, out=None):
        """E4M3 codes [rows, cols] (torch.float8_e4m3fn, rows a multiple of 16 bytes
        apart) and float32 scales [rows, ceil(cols / 128)] of x, or of
        silu(gate) * x.  out: (codes, scales) to write into."""
        self._here(x)
        if out is None:
            rows, cols = x.shape
            most = (cols + 15) & -16
            q = torch.empty((rows, most), dtype=torch.float8_e4m3fn, device=x.device)
            if most != cols:
                q = q[:, :cols]
            out = q, torch.empty((rows, (cols + 127) >> 7), dtype=torch.float32, device=x.device)
        lmop_quantize(self.ctx, x, out[0], out[1], gate)
        return out

    def matmul(self, a, a_scale, b, b_scale, dtype=torch.float16, add=None, out=None, fast=False):
        """a b^T (+ add) of E4M3 codes a [m, k], b [n, k] with block scales.  A float32
        result keeps every product whole, or (fast) has them cut as 16-bit ones do."""
        self._here(a)
        if out is None:
            out = torch.empty((a.shape[0], b.shape[0]), dtype=dtype, device=a.device)
        lmop_matmul(self.ctx, a, a_scale, b, b_scale, out, add, fast)
        return out

    def qk_norm_rope(self, q=None, k=None, v=None, *, pos, q_gain=None, k_gain=None, slot=None,
                     q_out=None, k_out=None, v_out=None, v_columns=False):
        """Normalises (where a gain is given) and rotates queries and keys, and writes
        keys and values by slot into k_out, v_out.  Returns the queries (q_out,
        or a new tensor; None without q)."""
        self._here(pos)
        if q is not None and q_out is None:
            q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        if (k is None) != (k_out is None) or (v is None) != (v_out is None):
            raise ValueError("k needs k_out, v needs v_out")
        lmop_qk_norm_rope(self.ctx, self.heads, pos.shape[0], q, k, v, pos, q_gain, k_gain, slot,
                          q_out, k_out, v_out, v_columns)
        return q_out
