"""What the operator calls refuse, checked on a host-only ctx: every argument
check runs there, and a call whose arguments are valid ends at UNSUPPORTED
(no device)."""
import ctypes as C
import dataclasses

import pytest
import torch

from paper_2606_31808_amd import lmop as L
from synth import SHAPES

F8 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def ctx():
    return L.Context(SHAPES["tiny"], device=-1)


def _status(fn, *a, **k):
    with pytest.raises(L.LmopError) as ei:
        fn(*a, **k)
    assert str(ei.value)
    return ei.value.status


def _args(struct, base, **change):
    a = struct()
    for f, v in {**base, **change}.items():
        setattr(a, f, v)
    return a


def _call(ctx, name, a):
    return getattr(L._lib, name)(ctx.ctx, C.byref(a) if a is not None else None)


# addresses that no call here reads: a host-only ctx checks them and stops
P = 1 << 20
QUANT = dict(x=P, q=P, scale=P, ldx=300, ldq=304, lds=3, rows=5, cols=300, dtype=L.LMOP_F16)
MM = dict(a=P, b=P, a_scale=P, b_scale=P, c=P, lda=304, ldb=304, ldas=3, ldbs=3, ldc=200, m=9,
          n=200, k=300, dtype=L.LMOP_F16)
QK = dict(q=P, k=P, v=P, pos=P, q_out=2 * P, k_out=2 * P, v_out=2 * P, ldq=256, ldk=256, ldv=256,
          ldqo=256, ldko=256, ldvo=256, n_tokens=7, n_slots=7, v_layout=L.LMOP_V_ROWS,
          dtype=L.LMOP_F16)
INV, UNS, OK = L.LMOP_ERR_INVALID_ARG, L.LMOP_ERR_UNSUPPORTED, L.LMOP_OK


@pytest.mark.parametrize("change,status", [
    ({}, UNS),
    (dict(rows=0), OK), (dict(cols=0), OK), (dict(rows=-1), INV), (dict(cols=-1), INV),
    (dict(dtype=3), INV), (dict(dtype=-1), INV),
    (dict(x=None), INV), (dict(q=None), INV), (dict(scale=None), INV),
    (dict(x=P + 1), INV), (dict(x=P + 2), UNS), (dict(x=P + 2, dtype=L.LMOP_F32), INV),
    (dict(q=P + 8), INV), (dict(scale=P + 2), INV),
    (dict(ldx=299), INV), (dict(ldx=0), INV), (dict(ldx=-300), INV),
    (dict(ldq=300), INV), (dict(ldq=288), INV), (dict(ldq=320), UNS), (dict(lds=2), INV),
    (dict(ldq=(1 << 23) + 16), UNS),
    (dict(rows=2 ** 31 - 1), UNS),
    (dict(gate=P, ldg=300), UNS), (dict(gate=P, ldg=10), INV), (dict(gate=P + 1, ldg=300), INV),
])
def test_quantize(ctx, change, status):
    assert _call(ctx, "lmop_quantize", _args(L.lmop_quantize_args, QUANT, **change)) == status


@pytest.mark.parametrize("change,status", [
    ({}, UNS),
    (dict(m=0), OK), (dict(n=0), OK), (dict(m=-1), INV), (dict(n=-1), INV), (dict(k=-1), INV),
    (dict(k=0, a=None, b=None, a_scale=None, b_scale=None), UNS),
    (dict(dtype=5), INV), (dict(fast=1), UNS), (dict(fast=2), INV), (dict(fast=-1), INV),
    (dict(a=None), INV), (dict(b=None), INV), (dict(a_scale=None), INV), (dict(b_scale=None), INV),
    (dict(c=None), INV),
    (dict(a=P + 8), INV), (dict(b=P + 1), INV), (dict(a_scale=P + 1), INV), (dict(c=P + 1), INV),
    (dict(lda=300), INV), (dict(ldb=288), INV), (dict(ldas=2), INV), (dict(ldbs=2), INV),
    (dict(ldc=199), INV), (dict(lda=(1 << 23) + 16), UNS), (dict(ldb=1 << 23), UNS),
    (dict(ldas=(1 << 21) + 1), UNS), (dict(m=2 ** 31 - 1, n=2 ** 31 - 1, ldc=2 ** 31), UNS),
    (dict(add=2 * P, ldadd=200), UNS), (dict(add=2 * P, ldadd=199), INV),
    (dict(add=2 * P + 2, ldadd=200), INV),
    (dict(add=P, ldadd=200), INV),                       # c in place, fp16
    (dict(add=P, ldadd=200, dtype=L.LMOP_F32), UNS),     # c in place, fp32
    (dict(add=P, ldadd=201, dtype=L.LMOP_F32), INV),
])
def test_matmul(ctx, change, status):
    assert _call(ctx, "lmop_matmul", _args(L.lmop_matmul_args, MM, **change)) == status


@pytest.mark.parametrize("change,status", [
    ({}, UNS),
    (dict(n_tokens=0), OK), (dict(n_tokens=-1), INV), (dict(n_slots=-1), INV),
    (dict(q=None, k=None, v=None), OK),
    (dict(q=None, q_out=None), UNS), (dict(k=None, k_out=None), UNS), (dict(v=None, v_out=None), UNS),
    (dict(q=None, k=None, pos=None), UNS),               # values alone need no position
    (dict(pos=None), INV), (dict(pos=P + 1), INV), (dict(slot=P + 2), INV),
    (dict(q_gain=P + 1), INV), (dict(k_gain=P + 2), INV), (dict(q_gain=P, k_gain=P), UNS),
    (dict(dtype=L.LMOP_F32), INV), (dict(dtype=L.LMOP_BF16), UNS), (dict(v_layout=2), INV),
    (dict(n_tokens=2 ** 31 - 1, n_slots=2 ** 31 - 1), UNS),
    (dict(n_slots=6), INV), (dict(n_slots=6, slot=P), UNS),
    (dict(q_out=None), INV), (dict(k_out=None), INV), (dict(v_out=None), INV),
    (dict(ldq=255), INV), (dict(ldk=255), INV), (dict(ldv=255), INV), (dict(ldqo=255), INV),
    (dict(ldko=255), INV), (dict(ldvo=255), INV), (dict(q=P + 1), INV), (dict(v_out=P + 1), INV),
    (dict(v_layout=L.LMOP_V_COLUMNS, ldvo=6), INV), (dict(v_layout=L.LMOP_V_COLUMNS, ldvo=7), UNS),
    (dict(q_out=P), UNS), (dict(q_out=P, ldqo=300), INV),
    (dict(k_out=P), UNS), (dict(k_out=P, slot=P), INV), (dict(k_out=P, ldko=300), INV),
    (dict(v_out=P), INV),
])
def test_qk_norm_rope(ctx, change, status):
    assert _call(ctx, "lmop_qk_norm_rope", _args(L.lmop_qk_norm_rope_args, QK, **change)) == status


@pytest.mark.parametrize("m,n,refused", [(2 ** 30, 16, False), (2 ** 30 + 1, 1, True), (2 ** 31 - 1, 1, True),
                                         (1, 2 ** 31 - 1, True), (16, 2 ** 30, False),
                                         (2 ** 30, 256, False), (2 ** 30, 257, True)])
def test_matmul_size_limits(ctx, m, n, refused):
    a = _args(L.lmop_matmul_args, MM, m=m, n=n, ldc=n)
    assert _call(ctx, "lmop_matmul", a) == UNS
    assert ("too large" in L._lib.lmop_last_error(ctx.ctx).decode()) == refused


@pytest.mark.parametrize("name", ["lmop_quantize", "lmop_matmul", "lmop_qk_norm_rope"])
def test_null(ctx, name):
    assert _call(ctx, name, None) == INV
    assert getattr(L._lib, name)(None, None) == INV


def test_binding_valid_calls_reach_the_library(ctx):
    assert _status(ctx.quantize, torch.zeros(3, 200, dtype=torch.bfloat16)) == UNS
    q, s = torch.zeros(3, 208, dtype=F8)[:, :200], torch.ones(3, 2)
    w, sw = torch.zeros(130, 208, dtype=F8)[:, :200], torch.ones(2, 2)
    assert _status(ctx.matmul, q, s, w, sw) == UNS
    one = torch.zeros(1, 256, dtype=torch.float16)
    assert _status(ctx.qk_norm_rope, one, pos=torch.zeros(1, dtype=torch.int32)) == UNS


def test_binding_refuses(ctx):
    q, s = torch.zeros(3, 208, dtype=F8)[:, :200], torch.ones(3, 2)
    w, sw = torch.zeros(130, 208, dtype=F8)[:, :200], torch.ones(2, 2)
    for a in [(q.float(), s, w, sw), (q, s.half(), w, sw), (q, s[:, :1], w, sw),
              (q, s, w[:, :100], sw), (q, s, w, sw[:1]), (q, s, w, sw.repeat(2, 1)),
              (q.t(), s, w, sw)]:
        with pytest.raises(ValueError):
            ctx.matmul(*a)
    with pytest.raises(ValueError):  # the last row's storage ends at its last code
        ctx.matmul(torch.zeros(3 * 208 - 8, dtype=F8).as_strided((3, 200), (208, 1)), s, w, sw)
    with pytest.raises(ValueError):
        ctx.matmul(q, s, w, sw, out=torch.zeros(3, 129))
    assert _status(ctx.matmul, q, s, w, sw, out=torch.zeros(3, 130).expand(3, 130)[:, :]) == UNS
    with pytest.raises(ValueError):  # columns of a matrix are not rows
        ctx.quantize(torch.zeros(200, 3, dtype=torch.float16).t())
    assert _status(ctx.quantize, torch.zeros(1, 200, dtype=torch.float16).expand(3, 200)) == INV
    with pytest.raises(ValueError):
        ctx.quantize(torch.zeros(3, 200, dtype=torch.float16), gate=torch.zeros(3, 200))
    x = torch.zeros(4, 256, dtype=torch.float16)
    pos = torch.zeros(4, dtype=torch.int32)
    for kw in [dict(q=x, pos=pos.long()), dict(q=x, pos=pos[:3]), dict(q=x[:, :128], pos=pos),
               dict(q=x.float(), pos=pos), dict(k=x, pos=pos), dict(pos=pos),
               dict(q=x, pos=pos, q_gain=torch.ones(32)),
               dict(q=x, pos=pos, q_gain=torch.ones(64, dtype=torch.float64)),
               dict(q=x, k=x.bfloat16(), k_out=x, pos=pos),
               dict(k=x, v=x, k_out=x.clone(), v_out=x[:3].clone(), pos=pos),
               dict(q=x, pos=pos, slot=pos[:2])]:
        with pytest.raises(ValueError):
            ctx.qk_norm_rope(**kw)
    with pytest.raises(ValueError):  # a tensor of another device
        L.Context(dataclasses.replace(SHAPES["tiny"]), device=-1).quantize(
            torch.empty(3, 200, dtype=torch.float16, device="meta"))


@pytest.mark.parametrize("tokens,heads,refused", [(1, 2 ** 23, True), (64, 2 ** 23, True), (64, 2 ** 22, False),
                                                  (1, 2 ** 22, False), (2 ** 22, 64, False)])
def test_qk_norm_rope_heads_fit_a_launch(tokens, heads, refused):
    """Values written as columns take heads * head_dim / 64 workgroups of 256 threads for each 64
    tokens: 2^24 of them are more threads than HIP launches at a time."""
    c = L.Context(dataclasses.replace(SHAPES["tiny"], n_heads=heads, n_kv_heads=heads, head_dim=128), device=-1)
    row = heads * 128
    a = _args(L.lmop_qk_norm_rope_args, QK, n_tokens=tokens, n_slots=tokens, v_layout=L.LMOP_V_COLUMNS, ldvo=tokens,
              **{f: row for f in ("ldq", "ldk", "ldv", "ldqo", "ldko")})
    assert _call(c, "lmop_qk_norm_rope", a) == UNS
    assert ("too many" in L._lib.lmop_last_error(c.ctx).decode()) == refused


def test_a_ctx_dropped_in_a_capture_is_freed_later(monkeypatch):
    """Freeing one waits and frees memory, which ends the capture; a garbage collection may come
    at any time."""
    freed = []
    monkeypatch.setattr(L, "lmop_destroy", lambda h: freed.append(h.value))
    capturing = [True]
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: capturing[0])
    ctx = L.Context(SHAPES["tiny"], device=-1)
    handle, ctx.device = ctx.ctx.value, 0
    del ctx
    assert freed == []
    capturing[0] = False
    other = L.Context(SHAPES["tiny"], device=-1)
    assert freed == [handle]
    other.device = 0
    handle = other.ctx.value
    del other
    assert freed[1:] == [handle]
    assert not L._dropped
