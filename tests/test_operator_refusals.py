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


# ---------------------------------------------------------------- the paged cache and its attention
CACHE = dict(k=P, v=P, page_stride=4096, n_pages=10, page_size=16, dtype=L.LMOP_F16)
BATCH = dict(table=P, length=P, start=P, ld_table=8, max_pages=8, n_seqs=3, n_tokens=7)
APPEND = dict(q=P, k=P, v=P, q_out=2 * P, ldq=256, ldk=256, ldv=256, ldqo=256, first=5, rotate=1, dtype=L.LMOP_F16)
ATTEND = dict(q=P, out=2 * P, ldq=256, ldo=256, max_tokens=5, max_length=100, dtype=L.LMOP_F16, workspace=P,
              workspace_bytes=1 << 30)
SELECT = dict(q=P, blocks=P, ldq=256, n_blocks=4, max_length=100, dtype=L.LMOP_F16)
PAGED = {"lmop_cache_append": (L.lmop_append_args, APPEND), "lmop_attend": (L.lmop_attend_args, ATTEND),
         "lmop_select_blocks": (L.lmop_select_args, SELECT)}
E8 = dict(cache_dtype=L.LMOP_E4M3, cache_k_exp=P, cache_v_exp=P)


def _paged(ctx, name, **change):
    struct, base = PAGED[name]
    parts = {"cache": dict(CACHE), "batch": dict(BATCH), "": dict(base)}
    if name == "lmop_select_blocks":
        parts["cache"]["k_mean"] = P
    for k, v in change.items():
        head, _, rest = k.partition("_")
        at, key = (head, rest) if head in ("cache", "batch") else ("", k)
        parts[at][key] = v
    a = _args(struct, parts[""])
    for n, t in (("cache", L.lmop_cache), ("batch", L.lmop_batch)):
        for f, v in parts[n].items():
            setattr(getattr(a, n), f, v)
    return a


@pytest.mark.parametrize("name", PAGED)
@pytest.mark.parametrize("change,status", [
    ({}, UNS), (dict(batch_n_tokens=0), OK), (dict(batch_n_seqs=0), OK), (dict(batch_n_tokens=-1), INV),
    (dict(batch_n_seqs=-1), INV), (dict(batch_max_pages=-1), INV), (dict(dtype=L.LMOP_F32), INV), (dict(dtype=-1), INV),
    (dict(dtype=L.LMOP_E4M3), INV), (dict(cache_page_size=0), INV), (dict(cache_page_size=8), INV),
    (dict(cache_page_size=48), INV), (dict(cache_page_size=512), INV), (dict(cache_n_pages=0), INV),
    (dict(cache_n_pages=-3), INV), (dict(batch_table=None), INV), (dict(batch_table=P + 2), INV),
    (dict(batch_ld_table=7), INV), (dict(batch_length=None), INV), (dict(batch_length=P + 1), INV),
    (dict(batch_start=P + 2), INV), (dict(batch_start=None), INV), (dict(q=P + 1), INV), (dict(ldq=255), INV),
    (dict(batch_n_tokens=2 ** 31 - 1, batch_n_seqs=2 ** 31 - 1), UNS),
    (dict(batch_max_pages=2 ** 31 - 1, batch_ld_table=2 ** 31), UNS),
])
def test_paged(ctx, name, change, status):
    if name == "lmop_attend" and change.get("batch_n_tokens", 1) > 2 ** 20:
        change = {**change, "max_tokens": 1, "batch_start": None}
    assert _call(ctx, name, _paged(ctx, name, **change)) == status


@pytest.mark.parametrize("name", ["lmop_cache_append", "lmop_attend"])
@pytest.mark.parametrize("change,status", [
    (E8, UNS), (dict(E8, dtype=L.LMOP_BF16), UNS), (dict(cache_dtype=L.LMOP_BF16), INV), (dict(cache_dtype=L.LMOP_F32), INV),
    (dict(cache_dtype=9), INV), (dict(cache_dtype=L.LMOP_BF16, dtype=L.LMOP_BF16), UNS), (dict(E8, cache_k_exp=None), INV),
    (dict(E8, cache_v_exp=P + 8), INV), (dict(cache_k_exp=P), INV), (dict(cache_k=None), INV), (dict(cache_v=P + 8), INV),
    (dict(cache_k_mean=P + 8), INV), (dict(cache_page_stride=4095), INV), (dict(cache_page_stride=4104), INV),
    (dict(cache_page_stride=4112), UNS), (dict(cache_page_stride=1 << 40), UNS),
])
def test_paged_cache(ctx, name, change, status):
    assert _call(ctx, name, _paged(ctx, name, **change)) == status


@pytest.mark.parametrize("change,status", [
    (dict(first=-1), INV), (dict(rotate=2), INV), (dict(rotate=0), UNS), (dict(k=None), INV), (dict(v=None), INV),
    (dict(ldk=255), INV), (dict(ldv=255), INV), (dict(q_out=None), INV), (dict(q=None, q_out=None), UNS),
    (dict(q_out=P), UNS), (dict(q_out=P, ldqo=300), INV), (dict(ldqo=255), INV),
    (dict(batch_start=None, batch_n_tokens=3), UNS),
])
def test_cache_append(ctx, change, status):
    assert _call(ctx, "lmop_cache_append", _paged(ctx, "lmop_cache_append", **change)) == status


@pytest.mark.parametrize("change,status", [
    (dict(out=None), INV), (dict(out=P), INV), (dict(ldo=255), INV), (dict(lse=P), UNS), (dict(lse=P + 2), INV),
    (dict(max_tokens=0), INV), (dict(max_tokens=8), INV), (dict(max_tokens=-1), INV), (dict(max_length=-1), INV),
    (dict(max_length=128), UNS), (dict(max_length=129), INV), (dict(max_length=0), UNS),
    (dict(prefix_length=-1), INV), (dict(prefix_length=3), INV), (dict(prefix_length=3, prefix=P), UNS),
    (dict(prefix_length=3, prefix=P + 1), INV), (dict(prefix_length=2 ** 30, prefix=P), UNS),
    (dict(n_blocks=-1), INV), (dict(n_blocks=3), INV), (dict(n_blocks=3, blocks=P), UNS), (dict(blocks=P), INV),
    (dict(n_blocks=3, blocks=P + 2), INV), (dict(n_blocks=3, blocks=P, prefix_length=3, prefix=P), INV),
    (dict(n_blocks=1025, blocks=P), UNS), (dict(scale=-1.0), INV), (dict(scale=float("nan")), INV),
    (dict(scale=float("inf")), INV), (dict(scale=1e-35), INV), (dict(scale=0.5), UNS),
    (dict(batch_start=None, batch_n_tokens=3), INV), (dict(batch_start=None, batch_n_tokens=3, max_tokens=1), UNS),
    (dict(batch_n_seqs=1, batch_n_tokens=1, max_tokens=1, batch_max_pages=2 ** 20, batch_ld_table=2 ** 20,
          max_length=2 ** 20, workspace_bytes=0), INV),
    (dict(batch_n_seqs=1, batch_n_tokens=1, max_tokens=1, batch_max_pages=2 ** 20, batch_ld_table=2 ** 20,
          max_length=2 ** 20, workspace=None), INV),
    (dict(batch_n_seqs=1, batch_n_tokens=1, max_tokens=1, batch_max_pages=2 ** 20, batch_ld_table=2 ** 20,
          max_length=2 ** 20, workspace=P + 8), INV),
    (dict(batch_n_seqs=1, batch_n_tokens=1, max_tokens=1, batch_max_pages=2 ** 20, batch_ld_table=2 ** 20,
          max_length=2 ** 20), UNS),
])
def test_attend(ctx, change, status):
    assert _call(ctx, "lmop_attend", _paged(ctx, "lmop_attend", **change)) == status


def test_attend_workspace(ctx):
    def size(**change):
        n = C.c_uint64(99)
        st = L._lib.lmop_attend_workspace(ctx.ctx, C.byref(_paged(ctx, "lmop_attend", **change)), C.byref(n))
        return st, n.value

    assert size(workspace=None, q=None, out=None, cache_k=None) == (OK, 0)
    assert size(batch_n_tokens=0) == (OK, 0)
    assert size(max_length=129)[0] == INV
    long = dict(batch_n_seqs=1, batch_n_tokens=1, max_tokens=1, batch_max_pages=2 ** 16, batch_ld_table=2 ** 16,
                max_length=2 ** 20)
    st, n = size(**long)
    assert st == OK and n > 0 and n % (4 * 66 * 4) == 0
    assert _call(ctx, "lmop_attend", _paged(ctx, "lmop_attend", **long, workspace_bytes=n - 1)) == INV
    assert _call(ctx, "lmop_attend", _paged(ctx, "lmop_attend", **long, workspace_bytes=n)) == UNS
    assert L._lib.lmop_attend_workspace(ctx.ctx, C.byref(_paged(ctx, "lmop_attend")), None) == INV
    assert L._lib.lmop_attend_workspace(ctx.ctx, None, C.byref(C.c_uint64())) == INV


@pytest.mark.parametrize("change,status", [
    (dict(blocks=None), INV), (dict(blocks=P + 2), INV), (dict(cache_k_mean=None), INV), (dict(cache_k_mean=P + 2), INV),
    (dict(n_blocks=0), OK), (dict(n_blocks=-1), INV), (dict(n_blocks=1024), UNS), (dict(n_blocks=1025), UNS),
    (dict(max_length=-1), INV), (dict(max_length=16384 * 16), UNS), (dict(max_length=16384 * 16 + 1), UNS),
    (dict(cache_k=None, cache_v=None, cache_dtype=77, cache_page_stride=0), UNS),
])
def test_select_blocks(ctx, change, status):
    assert _call(ctx, "lmop_select_blocks", _paged(ctx, "lmop_select_blocks", **change)) == status


@pytest.mark.parametrize("name", list(PAGED) + ["lmop_attend_workspace"])
def test_paged_null(ctx, name):
    extra = (None,) if name.endswith("workspace") else ()
    assert getattr(L._lib, name)(ctx.ctx, None, *extra) == INV
    assert getattr(L._lib, name)(None, None, *extra) == INV


def _host_cache(dt=torch.float16, mean=None, pages=6, **kw):
    k, v = (torch.zeros(pages, 4, 16, 64, dtype=dt) for _ in range(2))
    if dt is F8:
        kw.setdefault("k_exp", torch.zeros(pages, 4, 16, dtype=torch.uint8))
        kw.setdefault("v_exp", torch.zeros(pages, 4, 16, dtype=torch.uint8))
    return L.PagedCache(k, v, k_mean=mean, **kw)


def test_binding_paged_valid_calls_reach_the_library(ctx):
    x = torch.zeros(3, 256, dtype=torch.float16)
    one = dict(table=torch.zeros(3, 2, dtype=torch.int32), length=torch.ones(3, dtype=torch.int32))
    two = dict(one, start=torch.tensor([0, 1, 2, 3], dtype=torch.int32))
    c = _host_cache(mean=torch.zeros(6, 4, 64, dtype=torch.float16))
    for a in (one, two):
        assert _status(ctx.cache_append, c, x, x, q=x, **a) == UNS
        assert _status(ctx.attend, c, x, **a) == UNS
        assert _status(ctx.attend, c, x, prefix=torch.zeros(2, dtype=torch.int32), prefix_length=30, **a) == UNS
        assert _status(ctx.attend, c, x, blocks=torch.zeros(3, 4, 2, dtype=torch.int32), lse=torch.zeros(3, 4), **a) == UNS
        assert _status(ctx.select_blocks, c, x, 2, **a) == UNS
    assert _status(ctx.attend, _host_cache(F8), x.bfloat16(), **one) == UNS
    assert _status(ctx.attend, c, x, max_length=33, **one) == INV


def test_binding_paged_refuses(ctx):
    x = torch.zeros(3, 256, dtype=torch.float16)
    tab, ln, st = torch.zeros(3, 2, dtype=torch.int32), torch.ones(3, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)
    a = dict(table=tab, length=ln)
    mean = torch.zeros(6, 4, 64, dtype=torch.float16)
    c = _host_cache(mean=mean)
    k = torch.zeros(6, 4, 16, 64, dtype=torch.float16)
    for bad in (lambda: L.PagedCache(k[0], k[0]), lambda: L.PagedCache(k.float(), k.float()), lambda: L.PagedCache(k, k[:5]),
                lambda: L.PagedCache(k, k.bfloat16()), lambda: L.PagedCache(k.transpose(1, 2), k.transpose(1, 2)),
                lambda: L.PagedCache(k, torch.zeros(12, 4, 16, 64, dtype=torch.float16)[::2]),
                lambda: L.PagedCache(k, k, k_exp=torch.zeros(6, 4, 16, dtype=torch.uint8)),
                lambda: L.PagedCache(k.to(F8), k.to(F8)), lambda: _host_cache(F8, k_exp=torch.zeros(6, 4, 8, dtype=torch.uint8)),
                lambda: _host_cache(F8, v_exp=torch.zeros(6, 4, 16)), lambda: _host_cache(mean=mean.bfloat16()),
                lambda: _host_cache(mean=mean[:, :2]), lambda: _host_cache(F8, mean=mean.float()),
                lambda: L.PagedCache(k, k.to("meta"))):
        with pytest.raises(ValueError):
            bad()
    other = L.PagedCache(*(torch.zeros(6, 2, 16, 64, dtype=torch.float16) for _ in range(2)))
    for f in (lambda **kw: ctx.attend(**{**dict(cache=c, q=x), **a, **kw}),
              lambda **kw: ctx.select_blocks(**{**dict(cache=c, q=x, n_blocks=2), **a, **kw}),
              lambda **kw: ctx.cache_append(**{**dict(cache=c, k=kw.get("q", x), v=x), **a, **kw})):
        for kw in (dict(cache=other), dict(table=tab.long()), dict(table=tab.t()), dict(table=tab[:2]), dict(length=ln[:2]),
                   dict(length=ln.float()), dict(start=st[:3]), dict(start=st.long()), dict(q=x.float()), dict(q=x[:, :128]),
                   dict(q=x.bfloat16()), dict(q=x[:2])):
            with pytest.raises(ValueError):
                f(**kw)
    for kw in (dict(out=x[:2]), dict(out=x.float()), dict(lse=torch.zeros(3, 3)), dict(lse=torch.zeros(3, 8)[:, :4]),
               dict(lse=torch.zeros(3, 4, dtype=torch.float64)), dict(blocks=torch.zeros(3, 4, 2)),
               dict(blocks=torch.zeros(3, 2, 2, dtype=torch.int32)), dict(blocks=torch.zeros(4, 3, 2, dtype=torch.int32).transpose(0, 1)),
               dict(prefix_length=3), dict(prefix=tab[0], prefix_length=33), dict(prefix=tab[0].long(), prefix_length=3)):
        with pytest.raises(ValueError):
            ctx.attend(c, x, **a, **kw)
    for kw in (dict(v=x[:2]), dict(v=x.bfloat16()), dict(q=x, q_out=x[:2])):
        with pytest.raises(ValueError):
            ctx.cache_append(c, x, **{"v": x, **a, **kw})
    with pytest.raises(ValueError):
        ctx.select_blocks(_host_cache(), x, 2, **a)
    with pytest.raises(ValueError):
        ctx.select_blocks(c, x, 2, out=torch.zeros(3, 4, 2), **a)
    with pytest.raises(ValueError):  # a tensor of another device
        ctx.attend(c, x.to("meta"), **a)


def test_binding_attend_takes_its_workspace_from_the_caller(ctx):
    """Below Context nothing says which stream torch's allocations would be ordered with."""
    q, c = torch.zeros(1, 256, dtype=torch.float16), _host_cache()
    a = (ctx.ctx, ctx.heads, c, q, torch.empty_like(q), torch.zeros(1, 2 ** 16, dtype=torch.int32), torch.ones(1, dtype=torch.int32))
    assert _status(L.lmop_attend, *a, max_length=2 ** 20) == INV
    for bad in (lambda n: torch.zeros(n), lambda n: torch.zeros(2 * n, dtype=torch.uint8)[::2],
                lambda n: torch.zeros(n, dtype=torch.uint8, device="meta")):
        with pytest.raises(ValueError):
            L.lmop_attend(*a, max_length=2 ** 20, workspace=bad)
    assert _status(L.lmop_attend, *a, max_length=2 ** 20, workspace=lambda n: torch.zeros(n - 1, dtype=torch.uint8)) == INV
    assert _status(L.lmop_attend, *a, max_length=2 ** 20, workspace=lambda n: torch.zeros(n, dtype=torch.uint8)) == UNS


def test_binding_refuses_lists_of_no_blocks(ctx):
    """They would reach the library as a call without lists, whose tokens attend to all their keys."""
    x = torch.zeros(3, 256, dtype=torch.float16)
    a = dict(table=torch.zeros(3, 2, dtype=torch.int32), length=torch.ones(3, dtype=torch.int32))
    c = _host_cache(mean=torch.zeros(6, 4, 64, dtype=torch.float16))
    none = torch.zeros(3, 4, 0, dtype=torch.int32)
    with pytest.raises(ValueError, match="n_blocks at least 1"):
        ctx.attend(c, x, blocks=none, **a)
    with pytest.raises(ValueError, match="n_blocks at least 1"):
        ctx.attend(c, x, blocks=none, prefix=torch.zeros(2, dtype=torch.int32), prefix_length=30, **a)
    with pytest.raises(ValueError, match="n_blocks at least 1"):
        ctx.attend(c, x, blocks=torch.tensor(0, dtype=torch.int32), **a)
    with pytest.raises(ValueError, match="n_blocks at least 1"):
        ctx.select_blocks(c, x, 0, **a)
    with pytest.raises(ValueError, match="n_blocks at least 1"):
        ctx.select_blocks(c, x, 2, out=none, **a)


def test_binding_select_refuses_an_out_of_another_number_of_blocks(ctx):
    """The number asked for is the number chosen."""
    x = torch.zeros(3, 256, dtype=torch.float16)
    a = dict(table=torch.zeros(3, 2, dtype=torch.int32), length=torch.ones(3, dtype=torch.int32))
    c = _host_cache(mean=torch.zeros(6, 4, 64, dtype=torch.float16))
    assert _status(ctx.select_blocks, c, x, 2, out=torch.zeros(3, 4, 2, dtype=torch.int32), **a) == UNS
    for out in (torch.zeros(3, 4, 3, dtype=torch.int32), torch.zeros(3, 4, 1, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)):
        with pytest.raises(ValueError, match="for 2 blocks"):
            ctx.select_blocks(c, x, 2, out=out, **a)


def test_binding_append_refuses_queries_to_write_without_any(ctx):
    """They came back as they were, as if rotated."""
    x = torch.zeros(3, 256, dtype=torch.float16)
    a = dict(table=torch.zeros(3, 2, dtype=torch.int32), length=torch.ones(3, dtype=torch.int32))
    with pytest.raises(ValueError, match="q_out without q"):
        ctx.cache_append(_host_cache(), x, x, q_out=torch.zeros_like(x), **a)
    assert _status(ctx.cache_append, _host_cache(), x, x, **a) == UNS
