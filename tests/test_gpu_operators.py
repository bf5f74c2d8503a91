"""The block-scaled FP8 product, its quantiser and the query/key norm with
rotation, against plain implementations in 64 bits.

Tolerances.  A rounding to a type is off by at most half a step: eps / 2
relative (eps = torch.finfo(t).eps).  A sum of N fp32 terms is off by at most
N * 2^-23 of the sum of their magnitudes, whatever its order and however each
addition rounds."""
import math

import numpy as np
import pytest
import torch

from synth import SHAPES

pytestmark = pytest.mark.gpu

F8 = torch.float8_e4m3fn
DT = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
G = 128


@pytest.fixture(scope="module")
def L():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_31808_amd import lmop
    return lmop


class Shape:
    def __init__(self, nq=4, nkv=2, hd=64, eps=1e-5, theta=1e4):
        self.n_layers, self.d_model, self.d_ff, self.vocab, self.group_size = 0, 64, 64, 2, 32
        self.n_heads, self.n_kv_heads, self.head_dim = nq, nkv, hd
        self.rms_eps, self.rope_theta = eps, theta


def _ctx(L, *a, max_seq=4096, **k):
    return L.Context(Shape(*a, **k), device=0, stream=torch.cuda.current_stream().cuda_stream,
                     max_seq=max_seq)


@pytest.fixture(scope="module")
def ctx(L):
    return _ctx(L)


def _gen(seed):
    return torch.Generator().manual_seed(seed)


# ---------------------------------------------------------------- quantiser
def _e4m3(y):
    """Nearest E4M3 value of float64 y (|y| <= 448 and a little), and half its step."""
    y = np.asarray(y, np.float64)
    e = np.floor(np.log2(np.maximum(np.abs(y), 2.0 ** -6)))
    step = 2.0 ** (np.maximum(e, -6) - 3)
    return np.clip(np.round(y / step) * step, -448, 448), step / 2


def _quant_input(rows, cols, dt, seed, pad=0, shift=0):
    """[rows][cols] inside a wider tensor, `shift` elements off its alignment."""
    t = torch.full((rows, cols + pad + shift), float("nan"), dtype=dt)
    x = torch.randn(rows, cols, generator=_gen(seed)) * 3
    x[:, ::37] *= 30
    t[:, shift:shift + cols] = x.to(dt)
    return t.cuda()[:, shift:shift + cols]


def _check_codes(q, s, y64, rel):
    """Codes and scales of y64 (float64 [rows][cols]) that is known within `rel`."""
    rows, cols = y64.shape
    groups = -(-cols // G)
    yp = np.zeros((rows, groups * G))
    yp[:, :cols] = y64
    amax = np.maximum(np.abs(yp.reshape(rows, groups, G)).max(-1), 2.0 ** -40)
    # the scale: the maximum's own error and one division
    assert np.all(np.abs(s - amax / 448) <= amax / 448 * (rel + 2.0 ** -24))
    v = y64 * np.repeat(448 / amax, G, 1)[:, :cols]
    ref, half = _e4m3(v)
    # y, the maximum, 448 / amax and the product: each off by its own rounding
    slack = np.abs(v) * (2 * rel + 2 * 2.0 ** -24)
    assert np.all(np.abs(q - v) <= half + slack + 1e-30)
    return ref


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("rows,cols,pad,shift", [
    (1, 1, 0, 0), (1, 128, 0, 0), (3, 127, 0, 0), (5, 129, 7, 0), (2, 16, 0, 0), (17, 688, 0, 0),
    (33, 4096, 0, 0), (9, 1000, 24, 0), (4, 1000, 5, 3), (2, 14336, 0, 0), (7, 264, 8, 1),
    (130, 520, 0, 8)])
def test_quantize(ctx, dtype, rows, cols, pad, shift):
    print("quantize", dtype, rows, cols, pad, shift, flush=True)
    x = _quant_input(rows, cols, DT[dtype], rows * 31 + cols, pad, shift)
    q, s = ctx.quantize(x)
    y = x.double().cpu().numpy()
    got, sc = q.float().double().cpu().numpy(), s.double().cpu().numpy()
    ref = _check_codes(got, sc, y, 0.0)
    # the scale is the fp32 quotient; a code differs from the 64-bit one only at a tie
    yp = np.zeros((rows, s.shape[1] * G), np.float32)
    yp[:, :cols] = y
    amax = np.maximum(np.abs(yp.reshape(rows, -1, G)).max(-1), np.float32(2.0 ** -40))
    assert np.array_equal(s.cpu().numpy(), amax / np.float32(448))
    v32 = yp * np.repeat(np.float32(448) / amax, G, 1)
    assert np.array_equal(got, _e4m3(v32[:, :cols])[0])
    assert np.mean(got != ref) < 0.01


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("rows,cols,pad,shift", [(1, 1, 0, 0), (3, 130, 0, 0), (33, 688, 8, 0),
                                                 (5, 1001, 3, 1), (19, 2048, 0, 0)])
def test_quantize_gated(ctx, dtype, rows, cols, pad, shift):
    print("quantize gated", dtype, rows, cols, flush=True)
    x = _quant_input(rows, cols, DT[dtype], 5, pad, shift)
    gate = _quant_input(rows, cols, DT[dtype], 6, shift, pad)
    q, s = ctx.quantize(x, gate=gate)
    z = gate.double().cpu().numpy()
    y = z / (1 + np.exp(-z)) * x.double().cpu().numpy()
    # exp, one addition, a division and a product in fp32: a few 2^-24; the
    # exponent's rounding adds 2^-23 for each unit of |gate|
    rel = 2.0 ** -20 + np.abs(z).max() * 2.0 ** -23
    _check_codes(q.float().double().cpu().numpy(), s.double().cpu().numpy(), y, rel)


def test_quantize_extremes(ctx):
    """Zero groups, subnormals, the type's ends, infinities and NaN (which stay in their group)."""
    x = torch.ones(6, 3 * G, dtype=torch.float32)
    x[0, :G] = 0
    x[1, G:2 * G] = 1e-42
    x[2, G + 5] = float("inf")
    x[3, 2 * G + 127] = float("nan")
    x[4, 0] = 3e38
    x[5, :] = -2.0 ** -41
    q, s = ctx.quantize(x.cuda())
    q, s = q.float().cpu(), s.cpu()
    assert torch.all(q[0, :G] == 0) and s[0, 0] == torch.tensor(2.0 ** -40) / 448
    assert torch.all(q[1, G:2 * G] == 0)
    assert torch.isnan(s[2, 1]) and torch.isnan(q[2, G:2 * G]).all()
    assert torch.isnan(s[3, 2]) and torch.isnan(q[3, 2 * G:]).all()
    assert q[4, 0] == 448 and torch.all(q[4, 1:G] == 0)
    assert torch.all(q[5] == -224)
    ok = torch.ones(6, 3, dtype=torch.bool)
    ok[2, 1] = ok[3, 2] = False
    assert torch.isfinite(s[ok]).all()
    assert torch.isfinite(q.view(6, 3, G)[ok]).all()


@pytest.mark.parametrize("cols", [1, 100, 128, 200, 680])
def test_quantize_writes_its_rows_only(ctx, cols):
    rows, groups, up = 5, -(-cols // G), -(-cols // 16) * 16
    q = torch.full((rows, up + 32), 0x55, dtype=torch.uint8, device="cuda")
    s = torch.full((rows, groups + 2), 7.0, device="cuda")
    ctx.quantize(torch.randn(rows, cols, device="cuda"), out=(q[:, :cols], s[:, :groups]))
    assert torch.all(q[:, cols:up] == 0) and torch.all(q[:, up:] == 0x55)
    assert torch.all(s[:, groups:] == 7)


# ---------------------------------------------------------------- product
def _codes(rows, k, seed, pad=16):
    """Codes in rows a multiple of 16 bytes apart; what lies past k is NaN codes."""
    ld = -(-k // 16) * 16 + pad
    t = torch.full((rows, ld), 0x7F, dtype=torch.uint8)
    t[:, :k] = (torch.randn(rows, k, generator=_gen(seed)) * 60).clamp(-448, 448).to(F8).view(torch.uint8)
    return t.cuda().view(F8)[:, :k]


def _scales(rows, cols, seed, pad=1):
    s = torch.rand(rows, cols + pad, generator=_gen(seed)) * 0.01 + 1e-4
    return s.cuda()[:, :cols]


def _ref_matmul(a, sa, b, sb):
    """(A B^T, sum of magnitudes, sum over eights of features of the largest product's
    bound) in 64 bits."""
    f = torch.arange(a.shape[1], device=a.device) // G
    r = torch.arange(b.shape[0], device=a.device) // G
    A = a.float().double() * sa.double()[:, f]
    B = b.float().double() * sb.double()[r][:, f]

    def eights(x):
        x = torch.nn.functional.pad(x.abs(), (0, -x.shape[1] % 8))
        return x.view(x.shape[0], -1, 8).amax(-1)

    return (A @ B.t().contiguous(), A.abs() @ B.abs().t().contiguous(),
            eights(A) @ eights(B).t().contiguous())


def _check_product(c, a, sa, b, sb, add=None, fast=False):
    ref, mag, most = _ref_matmul(a, sa, b, sb)
    k = a.shape[1]
    if add is not None:
        ref, mag = ref + add.double(), mag + add.double().abs()
    # 128 terms of a group, the groups' fma chain, the scales' product, the addition
    tol = (G + -(-k // G) + 4) * 2.0 ** -23 * mag
    if c.dtype != torch.float32 or fast:
        # The 8-bit matrix instruction cuts off what lies below 2^-13 of the leading
        # bit of the largest of eight neighbouring products: less than 2^-13 of
        # that product (at most the product of the eights' largest values) from
        # each of the other seven.
        tol = tol + 7 * 2.0 ** -13 * most
    tol = tol + torch.finfo(c.dtype).eps / 2 * (ref.abs() + tol) + torch.finfo(c.dtype).tiny
    d = (c.double() - ref).abs()
    assert torch.all(d <= tol), f"off by {(d / tol).max():.3g} of the tolerance"


SIZES = [(1, 1, 1), (1, 16, 128), (2, 17, 15), (16, 64, 688), (17, 65, 129), (64, 128, 256),
         (65, 130, 1000), (129, 257, 384), (300, 200, 144), (1, 6144, 512), (24, 256, 2048),
         (257, 513, 640), (33, 96, 14336), (1, 128, 100), (7, 1024, 4096), (48, 2048, 1024),
         (100, 16, 256), (520, 520, 272), (1000, 48, 128), (31, 4100, 384)]


# where the larger tiles are the fastest
LARGE = [(2047, 4096, 1000), (300, 2050, 1100), (257, 4099, 700), (2500, 7001, 200),
         (3001, 5103, 1300), (4097, 6145, 130), (1001, 1103, 8448)]


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("m,n,k", SIZES + LARGE)
def test_matmul(ctx, dtype, m, n, k):
    print("matmul", dtype, m, n, k, flush=True)
    a, b = _codes(m, k, 1), _codes(n, k, 2, pad=0)
    sa, sb = _scales(m, -(-k // G), 3), _scales(-(-n // G), -(-k // G), 4, pad=0)
    c = ctx.matmul(a, sa, b, sb, dtype=DT[dtype])
    _check_product(c, a, sa, b, sb)
    add = torch.randn(m, n, generator=_gen(5)).cuda()
    wide = torch.full((m, n + 3), 9.0, dtype=DT[dtype], device="cuda")
    ctx.matmul(a, sa, b, sb, add=add, out=wide[:, :n])
    _check_product(wide[:, :n], a, sa, b, sb, add)
    assert torch.all(wide[:, n:] == 9)


@pytest.mark.parametrize("m,n,k", SIZES + LARGE)
def test_matmul_fast(ctx, m, n, k):
    print("fast", m, n, k, flush=True)
    a, b = _codes(m, k, 1), _codes(n, k, 2, pad=0)
    sa, sb = _scales(m, -(-k // G), 3), _scales(-(-n // G), -(-k // G), 4, pad=0)
    c = ctx.matmul(a, sa, b, sb, dtype=torch.float32, fast=True)
    _check_product(c, a, sa, b, sb, fast=True)
    # what the 16-bit results round
    assert torch.equal(c.half(), ctx.matmul(a, sa, b, sb, fast=True))
    assert torch.equal(c.bfloat16(), ctx.matmul(a, sa, b, sb, dtype=torch.bfloat16))
    add = torch.randn(m, n, generator=_gen(5)).cuda()
    want = add + c
    ctx.matmul(a, sa, b, sb, add=add, out=add, fast=True)
    assert torch.equal(add, want)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("n,k", [(200, 688), (1040, 1300), (5000, 256), (4100, 4096)])
def test_matmul_rows_do_not_depend_on_the_batch(ctx, n, k, dtype):
    """Any number of tokens gives a token the same bits: in any kernel and tile."""
    M = 2700
    a, b = _codes(M, k, 11), _codes(n, k, 12)
    sa, sb = _scales(M, -(-k // G), 13), _scales(-(-n // G), -(-k // G), 14)
    whole = ctx.matmul(a, sa, b, sb, dtype=DT[dtype])
    for m in (1, 2, 9, 16, 17, 32, 33, 48, 64, 65, 100, 128, 129, 200, 256, 257, 400, 513, 1024,
              2100):
        part = ctx.matmul(a[M - m:], sa[M - m:], b, sb, dtype=DT[dtype])
        assert torch.equal(part, whole[M - m:]), m


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("m,n,pad", [(4099, 16400, 8), (7001, 9000, 0), (300, 4100, 4)])
def test_matmul_large_results_are_written_once(ctx, dtype, m, n, pad):
    """Results too large for the caches are the rows of small calls, and nothing beside them
    is written."""
    print("large", dtype, m, n, flush=True)
    k = 144
    a, b = _codes(m, k, 1), _codes(n, k, 2, pad=0)
    sa, sb = _scales(m, -(-k // G), 3), _scales(-(-n // G), -(-k // G), 4, pad=0)
    wide = torch.full((m + 1, n + pad), 9.0, dtype=DT[dtype], device="cuda")
    c = wide[:m, :n]
    ctx.matmul(a, sa, b, sb, out=c)
    for r in (0, 37, m - 20):
        assert torch.equal(c[r:r + 20], ctx.matmul(a[r:r + 20], sa[r:r + 20], b, sb, dtype=DT[dtype]))
    _check_product(c[-40:], a[-40:], sa[-40:], b, sb)
    assert torch.all(wide[:m, n:] == 9) and torch.all(wide[m] == 9)
    if dtype == "f32":
        base = torch.randn(m, n, generator=_gen(5)).cuda()
        want = base + c
        wide[:m, :n] = base
        ctx.matmul(a, sa, b, sb, add=c, out=c)
        assert torch.equal(c, want)
        assert torch.all(wide[:m, n:] == 9) and torch.all(wide[m] == 9)


def test_matmul_columns_do_not_depend_on_the_weight(ctx):
    """A weight's first rows alone give the same bits."""
    m, n, k = 70, 2000, 1040
    a, b = _codes(m, k, 21), _codes(n, k, 22)
    sa, sb = _scales(m, -(-k // G), 23), _scales(-(-n // G), -(-k // G), 24)
    whole = ctx.matmul(a, sa, b, sb, dtype=torch.float32)
    for c in (1, 16, 100, 129, 700, 1999):
        assert torch.equal(ctx.matmul(a, sa, b[:c], sb[:-(-c // G)], dtype=torch.float32),
                           whole[:, :c]), c


def test_matmul_k_zero_and_in_place(ctx):
    e8, e32 = torch.empty(3, 0, dtype=F8, device="cuda"), torch.empty(3, 0, device="cuda")
    w8, w32 = torch.empty(5, 0, dtype=F8, device="cuda"), torch.empty(1, 0, device="cuda")
    assert torch.all(ctx.matmul(e8, e32, w8, w32) == 0)
    add = torch.randn(3, 5, device="cuda")
    assert torch.equal(ctx.matmul(e8, e32, w8, w32, dtype=torch.float32, add=add), add)
    for m, n, k in ((40, 300, 400), (1, 256, 4096), (300, 300, 300)):
        a, b = _codes(m, k, 1), _codes(n, k, 2)
        sa, sb = _scales(m, -(-k // G), 3), _scales(-(-n // G), -(-k // G), 4)
        x = torch.randn(m, n, device="cuda")
        want = ctx.matmul(a, sa, b, sb, dtype=torch.float32, add=x)
        ctx.matmul(a, sa, b, sb, add=x, out=x)
        assert torch.equal(x, want)


@pytest.mark.parametrize("m,n,k", [(5, 40, 300), (200, 300, 520), (20, 700, 1024)])
def test_matmul_nan_and_infinity_stay_where_they_are(ctx, m, n, k):
    a, b = _codes(m, k, 1), _codes(n, k, 2)
    sa, sb = _scales(m, -(-k // G), 3), _scales(-(-n // G), -(-k // G), 4)
    clean = ctx.matmul(a, sa, b, sb, dtype=torch.float32)
    a.view(torch.uint8)[1, k - 1] = 0x7F
    b.view(torch.uint8)[7, 0] = 0xFF
    sa[3, 0] = float("nan")
    sa[4, 1] = float("inf")
    c = ctx.matmul(a, sa, b, sb, dtype=torch.float32)
    rows = torch.tensor([r not in (1, 3, 4) for r in range(m)]).cuda()
    cols = torch.tensor([j != 7 for j in range(n)]).cuda()
    assert torch.equal(c[rows][:, cols], clean[rows][:, cols])
    assert torch.isnan(c[1]).all() and torch.isnan(c[3]).all() and torch.isnan(c[:, 7]).all()
    assert not torch.isfinite(c[4]).any()


def test_matmul_zero_rows(ctx):
    assert ctx.matmul(_codes(0, 128, 1), _scales(0, 1, 1), _codes(9, 128, 2), _scales(1, 1, 2)).shape == (0, 9)
    assert ctx.matmul(_codes(9, 128, 1), _scales(9, 1, 1), _codes(0, 128, 2), _scales(0, 1, 2)).shape == (9, 0)
    q, s = ctx.quantize(torch.empty(0, 300, dtype=torch.float16, device="cuda"))
    assert q.shape == (0, 300) and s.shape == (0, 3)


def test_matmul_rows_past_32_bits(ctx):
    """Rows whose byte offsets pass 2^32 (in the codes and in C)."""
    m, n, k = 2100, 72, 128
    ld = 1 << 21
    wide = torch.empty(m * ld, dtype=torch.uint8, device="cuda")
    a = wide.view(F8).as_strided((m, k), (ld, 1))
    a.view(torch.uint8).copy_(_codes(m, k, 1).view(torch.uint8))
    b, sa, sb = _codes(n, k, 2), _scales(m, 1, 3), _scales(1, 1, 4)
    out = torch.empty(m * (1 << 20), dtype=torch.float32, device="cuda").as_strided((m, n), (1 << 20, 1))
    ctx.matmul(a, sa, b, sb, out=out)
    _check_product(out, a, sa, b, sb)


# ---------------------------------------------------------------- norm, rotation, cache
def _ref_heads(x, nh, hd, gain, pos, eps, theta):
    """(rotated heads, |y1| + |y2| of each pair) in 64 bits."""
    T = x.shape[0]
    x = x.double().cpu().view(T, nh, hd)
    if gain is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * gain.double().cpu()
    half = hd // 2
    ang = pos.double().cpu()[:, None, None] * theta ** (-2.0 * torch.arange(half).double() / hd)
    c, s = ang.cos(), ang.sin()
    x1, x2 = x[..., :half], x[..., half:]
    mag = x1.abs() + x2.abs()
    return (torch.cat((x1 * c - x2 * s, x1 * s + x2 * c), -1).view(T, -1),
            torch.cat((mag, mag), -1).view(T, -1))


def _close_heads(got, ref, mag, dt):
    # the mean of squares (64 partial sums at most), square root, quotient and
    # two products, the table's rounding, two products and an addition: under
    # 32 roundings of 2^-24; then one to the type (smallest step: 2^-24 in fp16)
    tol = 32 * 2.0 ** -24 * mag
    tol = tol + torch.finfo(dt).eps / 2 * (ref.abs() + tol) + 2.0 ** -25
    d = (got.double().cpu() - ref).abs()
    assert torch.all(d <= tol), f"off by {(d / tol).max():.3g} of the tolerance"


def _wide(T, n, dt, seed, pad, shift=0):
    t = torch.full((T, n + pad + shift), float("nan"), dtype=dt)
    t[:, shift:shift + n] = (torch.randn(T, n, generator=_gen(seed)) * 2).to(dt)
    return t.cuda()[:, shift:shift + n]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("columns", [False, True])
@pytest.mark.parametrize("T,nq,nkv,hd,pad,shift", [
    (1, 32, 8, 128, 0, 0), (1, 1, 1, 64, 0, 0), (9, 32, 8, 128, 0, 0), (63, 7, 1, 64, 8, 0),
    (64, 6, 2, 128, 0, 0), (65, 8, 8, 64, 0, 0), (200, 4, 4, 64, 0, 0), (130, 12, 4, 128, 16, 0),
    (33, 5, 5, 64, 3, 1), (77, 3, 1, 128, 8, 8)])
def test_qk_norm_rope(L, dtype, columns, T, nq, nkv, hd, pad, shift):
    print("qk", dtype, columns, T, nq, nkv, hd, pad, shift, flush=True)
    dt, theta, eps = DT[dtype], 5e5, 1e-5
    ctx = _ctx(L, nq, nkv, hd, eps=eps, theta=theta, max_seq=1000)
    q, k, v = (_wide(T, n * hd, dt, 7 + i, pad, shift) for i, n in enumerate((nq, nkv, nkv)))
    qg, kg = (1 + 0.3 * torch.randn(hd, generator=_gen(17 + i)).cuda() for i in range(2))
    pos = torch.randint(0, 1000, (T,), generator=_gen(19)).to(torch.int32).cuda()
    n_slots = 2 * T + 3
    slot = torch.randperm(n_slots, generator=_gen(20))[:T].to(torch.int32)
    slot[::5] = torch.where(torch.arange(T)[::5] % 2 == 0, -1, n_slots).to(torch.int32)
    ks = torch.full((n_slots, nkv * hd + pad), 3.0, dtype=dt, device="cuda")
    vs = torch.full((nkv * hd, n_slots + pad) if columns else (n_slots, nkv * hd + pad), 3.0,
                    dtype=dt, device="cuda")
    ko, vo = ks[:, :nkv * hd], vs[:, :n_slots] if columns else vs[:, :nkv * hd]
    out = ctx.qk_norm_rope(q, k, v, pos=pos, q_gain=qg, k_gain=kg, slot=slot.cuda(), k_out=ko,
                           v_out=vo, v_columns=columns)
    _close_heads(out, *_ref_heads(q, nq, hd, qg, pos, eps, theta), dt)
    live = (slot >= 0) & (slot < n_slots)
    at = slot[live].long()
    ref, mag = _ref_heads(k, nkv, hd, kg, pos, eps, theta)
    _close_heads(ko.cpu()[at], ref[live], mag[live], dt)
    vt = (vo.t() if columns else vo).cpu()
    assert torch.equal(vt[at], v.cpu()[live])
    rest = torch.ones(n_slots, dtype=torch.bool)
    rest[at] = False
    assert torch.all(ko.cpu()[rest] == 3) and torch.all(vt[rest] == 3)
    if pad:
        assert torch.all(ks[:, nkv * hd:] == 3)
        assert torch.all(vs[:, n_slots if columns else nkv * hd:] == 3)


@pytest.mark.parametrize("hd", [64, 128])
def test_qk_consecutive_slots(L, hd):
    """Runs of consecutive slots from any first slot, with holes between the runs."""
    nkv, T = 2, 300
    ctx = _ctx(L, 2, nkv, hd)
    v = _wide(T, nkv * hd, torch.float16, 1, 0)
    for first, hole in ((0, 1000), (8, 37), (3, 64), (61, 5)):
        i = torch.arange(T)
        slot = (first + i + i // hole).to(torch.int32)
        cap = int(slot.max()) + 9
        vo = torch.full((nkv * hd, cap), 3.0, dtype=torch.float16, device="cuda")
        ctx.qk_norm_rope(None, None, v, pos=torch.zeros(T, dtype=torch.int32, device="cuda"),
                         slot=slot.cuda(), v_out=vo, v_columns=True)
        want = torch.full((nkv * hd, cap), 3.0, dtype=torch.float16)
        want[:, slot.long()] = v.cpu().t()
        assert torch.equal(vo.cpu(), want)


def test_qk_parts_and_in_place(L):
    """Any of q, k, v alone; no gains; in place; without slots; the same bits each way."""
    nq, nkv, hd, T = 6, 2, 64, 50
    ctx = _ctx(L, nq, nkv, hd)
    q, k, v = (_wide(T, n * hd, torch.bfloat16, 3, 0) for n in (nq, nkv, nkv))
    pos = torch.arange(T, dtype=torch.int32).cuda()
    qg = torch.rand(hd).cuda()
    ko, vo = torch.empty_like(k), torch.empty_like(v)
    out = ctx.qk_norm_rope(q, k, v, pos=pos, q_gain=qg, k_out=ko, v_out=vo)
    ref, mag = _ref_heads(k, nkv, hd, None, pos, 1e-5, 1e4)
    _close_heads(ko, ref, mag, torch.bfloat16)
    assert torch.equal(vo, v)
    assert torch.equal(ctx.qk_norm_rope(q, pos=pos, q_gain=qg), out)
    k2, v2 = torch.empty_like(k), torch.empty_like(v)
    assert ctx.qk_norm_rope(None, k, None, pos=pos, k_out=k2) is None
    ctx.qk_norm_rope(None, None, v, pos=pos, v_out=v2)
    assert torch.equal(k2, ko) and torch.equal(v2, v)
    q3, k3 = q.clone(), k.clone()
    ctx.qk_norm_rope(q3, k3, pos=pos, q_gain=qg, q_out=q3, k_out=k3)
    assert torch.equal(q3, out) and torch.equal(k3, ko)


@pytest.mark.parametrize("hd", [64, 128])
def test_qk_positions_outside(L, hd):
    nq, nkv, T = 3, 1, 6
    ctx = _ctx(L, nq, nkv, hd, max_seq=100)
    q, k = _wide(T, nq * hd, torch.float16, 1, 0), _wide(T, nkv * hd, torch.float16, 2, 0)
    pos = torch.tensor([0, 99, 100, -1, 2 ** 31 - 1, 5], dtype=torch.int32).cuda()
    ko = torch.empty_like(k)
    out = ctx.qk_norm_rope(q, k, pos=pos, k_out=ko)
    for t, ok in enumerate((True, True, False, False, False, True)):
        for x in (out, ko):
            assert torch.isfinite(x[t]).all() if ok else torch.isnan(x[t]).all()


def test_qk_extremes(L):
    """Zero heads, heads of the type's largest values, NaN and infinity (they stay in their head)."""
    nq, nkv, hd = 4, 4, 64
    ctx = _ctx(L, nq, nkv, hd)
    gain = torch.ones(hd, device="cuda")
    q = torch.randn(1, nq * hd, device="cuda").half()
    q[0, :hd] = 0
    q[0, hd:2 * hd] = 65504
    q[0, 2 * hd + 3] = float("nan")
    pos = torch.tensor([17], dtype=torch.int32, device="cuda")
    out = ctx.qk_norm_rope(q, pos=pos, q_gain=gain).float().view(nq, hd)
    assert torch.all(out[0] == 0) and torch.isnan(out[2]).all()
    assert torch.isfinite(out[1]).all() and torch.isfinite(out[3]).all()
    ref, mag = _ref_heads(q[:, hd:2 * hd], 1, hd, gain, pos, 1e-5, 1e4)
    _close_heads(out[1:2], ref, mag, torch.float16)


# ---------------------------------------------------------------- together, streams, graphs
def _half_layer(ctx, h, gate, W, sW, pos, slot, ks, vs, gains, hd, nq, nkv):
    """Quantise, project, normalise, rotate, write the cache; then the MLP's middle."""
    n = (nq + 2 * nkv) * hd
    hq, hs = ctx.quantize(h)
    qkv = ctx.matmul(hq, hs, W[:n], sW[:-(-n // G)])
    q, k, v = qkv.split((nq * hd, nkv * hd, nkv * hd), 1)
    out = ctx.qk_norm_rope(q, k, v, pos=pos, q_gain=gains[0], k_gain=gains[1], slot=slot, k_out=ks,
                           v_out=vs, v_columns=True)
    mq, ms = ctx.quantize(h, gate=gate)
    return qkv, out, ctx.matmul(mq, ms, W, sW, dtype=torch.float32), (hq, hs, mq, ms)


def _half_layer_inputs(T, nq, nkv, hd, d):
    n = (nq + 2 * nkv) * hd
    W, sW = _codes(n, d, 31, pad=0), _scales(-(-n // G), -(-d // G), 32, pad=0)
    h = torch.randn(T, d, generator=_gen(33)).half().cuda()
    gate = torch.randn(T, d, generator=_gen(34)).half().cuda()
    gains = [torch.rand(hd, generator=_gen(35 + i)).cuda() + 0.5 for i in range(2)]
    pos = torch.arange(T, dtype=torch.int32).cuda()
    ks = torch.zeros(T + 8, nkv * hd, dtype=torch.float16, device="cuda")
    vs = torch.zeros(nkv * hd, T + 8, dtype=torch.float16, device="cuda")
    return h, gate, W, sW, pos, (pos + 8).contiguous(), ks, vs, gains


@pytest.mark.parametrize("T", [1, 37, 300])
def test_together(L, T):
    nq, nkv, hd, d = 4, 2, 128, 1040
    ctx = _ctx(L, nq, nkv, hd)
    h, gate, W, sW, pos, slot, ks, vs, gains = args = _half_layer_inputs(T, nq, nkv, hd, d)
    qkv, out, mlp, (hq, hs, mq, ms) = _half_layer(ctx, *args, hd, nq, nkv)
    _check_codes(hq.float().double().cpu().numpy(), hs.double().cpu().numpy(), h.double().cpu().numpy(), 0.0)
    _check_product(qkv, hq, hs, W, sW)
    _check_product(mlp, mq, ms, W, sW)
    q, k, v = qkv.split((nq * hd, nkv * hd, nkv * hd), 1)
    _close_heads(out, *_ref_heads(q, nq, hd, gains[0], pos, 1e-5, 1e4), torch.float16)
    _close_heads(ks[8:], *_ref_heads(k, nkv, hd, gains[1], pos, 1e-5, 1e4), torch.float16)
    assert torch.equal(vs[:, 8:].t(), v) and torch.all(vs[:, :8] == 0) and torch.all(ks[:8] == 0)


@pytest.mark.parametrize("T", [1, 130])
def test_captured(L, T):
    """A captured run, replayed with new inputs between eager calls of the same operators."""
    nq, nkv, hd, d = 4, 2, 64, 700
    stream = torch.cuda.Stream()
    ctx = L.Context(Shape(nq, nkv, hd), device=0, stream=stream.cuda_stream)
    with torch.cuda.stream(stream):
        args = _half_layer_inputs(T, nq, nkv, hd, d)
        _half_layer(ctx, *args, hd, nq, nkv)
        stream.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            captured = _half_layer(ctx, *args, hd, nq, nkv)
        for i in range(4):
            args[0].copy_(torch.randn(T, d, generator=_gen(50 + i)).half())
            args[6].zero_(), args[7].zero_()
            g.replay()
            got = [t.clone() for t in (captured[0], captured[1], captured[2], args[6], args[7])]
            args[6].zero_(), args[7].zero_()
            eager = _half_layer(ctx, *args, hd, nq, nkv)
            stream.synchronize()
            for a, b in zip(got, (eager[0], eager[1], eager[2], args[6], args[7])):
                assert torch.equal(a, b), i
        # timing cannot be captured
        ctx.set_profiling(1)
        g2 = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g2, stream=stream):
            with pytest.raises(L.LmopError) as ei:
                ctx.quantize(args[0])
        assert ei.value.status == L.LMOP_ERR_STATE
        ctx.set_profiling(0)
        assert torch.equal(ctx.matmul(eager[3][0], eager[3][1], args[2], args[3]), eager[0])


def test_ctx_dropped_in_a_capture(L):
    """A ctx that goes while another's operators are captured leaves the capture whole."""
    stream = torch.cuda.Stream()
    ctx, other = (L.Context(Shape(), device=0, stream=stream.cuda_stream) for _ in range(2))
    with torch.cuda.stream(stream):
        x = torch.randn(9, 300, device="cuda")
        want = [t.clone() for t in ctx.quantize(x)]
        stream.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            got = ctx.quantize(x)
            del other
        for _ in range(3):
            got[0].view(torch.uint8).zero_(), got[1].zero_()
            g.replay()
            stream.synchronize()
            for t, w in zip(got, want):
                assert torch.equal(t.contiguous().view(torch.uint8), w.contiguous().view(torch.uint8))


def test_streams(L):
    """A ctx of another stream than torch's current one refuses; its own stream serves."""
    stream = torch.cuda.Stream()
    ctx = L.Context(Shape(), device=0, stream=stream.cuda_stream)
    x = torch.randn(40, 300, device="cuda")
    torch.cuda.synchronize()
    with pytest.raises(ValueError):
        ctx.quantize(x)
    with torch.cuda.stream(stream):
        q, s = ctx.quantize(x)
    stream.synchronize()
    q0, s0 = _ctx(L).quantize(x)
    assert torch.equal(q.view(torch.uint8), q0.view(torch.uint8)) and torch.equal(s, s0)
    with torch.cuda.stream(stream):
        with pytest.raises(ValueError):  # made for the null stream
            _null = L.Context(Shape(), device=0)
            _null.quantize(x)


def test_two_contexts_at_once(L):
    """Two ctxs on two streams, calls interleaved: each as if alone."""
    streams = [torch.cuda.Stream() for _ in range(2)]
    ctxs = [L.Context(Shape(4, 2, 64), device=0, stream=s.cuda_stream) for s in streams]
    inputs = [_half_layer_inputs(60 + 9 * i, 4, 2, 64, 512) for i in range(2)]
    alone = [_half_layer(_ctx(L, 4, 2, 64), *inputs[i], 64, 4, 2)[2] for i in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i].append(_half_layer(ctxs[i], *inputs[i], 64, 4, 2)[2])
    torch.cuda.synchronize()
    for i in range(2):
        for c in got[i]:
            assert torch.equal(c, alone[i])


def test_two_contexts_without_streams(L):
    """Outputs that are freed at once, so that the two ctxs' calls write the same memory in turn."""
    ctxs = [_ctx(L, 4, 2, 64) for _ in range(2)]
    m, n, k = 512, 4096, 4096
    inputs = [(_codes(m, k, i), _scales(m, k // G, i), _codes(n, k, 9 + i), _scales(n // G, k // G, i))
              for i in range(2)]
    alone = []
    for i in range(2):
        alone.append(ctxs[i].matmul(*inputs[i]).clone())
        torch.cuda.synchronize()
    for _ in range(20):
        ctxs[0].matmul(*inputs[0])
        ctxs[1].matmul(*inputs[1])
        c = ctxs[0].matmul(*inputs[0])
        torch.cuda.synchronize()
        assert torch.equal(c, alone[0])
        del c


def test_profiled(L):
    ctx = _ctx(L)
    ctx.set_profiling(1)
    q, s = ctx.quantize(torch.randn(64, 256, device="cuda"))
    ctx.matmul(q, s, _codes(128, 256, 1), _scales(1, 2, 2))
    st = ctx.kernel_stats()
    assert st["quantize"]["launches"] == 1 and st["matmul_fp8"]["launches"] == 1
    assert st["matmul_fp8"]["flops"] == 2 * 64 * 128 * 256 and st["matmul_fp8"]["ms"] > 0


def test_other_users_keep_their_results(L):
    """Operators between row evaluations on one ctx change nothing there."""
    from synth import make_weights, make_workload
    shape = SHAPES["tiny"]
    ctx = L.Context(shape, device=0, stream=torch.cuda.current_stream().cuda_stream)
    ctx.load_weights(make_weights(shape, seed=3))
    wl = make_workload("filter_tiny", n_rows=12)
    pre = ctx.set_prefix(wl.prefix)
    a, _ = ctx.eval_rows(wl.tokens, wl.offsets, wl.kind, wl.allowed, prefix=pre)
    q, s = ctx.quantize(torch.randn(64, 256, device="cuda"))
    c = ctx.matmul(q, s, _codes(300, 256, 1), _scales(3, 2, 2), dtype=torch.float32)
    b, _ = ctx.eval_rows(wl.tokens, wl.offsets, wl.kind, wl.allowed, prefix=pre)
    assert a.tobytes() == b.tobytes()
    assert torch.equal(c, ctx.matmul(q, s, _codes(300, 256, 1), _scales(3, 2, 2), dtype=torch.float32))


# ---------------------------------------------------------------- the gate at any size
def test_quantize_gate_is_as_exact_at_any_size(ctx):
    """A row of one feature has |y| / 448 as its scale.  x * silu(gate) is known there within
    12 roundings of 2^-24: the exponential (the instruction's 2, its correction 1, what is left
    of the exponent 1), the sum (1), the reciprocal (2), two products (2), the scale's division
    and the product that undoes it here (2), and one more of the last bits of log2 e."""
    x = 2.0 ** 70 * (1 + torch.rand(8001, 1, generator=_gen(1)))
    gate = torch.linspace(-84, 84, 8001).view(-1, 1)
    _, s = ctx.quantize(x.cuda(), gate=gate.cuda())
    z = gate.double()
    y = (x.double() * z * torch.sigmoid(z)).abs().clamp(min=2.0 ** -40)
    off = (s.double().cpu() * 448 / y - 1).abs()
    assert off.max() <= 12 * 2.0 ** -24, off.max() / 2.0 ** -24


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_quantize_gate_extremes(ctx, dtype):
    """Gates whose silu is zero in the type, the largest gates, infinities and NaN."""
    dt = DT[dtype]
    x = torch.tensor([1.0, 2.0 ** 20, 1.0, 2.0 ** -60, 2.0 ** -60, 0.0, 1.0, 1.0, 1.0])
    z = torch.tensor([-100.0, -250.0, -3e38, 1e9, 3e38, 3e38, float("inf"), float("-inf"), float("nan")])
    x, z = x.to(dt).view(-1, 1), z.to(dt).view(-1, 1)
    q, s = ctx.quantize(x.cuda(), gate=z.cuda())
    q, s = q.float().cpu().view(-1), s.double().cpu().view(-1)
    y = (x.double() * z.double() / (1 + (-z.double()).exp())).view(-1)[:6]
    want = y.abs().clamp(min=2.0 ** -40) / 448
    assert torch.all((s[:6] / want - 1).abs() <= 12 * 2.0 ** -24)
    assert torch.equal(q[:6], torch.where(y.abs() >= 2.0 ** -40, 448 * y.sign(), torch.zeros(6).double()).float())
    assert torch.isnan(q[6:]).all() and torch.isnan(s[6:]).all()


# ---------------------------------------------------------------- more threads than one launch has
def test_quantize_more_groups_than_a_launch(ctx):
    """2^29 groups and some (8 threads each: 2^32), which HIP does not launch at a time."""
    n, base = 2 ** 29 + 77, torch.randn(4099, 1, generator=_gen(3)).half().cuda()
    few_q, few_s = ctx.quantize(base)
    q, s = ctx.quantize(base.repeat(n // 4099 + 1, 1)[:n])
    assert torch.equal(s, few_s.repeat(n // 4099 + 1, 1)[:n])
    assert torch.equal(q.view(torch.uint8), few_q.view(torch.uint8).repeat(n // 4099 + 1, 1)[:n])


@pytest.mark.parametrize("m,n,dtype", [(2 ** 30, 16, "f16"), (2 ** 30 - 5, 1, "f32")])
def test_matmul_more_tiles_than_a_launch(ctx, m, n, dtype):
    """2^24 tiles of 256 threads."""
    print("large", m, n, dtype, flush=True)
    k, few = 16, 4099
    a, b = _codes(few, k, 1, pad=0), _codes(n, k, 2, pad=0)
    sa, sb = _scales(few, 1, 3, pad=0), _scales(1, 1, 4, pad=0)
    want = ctx.matmul(a, sa, b, sb, dtype=DT[dtype])
    times = -(-m // few)
    c = ctx.matmul(a.view(torch.uint8).repeat(times, 1)[:m].view(F8), sa.repeat(times, 1)[:m], b, sb,
                   dtype=DT[dtype])
    assert torch.equal(c, want.repeat(times, 1)[:m])


def test_matmul_more_values_than_a_launch(ctx):
    """No features: more than 2^32 results."""
    m, n = 65541, 65536
    a, sa = torch.empty(m, 0, dtype=F8, device="cuda"), torch.empty(m, 0, device="cuda")
    b, sb = torch.empty(n, 0, dtype=F8, device="cuda"), torch.empty(n // G, 0, device="cuda")
    c = torch.full((m, n), 9.0, dtype=torch.float16, device="cuda")
    ctx.matmul(a, sa, b, sb, out=c)
    assert not c.any()


def test_profiled_operators_hold_a_bounded_number_of_events(ctx):
    """Nothing waits for operators: 1024 timed launches are under way at most, later ones counted
    only, and timing goes on when those have ended."""
    m, n, k = 4096, 16384, 4096  # 0.2 ms
    a, b = _codes(m, k, 1, pad=0), _codes(n, k, 2, pad=0)
    sa, sb = _scales(m, k // G, 3), _scales(n // G, k // G, 4)
    c, x = torch.empty(m, n, dtype=torch.float16, device="cuda"), torch.zeros(1, 128, device="cuda")
    out = ctx.quantize(x)
    ctx.set_profiling(1)
    for _ in range(1000):
        ctx.matmul(a, sa, b, sb, out=c)
    for _ in range(600):
        ctx.quantize(x, out=out)
    st = ctx.kernel_stats()
    assert st["matmul_fp8"]["launches"] == 1000 and st["quantize"]["launches"] == 600
    timed = st["matmul_fp8"]["timed"] + st["quantize"]["timed"]
    assert 1024 <= timed < 1600
    for _ in range(5):
        ctx.quantize(x, out=out)
    assert ctx.kernel_stats()["quantize"]["timed"] == st["quantize"]["timed"] + 5
    ctx.set_profiling(0)


# ---------------------------------------------------------------- what the 8-bit instruction cuts off
def _exponents(x):
    """The exponent of E4M3 values (float64): of the leading bit, -6 for subnormal ones."""
    return torch.where(x == 0, -999, torch.frexp(x)[1].clamp(min=-5) - 1)


def _cut_groups(a, b):
    """Of each group of 128 features, in 64 bits: the sums of eights of adjacent products that
    are cut towards zero at 2^-13 of the leading bit of the largest (2 to the sum of its
    exponents); and whether their addition is exact in fp32, in any order: all are multiples
    of one u, and their magnitudes add up to less than 2^24 u."""
    pad = -a.shape[1] % G
    a, b = (torch.nn.functional.pad(x.double(), (0, pad)) for x in (a.float(), b.float()))
    for g in range(a.shape[1] // G):
        A, B = a[:, None, g * G:(g + 1) * G], b[None, :, g * G:(g + 1) * G]
        e = (_exponents(A) + _exponents(B)).unflatten(-1, (16, 8)).amax(-1).clamp(min=-99)
        step = torch.pow(2.0, (e - 13).double())
        eights = ((A * B).unflatten(-1, (16, 8)) / step[..., None]).trunc().sum(-1) * step
        u = torch.where(eights == 0, math.inf, step).amin(-1)
        yield eights.sum(-1), eights.abs().sum(-1) < 2.0 ** 24 * u


def _cut_product(a, sa, b, sb):
    """The fast fp32 result step by step: the cut sums, scaled and added in fp32 group by group."""
    acc, peak, exact = None, 0, True
    for g, (d, fits) in enumerate(_cut_groups(a, b)):
        s = (sa[:, g, None] * sb[torch.arange(b.shape[0], device=b.device) // G, g][None]).double()
        acc = (d * s + (0 if acc is None else acc.double())).float()
        peak = acc.abs() if g == 0 else torch.maximum(peak, acc.abs())
        exact = exact & fits
    return acc, peak, exact


@pytest.mark.parametrize("big", [False, True])
@pytest.mark.parametrize("m,n,k", [(1, 200, 1024), (24, 72, 1100), (70, 130, 4096), (300, 200, 688), (600, 300, 128)])
def test_matmul_fast_cuts_what_it_says(ctx, m, n, k, big):
    """Bits below 2^-13 of the largest of eight products, and nothing more."""
    print("cut", m, n, k, big, flush=True)
    a, b = _codes(m, k, 1), _codes(n, k, 2)
    if big:  # a feature in a hundred ten times as large, quantised to its maximum
        x = torch.randn(m, k, generator=_gen(8)) * torch.where(torch.arange(k) % 97 == 5, 10.0, 1.0)
        a.copy_((x * 11).clamp(-448, 448).to(F8).cuda())
    sa, sb = _scales(m, -(-k // G), 3), _scales(-(-n // G), -(-k // G), 4)
    want, peak, exact = _cut_product(a, sa, b, sb)
    got = ctx.matmul(a, sa, b, sb, dtype=torch.float32, fast=True)
    assert exact.double().mean() > 0.5
    # the fma is done in 64 bits here and rounded twice: for each group, a step of the sum so far
    near = (got - want).abs() <= -(-k // G) * 2.0 ** -23 * peak
    assert near[exact].all()
    assert (got == want)[exact].double().mean() > 0.99  # twice rounded seldom differs
