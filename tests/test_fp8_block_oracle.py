"""The oracle's block-scaled FP8 maps and query/key norms against brute force, and
the host checks of the calls that load them."""
import dataclasses

import numpy as np
import pytest
import torch

from oracle import OracleLM
from oracle.lmop_oracle import (KIND_ENUM, dequant_fp8_block, quantize_rows, rms_norm, round_e4m3)
from paper_2606_31808_amd import lmop as L
from synth import SHAPES, ModelShape, make_weights, quantize_fp8_block
from tests import test_gpu_fp8_block as gpu

TINY = SHAPES["tiny"]
MICRO = ModelShape("micro", 2, 64, 4, 2, 16, 96, 64, 1e4)


def test_round_e4m3_matches_torch():
    y = torch.cat([torch.linspace(-448, 448, 20001, dtype=torch.float64),
                   torch.logspace(-12, 2, 4001, base=2, dtype=torch.float64),
                   torch.tensor([0.0, 2.0 ** -10, 3 * 2.0 ** -10, 17.0, 19.0, -17.0], dtype=torch.float64)])
    y = y.float()
    want = y.to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(round_e4m3(y.double().numpy()), want)


def test_quantize_rows_by_hand():
    x = np.zeros((2, 200))
    x[0, :128] = np.arange(128) - 64.0
    x[0, 128:] = 1e-3
    x[1, 130] = -7.0
    got = quantize_rows(x)
    for r in range(2):
        for g in (slice(0, 128), slice(128, 200)):
            s = max(np.abs(x[r, g]).max(), 2.0 ** -40) / 448
            want = torch.from_numpy((x[r, g] / s).astype(np.float32)).to(torch.float8_e4m3fn).double()
            assert np.allclose(got[r, g], want.numpy() * s, rtol=1e-12, atol=0)
    # a step of E4M3 is an eighth of a power of two: half of it off at most
    assert np.all(np.abs(got - x) <= np.abs(x) / 16 + 1e-12 + 64 / 448 * 2.0 ** -10)


def test_block_weights():
    w = torch.randn(200, 300, generator=torch.Generator().manual_seed(1))
    w[:128, 128:256] = 0
    q, s = quantize_fp8_block(w)
    assert q.shape == (200, 300) and s.shape == (2, 3) and s[0, 1] == 1
    deq = dequant_fp8_block(q.numpy(), s.numpy())
    for i in range(2):
        for j in range(3):
            b = (slice(128 * i, 128 * i + 128), slice(128 * j, 128 * j + 128))
            v = q[b].view(torch.float8_e4m3fn).double().numpy() * float(s[i, j])
            assert np.array_equal(deq[b], v)
            assert np.abs(deq[b] - w[b].double().numpy()).max() <= float(w[b].abs().max()) / 16 + 1e-12


@pytest.mark.parametrize("fmt,norm", [("fp8_block", False), ("fp8_block", True), ("int4_g32", True)])
def test_model_prefix_cached_equals_full_forward(fmt, norm):
    w = make_weights(MICRO, seed=13, fmt=fmt, qk_norm=norm)
    orc = OracleLM(w, MICRO)
    rng = np.random.default_rng(17)
    prefix = rng.integers(0, MICRO.vocab, size=9)
    rows = [rng.integers(0, MICRO.vocab, size=n) for n in (1, 7, 3)]
    res = orc.eval_rows(prefix, rows, KIND_ENUM, np.array([3, 50, 7]), keep_logits=True)
    for r in range(3):
        z = orc.logits(orc.forward_sequence(np.concatenate([prefix, rows[r]]))[-1])[0]
        assert np.allclose(res["logits"][r][0], z, atol=1e-11)


def test_norms_are_taken_per_head_before_the_rotation():
    """Doubling a query projection changes nothing behind its norm; a gain scales it."""
    w = make_weights(MICRO, seed=3, qk_norm=True)
    orc = OracleLM(w, MICRO)
    h = np.random.default_rng(1).normal(size=(5, 64))
    _, _, ws = orc.layer_weights(0)
    pos = np.arange(5)
    q, k, _ = orc._qkv(0, h, ws, pos)
    q2, _, _ = orc._qkv(0, h, {**ws, "wq": 1000 * ws["wq"]}, pos)
    assert np.allclose(q, q2, rtol=1e-3)
    raw = (h @ ws["wk"].T).reshape(5, 2, 16)
    want = rms_norm(raw, w.layers[0].k_norm.numpy(), MICRO.rms_eps)
    assert np.allclose(np.linalg.norm(k, axis=-1), np.linalg.norm(want, axis=-1))


def _expect(status, fn, *a, **k):
    with pytest.raises(L.LmopError) as ei:
        fn(*a, **k)
    assert ei.value.status == status


def test_loading_on_a_host_ctx():
    ctx = L.Context(TINY, device=-1)
    g = torch.ones(TINY.n_layers, TINY.head_dim)
    _expect(L.LMOP_ERR_STATE, ctx.load_qk_norms, g, g)
    w = make_weights(TINY, seed=5, fmt="fp8_block", qk_norm=True)
    ctx.load_weights(w)
    _expect(L.LMOP_ERR_INVALID_ARG, ctx.load_qk_norms, g, None)
    with pytest.raises(ValueError):
        ctx.load_qk_norms(g[:, :32], g)
    # norms change what a prefix's keys are: prefixes are released
    pre = ctx.set_prefix([1, 2, 3])
    ctx.load_qk_norms(g, g)
    _expect(L.LMOP_ERR_INVALID_ARG, ctx.release_prefix, pre)
    ctx.load_qk_norms()
    w.layers[1].q_norm = None
    with pytest.raises(ValueError):
        ctx.load_weights(w)
    bad = make_weights(TINY, seed=5, fmt="fp8_block")
    bad.layers[0] = dataclasses.replace(bad.layers[0], wo=bad.layers[0].w_up)
    _expect(L.LMOP_ERR_INVALID_ARG, ctx.load_weights, bad)
    bad.layers[0] = dataclasses.replace(bad.layers[0], wo=dataclasses.replace(
        bad.layers[1].wo, fmt="int4_g32"))
    with pytest.raises(ValueError):
        ctx.load_weights(bad)


@pytest.mark.parametrize("which,n", [("q_norm", 32), ("k_norm", 128), ("k_norm", 1)])
def test_norms_of_another_length_load_nothing(which, n):
    w = make_weights(TINY, seed=5, fmt="fp8_block", qk_norm=True)
    setattr(w.layers[1], which, torch.ones(n))
    ctx = L.Context(TINY, device=-1)
    with pytest.raises(ValueError):
        ctx.load_weights(w)
    _expect(L.LMOP_ERR_STATE, ctx.load_qk_norms)
    for l in w.layers:
        l.q_norm = l.k_norm = torch.ones(n)
    with pytest.raises(ValueError):
        ctx.load_weights(w)


@pytest.mark.parametrize("rows,dec", [(1, 1), (40, 1), (40, 4)])
def test_plan_covers_block_scaled_passes(rows, dec):
    """The scratch of a plan holds the operand codes and the widest result of a pass."""
    ctx = L.Context(TINY, device=-1)
    ctx.load_weights(make_weights(TINY, seed=5, fmt="fp8_block"))
    n = 20
    kw = dict(kind=L.LMOP_INT, allowed=list(range(10)), eos=11, max_tokens=dec) if dec > 1 else \
        dict(kind=L.LMOP_BOOL, allowed=[3, 4])
    toks = np.arange(rows * n) % TINY.vocab
    pl = ctx.plan_rows(toks, np.arange(rows + 1) * n, no_dedup=True, **kw)
    T = min(rows * n, pl["max_batch_tokens"])
    wide = 256 * -(-TINY.d_ff // 128)
    need = T * (TINY.d_model * 6 + TINY.n_heads * TINY.head_dim * 4 + 2 * wide + 688 + 4 * 6)
    assert pl["scratch_bytes"] >= need
    assert 0 < pl["min_workspace_bytes"] <= pl["scratch_bytes"]


def test_plan_covers_norms_of_the_packed_formats():
    """Their passes read one position for every token: 4 bytes each."""
    ctx = L.Context(TINY, device=-1)
    ctx.load_weights(make_weights(TINY, seed=5))
    args = (np.arange(800) % TINY.vocab, np.arange(41) * 20, L.LMOP_BOOL, [3, 4])
    g = torch.ones(TINY.n_layers, TINY.head_dim)
    plain = ctx.plan_rows(*args, no_dedup=True)
    ctx.load_qk_norms(g, g)
    pl = ctx.plan_rows(*args, no_dedup=True)
    assert pl["scratch_bytes"] == plain["scratch_bytes"] + -(-4 * 800 // 256) * 256
    ctx.load_qk_norms()
    assert ctx.plan_rows(*args, no_dedup=True)["scratch_bytes"] == plain["scratch_bytes"]
    ctx.load_qk_norms(g, g)
    ctx.load_weights(make_weights(TINY, seed=5))
    assert ctx.plan_rows(*args, no_dedup=True)["scratch_bytes"] == plain["scratch_bytes"]


def test_c_named_calls_check_the_norms_shape():
    """The library copies n_layers * head_dim values from each pointer."""
    ctx = L.Context(TINY, device=-1)
    w = make_weights(TINY, seed=5, qk_norm=True)
    for l in w.layers:
        l.q_norm = l.k_norm = torch.ones(TINY.head_dim // 2)
    with pytest.raises(ValueError):
        L.lmop_load_weights(ctx.ctx, w)
    _expect(L.LMOP_ERR_STATE, L.lmop_load_qk_norms, ctx.ctx)  # nothing was loaded
    L.lmop_load_weights(ctx.ctx, make_weights(TINY, seed=5, qk_norm=True))
    g = torch.ones(TINY.n_layers, TINY.head_dim)
    for bad in (g[:1], g[:, :1], g[0], g.view(-1), torch.ones(0, TINY.head_dim)):
        for pair in ((bad, g), (g, bad)):
            with pytest.raises(ValueError):
                L.lmop_load_qk_norms(ctx.ctx, *pair)
    L.lmop_load_qk_norms(ctx.ctx, g.numpy(), g.double())


@pytest.mark.parametrize("d_ff,d,heads,fmt,status", [
    (2 ** 23, 64, 1, L.LMOP_W_FP8_BLOCK, L.LMOP_OK), (2 ** 23 + 16, 64, 1, L.LMOP_W_FP8_BLOCK, L.LMOP_ERR_UNSUPPORTED),
    (64, 2 ** 23 + 64, 1, L.LMOP_W_FP8_BLOCK, L.LMOP_ERR_UNSUPPORTED),
    (64, 64, 2 ** 17 + 1, L.LMOP_W_FP8_BLOCK, L.LMOP_ERR_UNSUPPORTED), (2 ** 24, 64, 1, L.LMOP_W_INT4_G32, L.LMOP_OK)])
def test_rows_of_codes_that_a_tile_cannot_address(d_ff, d, heads, fmt, status):
    """A tile's row offsets are 32 bits: 256 rows of 2^24 bytes would pass them (addresses that
    are not read: a host-only ctx checks the shapes)."""
    shape = dataclasses.replace(TINY, n_layers=1, d_model=d, n_heads=heads, n_kv_heads=1, head_dim=64, d_ff=d_ff)
    ctx = L.Context(shape, device=-1)

    def m(n, k):
        return L.lmop_qmat(4096, 4096, n, k)

    nq, layer = heads * 64, (L.lmop_layer * 1)()
    layer[0] = L.lmop_layer(4096, 4096, m(nq, d), m(64, d), m(64, d), m(d, nq), m(d_ff, d), m(d_ff, d), m(d, d_ff))
    w = L.lmop_weights(4096, 4096, 4096, layer, 1, 0, fmt)
    assert L._lib.lmop_load_weights(ctx.ctx, L.C.byref(w)) == status


class _Wrong(OracleLM):
    """The oracle with one mistake in its queries, keys or values."""

    def __init__(self, what, *a, **k):
        super().__init__(*a, **k)
        self.what, own = what, self.qk_norms
        if what == "gains swapped":
            self.qk_norms = [[b, a] for a, b in own]
        if what == "no key gain":
            self.qk_norms = [[a, np.ones_like(b)] for a, b in own]
        if what == "first layer's gains":
            self.qk_norms = [own[0]] * len(own)
        if what == "no norms":
            self.qk_norms = [[None, None] for _ in own]

    def _qkv(self, l, h, w, pos):
        q, k, v = super()._qkv(l, h, w, pos * 0 if self.what == "no rotation" else pos)
        if self.what == "queries one position on":
            q = super()._qkv(l, h, w, pos + 1)[0]
        if self.what == "keys one slot on":
            k = np.roll(k, 1, 0)
        if self.what == "values one slot on":
            v = np.roll(v, 1, 0)
        return q, k, v


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("sizes", gpu.TELLING, ids=["hd64", "hd128", "tiny"])
def test_mistakes_in_queries_and_keys_are_seen(sizes, norm):
    """What the GPU test of queries and keys allows, each of these mistakes exceeds by half."""
    t = gpu.Telling(sizes, norm)
    wrong = ["no rotation", "queries one position on", "keys one slot on", "values one slot on"]
    if norm:
        wrong += ["gains swapped", "no key gain", "first layer's gains", "no norms"]
    for what in wrong:
        off = t.off(t.logits(_Wrong(what, t.w, t.shape)))
        print(what, f"{off:.3f}, bound {t.bound:.3f}")
        assert off > 1.5 * t.bound, what
