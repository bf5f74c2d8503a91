"""The paged cache, attention over it and over a shared prefix, and the choice of blocks, against
plain implementations in 64 bits.

Tolerances.  A rounding to a type is off by at most half a step: eps / 2 relative.  A sum of N fp32
terms is off by at most N * 2^-23 of the sum of their magnitudes, whatever its order.

Attention: out = sum w_i v_i with w_i = p_i / sum p.  A score is a sum of head_dim exact products
(head_dim * 2^-23 of the sum of their magnitudes), scaled by a rounded constant and brought to the
reference (another four roundings of 2^-24, of the score and of the reference, which is a score); the exponential is good to
2^-22; p is rounded to the tokens' type (fp16: below 2^-14, in steps of 2^-24; the largest p is at
least 1, as the reference never exceeds the largest score).  Each acts on the numerator and
on the divisor.  The two sums have N terms, and are rescaled together."""
import ctypes as C
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"f16": torch.float16, "bf16": torch.bfloat16}
E4M3 = torch.float8_e4m3fn
NAN = float("nan")


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


def _ctx(L, nq=4, nkv=2, hd=64, max_seq=4096, theta=1e4):
    return L.Context(Shape(nq, nkv, hd, theta=theta), device=0, stream=torch.cuda.current_stream().cuda_stream,
                     max_seq=max_seq)


def _gen(seed):
    return torch.Generator().manual_seed(seed)


# ---------------------------------------------------------------- batches and caches
class Batch:
    """Sequences of new[i] tokens that make length[i] keys; pages in a mixed order, the rest of the pool and
    of the pages NaN."""

    def __init__(self, nq, nkv, hd, dtype, cache, page, new, length, prefix=0, seed=0, lead=0, tail=0, spare=1,
                 q_size=2.0):
        g = _gen(seed)
        self.nq, self.nkv, self.hd, self.page, self.dt = nq, nkv, hd, page, DT[dtype]
        self.cache_type, self.new, self.len, self.prefix = cache, new, length, prefix
        used = [-(-n // page) for n in length]
        shared = -(-prefix // page)
        pool = sum(used) + shared + 2
        order = torch.randperm(pool, generator=g)
        self.prefix_pages = order[:shared].to(torch.int32)
        wide = max(used + [1]) + spare
        table = torch.full((len(new), wide), -7, dtype=torch.int32)
        at = shared
        for i, u in enumerate(used):
            table[i, :u] = order[at:at + u]
            at += u
        self.table = table
        self.start = torch.tensor([lead + sum(new[:i]) for i in range(len(new) + 1)], dtype=torch.int32)
        self.tokens = lead + sum(new) + tail
        self.lead = lead
        shape = (pool, nkv, page, hd)
        live = torch.zeros(pool, page, dtype=torch.bool)  # slots that hold keys
        for pages, n in [(self.prefix_pages, prefix)] + [(table[i, :u], n) for i, (u, n) in enumerate(zip(used, length))]:
            for b, pg in enumerate(pages):
                live[int(pg), :max(0, min(page, n - b * page))] = True
        self.live = live
        k, v = torch.randn(shape, generator=g), torch.randn(shape, generator=g)
        if cache == "e4m3":
            self.k8, self.v8 = ((x * 64).clamp(-448, 448).to(E4M3).view(torch.uint8) for x in (k, v))
            self.ke, self.ve = (torch.randint(118, 123, shape[:3], generator=g, dtype=torch.uint8) for _ in range(2))
            dead = ~live[:, None, :].expand(shape[:3])
            for x in (self.k8, self.v8):
                x[dead] = 0x7F
        else:
            self.k16, self.v16 = k.to(self.dt), v.to(self.dt)
            dead = ~live[:, None, :].expand(shape[:3])
            self.k16[dead] = NAN
            self.v16[dead] = float("inf")
        self.q = (torch.randn(self.tokens, nq * hd, generator=g) * q_size).to(self.dt)

    def cache(self, L, mean=None):
        if self.cache_type == "e4m3":
            return L.PagedCache(self.k8.view(E4M3).cuda(), self.v8.view(E4M3).cuda(), self.ke.cuda(), self.ve.cuda(),
                                k_mean=mean)
        return L.PagedCache(self.k16.cuda(), self.v16.cuda(), k_mean=mean)

    def values(self, store):
        """The whole pool in 64 bits."""
        if self.cache_type == "e4m3":
            code, e = (self.k8, self.ke) if store == "k" else (self.v8, self.ve)
            return code.view(E4M3).double() * torch.pow(2.0, e.double() - 127).unsqueeze(-1)
        return (self.k16 if store == "k" else self.v16).double()

    def keys_of(self, store, i, pool=None):
        """Sequence i's keys or values (None: the prefix's) [n, nkv, hd]."""
        x = self.values(store) if pool is None else pool
        pages, n = (self.prefix_pages, self.prefix) if i is None else (self.table[i], self.len[i])
        pages = pages[:-(-n // self.page)].long()
        return x[pages].transpose(1, 2).reshape(-1, self.nkv, self.hd)[:n]

    def args(self, L, starts=None, **more):
        starts = (max(self.new) != 1 or min(self.new) != 1 or self.lead or self.tokens != sum(self.new)) \
            if starts is None else starts
        return dict(table=self.table.cuda(), length=torch.tensor(self.len, dtype=torch.int32).cuda(),
                    start=self.start.cuda() if starts else None, **more)

    def attend(self, ctx, L, cache=None, **more):
        a = self.args(L, max_tokens=max(max(self.new), 1), max_length=max(self.len))
        if self.prefix:
            a.update(prefix=self.prefix_pages.cuda(), prefix_length=self.prefix)
        return ctx.attend(self.cache(L) if cache is None else cache, self.q.cuda(), **{**a, **more})


def _reference(b, blocks=None, scale=None):
    """(out, lse, tolerance) in 64 bits; NaN where no sequence has the token."""
    nq, nkv, hd = b.nq, b.nkv, b.hd
    scale = hd ** -0.5 if scale is None else scale
    eps = torch.finfo(b.dt).eps
    out = torch.full((b.tokens, nq, hd), NAN, dtype=torch.float64)
    lse = torch.full((b.tokens, nq), NAN, dtype=torch.float64)
    tol, tol_lse = torch.zeros_like(out), torch.zeros_like(lse)
    kp, vp = b.values("k"), b.values("v")
    q = b.q.double().view(b.tokens, nq, hd)
    pre = b.keys_of("k", None, kp), b.keys_of("v", None, vp)
    for i, (n, m) in enumerate(zip(b.new, b.len)):
        if n == 0:
            continue
        k, v = (torch.cat((pre[j], b.keys_of(s, i, pool))) for j, (s, pool) in enumerate((("k", kp), ("v", vp))))
        here = b.lead + sum(b.new[:i])
        index = torch.arange(k.shape[0]) - b.prefix  # of an own key
        kh, vh = k.transpose(0, 1).contiguous(), v.transpose(0, 1).contiguous()  # [nkv][keys][hd]
        for j in range(n):
            t = here + j
            seen = (index <= m - n + j).expand(nkv, -1)
            if blocks is not None:
                seen = seen & (index[None, :, None] // b.page == blocks[t][:, None]).any(-1)
            seen = seen[:, None]
            # what is not seen may hold anything
            ks = torch.where(seen[..., None], kh[:, None], 0.0)[:, 0]
            vs = torch.where(seen[..., None], vh[:, None], 0.0)[:, 0]
            qh = q[t].view(nkv, -1, hd)
            z = torch.where(seen, torch.matmul(qh, ks.transpose(1, 2)) * scale, -math.inf)
            mag = torch.matmul(qh.abs(), ks.abs().transpose(1, 2)).amax(-1) if k.shape[0] else torch.zeros(nkv, nq // nkv)
            top = z.amax(-1, keepdim=True) if k.shape[0] else torch.full((nkv, nq // nkv, 1), -math.inf)
            none = torch.isinf(top)
            w = torch.where(none, 0.0, torch.exp(z - torch.where(none, 0.0, top)))
            total = w.sum(-1, keepdim=True)
            total = torch.where(none, 1.0, total)
            out[t] = (torch.matmul(w, vs) / total).view(nq, hd)
            lse[t] = torch.where(none, -math.inf, top + total.log()).view(nq)
            most = torch.where(seen, z.abs(), 0.0).amax(-1, keepdim=True) if k.shape[0] else torch.zeros_like(top)
            e_score = hd * 2.0 ** -23 * mag[..., None] * scale + 4 * most * 2.0 ** -23 + 2.0 ** -21
            size = torch.matmul(w, vs.abs()) / total
            N = seen.sum(-1, keepdim=True).double()
            tt = size * (2 * (eps / 2 + e_score) + 2 * (N + 64) * 2.0 ** -23)
            tl = e_score + eps / 2 + (N + 64) * 2.0 ** -23 + lse[t].view(nkv, -1, 1).abs() * 2.0 ** -22
            if b.dt == torch.float16:
                tt = tt + 2 * 2.0 ** -25 * (vs.abs().sum(1, keepdim=True) + N * size) + 2.0 ** -25
                tl = tl + N * 2.0 ** -25
            tol[t], tol_lse[t] = tt.reshape(nq, hd), tl.reshape(nq)
    tol = tol + eps / 2 * (out.abs() + tol)
    return out.view(b.tokens, -1), lse, tol.view(b.tokens, -1), tol_lse


def _check(b, got, lse, ref):
    out, want_lse, tol, tol_lse = ref
    live = ~torch.isnan(want_lse[:, 0])
    d = (got.double().cpu() - out).abs()[live]
    assert torch.isfinite(d).all()
    assert torch.all(d <= tol[live]), f"off by {(d / tol[live].clamp(min=1e-30)).max():.3g} of the tolerance"
    if lse is not None:
        g = lse.double().cpu()[live]
        w = want_lse[live]
        none = torch.isinf(w)
        assert torch.equal(torch.isinf(g) & (g < 0), none)
        d = (g - w).abs()[~none]
        assert torch.all(d <= tol_lse[live][~none]), f"lse off by {d.max():.3g}"
    return live


def _run(L, b, blocks=None, scale=None, **more):
    ctx = _ctx(L, b.nq, b.nkv, b.hd)
    out = torch.full((b.tokens, b.nq * b.hd), 7.0, dtype=b.dt, device="cuda")
    lse = torch.full((b.tokens, b.nq), 7.0, device="cuda")
    if blocks is not None:
        more["blocks"] = blocks.cuda()
    b.attend(ctx, L, out=out, lse=lse, scale=scale or 0.0, **more)
    live = _check(b, out, lse, _reference(b, blocks, scale))
    assert torch.all(out[~live] == 7) and torch.all(lse[~live] == 7)
    return out, lse


LAYOUTS = [("f16", "f16", 64), ("bf16", "bf16", 128), ("f16", "f16", 128), ("bf16", "bf16", 64), ("f16", "e4m3", 128),
           ("bf16", "e4m3", 64), ("bf16", "e4m3", 128), ("f16", "e4m3", 64)]


# ---------------------------------------------------------------- attention: single tokens
SINGLE = [
    (4, 2, 16, [1], 0), (4, 2, 16, [15, 16, 17, 0, 1, 33], 0), (8, 2, 64, [63, 64, 65, 200], 0),
    (3, 1, 32, [5, 100, 31], 45), (8, 1, 16, [300, 1, 77], 1), (7, 1, 128, [129, 500], 130),
    (2, 2, 256, [256, 257, 2], 255), (4, 4, 16, [40, 7], 64), (17, 1, 16, [50, 9], 20), (40, 2, 32, [70], 0)]


@pytest.mark.parametrize("dtype,cache,hd", LAYOUTS)
@pytest.mark.parametrize("nq,nkv,page,length,prefix", SINGLE)
def test_attend_single_tokens(L, dtype, cache, hd, nq, nkv, page, length, prefix):
    print("single", dtype, cache, hd, nq, nkv, page, length, prefix, flush=True)
    _run(L, Batch(nq, nkv, hd, dtype, cache, page, [1] * len(length), length, prefix, seed=len(length)))


LONG = [(4, 1, 16, [9001, 700], 0), (8, 2, 64, [5000], 0), (4, 2, 32, [3], 4100), (2, 1, 64, [30] * 3, 3001)]
# many sequences: a wave each, or four
MANY = [(8, 8, 16, [i % 70 for i in range(300)], 0), (16, 8, 32, [i % 90 for i in range(260)], 200),
        (4, 2, 16, [6 * i for i in range(100)], 0), (4, 2, 16, [3 * i for i in range(100)], 2100),
        (128, 128, 16, [i for i in range(16)], 200), (4, 2, 64, [5 * i for i in range(16)], 12600)]


@pytest.mark.parametrize("dtype,cache,hd", [("f16", "f16", 128), ("bf16", "bf16", 64), ("bf16", "e4m3", 128)])
@pytest.mark.parametrize("nq,nkv,page,length,prefix", MANY)
def test_attend_many_sequences(L, dtype, cache, hd, nq, nkv, page, length, prefix):
    print("many", dtype, cache, hd, nq, nkv, page, len(length), prefix, flush=True)
    _run(L, Batch(nq, nkv, hd, dtype, cache, page, [1] * len(length), length, prefix, seed=len(length)))


@pytest.mark.parametrize("dtype,cache,hd", LAYOUTS)
@pytest.mark.parametrize("nq,nkv,page,length,prefix", LONG)
def test_attend_long_axis_is_split_and_joined(L, dtype, cache, hd, nq, nkv, page, length, prefix):
    print("split", dtype, cache, hd, nq, nkv, page, length, prefix, flush=True)
    _run(L, Batch(nq, nkv, hd, dtype, cache, page, [1] * len(length), length, prefix, seed=3))


# ---------------------------------------------------------------- attention: several tokens
SEVERAL = [
    (4, 2, 16, [2, 1, 3], [2, 17, 40], 0),        # few vectors, causal
    (4, 1, 32, [4, 2, 0, 1], [4, 33, 9, 1], 37),  # few vectors behind a prefix; a sequence without tokens
    (2, 2, 64, [16], [90], 0),
    (4, 2, 16, [33, 9, 70], [33, 30, 200], 0),    # tiles
    (8, 2, 64, [64, 1, 31, 90], [64, 65, 31, 90], 100),
    (3, 1, 128, [43], [170], 5),
    (4, 4, 32, [129, 127], [129, 300], 64),
    (16, 1, 16, [9, 20], [12, 20], 0),
    (40, 2, 64, [7], [66], 10),
    (2, 1, 32, [70], [3000], 0)]                  # tiles, their keys split


@pytest.mark.parametrize("dtype,cache,hd", LAYOUTS)
@pytest.mark.parametrize("nq,nkv,page,new,length,prefix", SEVERAL)
def test_attend_several_tokens(L, dtype, cache, hd, nq, nkv, page, new, length, prefix):
    print("several", dtype, cache, hd, nq, nkv, page, new, length, prefix, flush=True)
    _run(L, Batch(nq, nkv, hd, dtype, cache, page, new, length, prefix, seed=sum(new)))


# ---------------------------------------------------------------- attention: what is masked
@pytest.mark.parametrize("dtype,cache,hd", LAYOUTS)
@pytest.mark.parametrize("nq,nkv,new", [(2, 2, [9, 3]), (4, 2, [60, 41]), (1, 1, [16, 2])])
@pytest.mark.parametrize("bad", [NAN, float("inf"), float("-inf")])
def test_attend_unseen_keys_may_hold_anything(L, dtype, cache, hd, nq, nkv, new, bad):
    """A token's key and value are seen by it and later ones only."""
    print("unseen", dtype, cache, hd, nq, nkv, new, bad, flush=True)
    b = Batch(nq, nkv, hd, dtype, cache, 16, new, [n + 5 for n in new], prefix=20, seed=1)
    ctx = _ctx(L, nq, nkv, hd)
    clean = b.attend(ctx, L)
    last = b.len[0] - 2
    page, slot = int(b.table[0, last // 16]), last % 16
    if cache == "e4m3":
        b.k8[page, :, slot], b.v8[page, :, slot] = 0x7F, 0xFF
    else:
        b.k16[page, :, slot], b.v16[page, :, slot] = bad, bad
    got = b.attend(ctx, L)
    other = torch.ones(b.tokens, dtype=torch.bool)
    other[new[0] - 2:new[0]] = False
    assert torch.equal(got[other.cuda()], clean[other.cuda()])
    assert torch.isnan(got[new[0] - 2:new[0]]).all()
    # a value alone
    if cache != "e4m3":
        b.k16[page, :, slot] = 0.25
        got = b.attend(ctx, L)
        assert torch.equal(got[other.cuda()], clean[other.cuda()])
        assert not torch.isfinite(got[new[0] - 2:new[0]]).any()


@pytest.mark.parametrize("dtype,cache,hd", LAYOUTS[:6])
@pytest.mark.parametrize("new,length", [([1, 1, 1], [0, 20, 0]), ([3, 5], [1, 0]), ([40, 60], [10, 0])])
def test_attend_tokens_that_see_nothing(L, dtype, cache, hd, new, length):
    print("nothing", dtype, cache, hd, new, length, flush=True)
    out, lse = _run(L, Batch(4, 2, hd, dtype, cache, 16, new, length, seed=5))
    assert torch.all(out[0 if length[0] == 0 else 0] == 0) or length[0] > 0
    assert torch.all(out[-1] == 0) and torch.all(torch.isinf(lse[-1]))


@pytest.mark.parametrize("cache", ["f16", "e4m3"])
@pytest.mark.parametrize("new,prefix", [([1, 1, 1], 0), ([1, 1, 1], 70), ([1, 1, 1], 70000), ([5, 3, 4], 70), ([40, 50, 60], 0),
                                        ([40, 50, 60], 70)])
def test_attend_pages_and_lengths_that_do_not_fit(L, cache, new, prefix):
    """Each makes its own tokens' results NaN and leaves the others'."""
    print("misfit", cache, new, prefix, flush=True)
    b = Batch(4, 2, 64, "f16", cache, 16, new, [90, 80, 70], prefix, seed=2)
    ctx = _ctx(L, 4, 2, 64)
    clean = b.attend(ctx, L)
    seq = torch.repeat_interleave(torch.arange(3), torch.tensor(new)).cuda()
    args = b.args(L)
    for bad in (-1, 10 ** 6, b.table.max().item() + 10 ** 9):
        table = args["table"].clone()
        table[1, 1] = bad
        got = b.attend(ctx, L, table=table)
        sees = torch.tensor([seq[t] == 1 and (b.len[1] - new[1] + t - new[0]) >= 16 for t in range(b.tokens)]).cuda()
        assert torch.isnan(got[sees]).all() and torch.equal(got[~sees], clean[~sees])
    for n in (-1, -2 ** 31, 91, 2 ** 31 - 1):
        length = args["length"].clone()
        length[1] = n
        got = b.attend(ctx, L, length=length)
        assert torch.isnan(got[seq == 1]).all() and torch.equal(got[seq != 1], clean[seq != 1])
    if prefix:
        pages = b.prefix_pages.cuda()
        pages[-1] = -5
        assert torch.isnan(b.attend(ctx, L, prefix=pages)).all()
    if max(new) > 1:
        got = b.attend(ctx, L, max_tokens=sorted(new)[1])
        big = seq == new.index(max(new))
        assert torch.isnan(got[big]).all()
        # (the others' sums may be divided otherwise)
        assert torch.allclose(got[~big].float(), clean[~big].float(), atol=4e-3)


def test_attend_scores_far_apart(L):
    """The reference moves in steps; scores that leap, fall, and are all large."""
    for dtype in ("f16", "bf16"):
        b = Batch(4, 2, 64, dtype, dtype, 16, [1, 40], [400, 300], seed=3)
        ramp = torch.linspace(-30, 30, b.k16.shape[0])[:, None, None, None]
        for scale in (ramp, -ramp, torch.full_like(ramp, 40.0), ramp.abs()):
            c = Batch(4, 2, 64, dtype, dtype, 16, [1, 40], [400, 300], seed=3)
            c.k16 = (b.k16.float() * scale).to(b.dt)
            _run(L, c)
            _run(L, c, scale=0.01)


def test_attend_a_dominant_key_is_its_value(L):
    """One weight is all: the result is that value, to the bit (the divisor is the sum of rounded weights)."""
    for dtype in ("f16", "bf16"):
        for new in ([1, 1], [30, 40]):
            b = Batch(4, 2, 128, dtype, dtype, 64, new, [300, 200], seed=4)
            b.q[:] = 1.0
            b.k16[b.live[:, None, :].expand(b.k16.shape[:3])] = 0.25
            page = int(b.table[0, 0])
            b.k16[page, :, 7] = 60.0
            out = b.attend(_ctx(L, 4, 2, 128), L).view(-1, 4, 128)
            assert torch.equal(out[:new[0]].cpu(), b.v16[page, :, 7].repeat_interleave(2, 0).expand(new[0], 4, 128))


# ---------------------------------------------------------------- strides, streams, graphs
@pytest.mark.parametrize("dtype,cache,hd", LAYOUTS[:6])
def test_attend_strides_and_rows_of_no_sequence(L, dtype, cache, hd):
    print("strides", dtype, cache, hd, flush=True)
    for new, prefix in (([1, 2, 1], 0), ([1, 2, 1], 33), ([1, 2, 1], 70000), ([30, 50], 33)):
        b = Batch(4, 2, hd, dtype, cache, 16, new, [60, 70, 80][:len(new)], prefix, seed=6, lead=3, tail=5)
        _run(L, b)
        ctx = _ctx(L, 4, 2, hd)
        want = b.attend(ctx, L, out=torch.zeros(b.tokens, 4 * hd, dtype=b.dt, device="cuda"))
        wide = torch.full((b.tokens, 4 * hd + 11), 3.0, dtype=b.dt, device="cuda")
        q = torch.full((b.tokens, 4 * hd + 7), NAN, dtype=b.dt, device="cuda")
        q[:, 3:3 + 4 * hd] = b.q.cuda()
        table = torch.full((len(new), b.table.shape[1] + 3), -9, dtype=torch.int32, device="cuda")
        table[:, 1:-2] = b.table.cuda()
        a = b.args(L, max_tokens=max(new), max_length=max(b.len))
        a["table"] = table[:, 1:-2]
        if prefix:
            a.update(prefix=b.prefix_pages.cuda(), prefix_length=prefix)
        ctx.attend(b.cache(L), q[:, 3:3 + 4 * hd], out=wide[:, 5:5 + 4 * hd], **a)
        live = slice(3, b.tokens - 5)
        assert torch.equal(wide[live, 5:5 + 4 * hd], want[live])
        assert torch.all(wide[:, :5] == 3) and torch.all(wide[:, 5 + 4 * hd:] == 3)
        assert torch.all(wide[:3] == 3) and torch.all(wide[-5:] == 3)


def test_attend_pages_apart(L):
    """Keys and values interleaved in one tensor."""
    b = Batch(4, 2, 64, "f16", "f16", 16, [1, 7], [40, 50], seed=6)
    both = torch.full((b.k16.shape[0], 2, *b.k16.shape[1:]), NAN, dtype=torch.float16)
    both[:, 0], both[:, 1] = b.k16, b.v16
    both = both.cuda()
    ctx = _ctx(L, 4, 2, 64)
    assert torch.equal(b.attend(ctx, L, cache=L.PagedCache(both[:, 0], both[:, 1])), b.attend(ctx, L))


# ---------------------------------------------------------------- appending
def _rotated(x, pos, hd, theta):
    """x [tokens][heads][hd] in 64 bits, rotated; and the sum of magnitudes of each result's products."""
    half = hd // 2
    angle = pos.double()[:, None, None] * theta ** (-2.0 * torch.arange(half, dtype=torch.float64) / hd)
    x1, x2 = x[..., :half], x[..., half:]
    c, s = angle.cos(), angle.sin()
    return (torch.cat((x1 * c - x2 * s, x1 * s + x2 * c), -1),
            torch.cat(((x1 * c).abs() + (x2 * s).abs(), (x1 * s).abs() + (x2 * c).abs()), -1))


def _check_stored(b, cache_type, dt, store, exp, y, mag, page, slot):
    """Heads y [n][nkv][hd] (64 bits, known within 4 * 2^-24 of mag) in their places."""
    off = 4 * 2.0 ** -24 * mag
    if cache_type != "e4m3":
        got = store[page, :, slot].double()
        eps = torch.finfo(dt).eps
        sub = 2.0 ** -25 if dt == torch.float16 else 0
        assert torch.all((got - y).abs() <= off + eps / 2 * (y.abs() + off) + sub)
        return
    if dt == torch.float16:
        y = y.clamp(-61440, 61440)
    e = exp[page, :, slot].double() - 127
    top = y.abs().amax(-1)
    near = 1 + 2.0 ** -20
    assert torch.all((top <= 448 * torch.pow(2.0, e) * near) | (top == 0))
    assert torch.all((top * near > 448 * torch.pow(2.0, e - 1)) | (e == -126))
    v = y * torch.pow(2.0, -e).unsqueeze(-1)
    got = store[page, :, slot].view(E4M3).double()
    step = torch.pow(2.0, torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
    assert torch.all((got - v).abs() <= step / 2 + off * torch.pow(2.0, -e).unsqueeze(-1) + 1e-12)


def _append(L, nq, nkv, hd, dtype, cache, page, new, length, first=0, means=True, rotate=True, seed=0, lead=0, tail=0,
            size=1.0, with_q=True, max_seq=4096):
    """Appends to a cache that holds other tokens already, and checks every byte of it."""
    b = Batch(nq, nkv, hd, dtype, cache, page, new, length, seed=seed, lead=lead, tail=tail)
    g = _gen(seed + 1)
    qkv = (torch.randn(b.tokens, (nq + 2 * nkv) * hd, generator=g) * size).to(b.dt)
    dev = qkv.cuda()
    q, k, v = dev.split((nq * hd, nkv * hd, nkv * hd), 1)
    mean = torch.full((b.table.max() + 5, nkv, hd), 9.0, dtype=b.dt)[:len(b.live)].cuda() if means else None
    if means and len(mean) < len(b.live):
        mean = torch.full((len(b.live), nkv, hd), 9.0, dtype=b.dt, device="cuda")
    c = b.cache(L, mean)
    before = [t.clone().cpu() for t in (c.k, c.v)]
    ctx = _ctx(L, nq, nkv, hd, max_seq=max_seq)
    out = ctx.cache_append(c, k, v, **b.args(L), first=first, rotate=rotate, q=q if with_q else None)
    x = qkv.double().view(b.tokens, nq + 2 * nkv, hd)
    written = torch.zeros(before[0].shape[0], page, dtype=torch.bool)
    kc, vc = c.k.cpu(), c.v.cpu()
    ke, ve = (c.k_exp.cpu(), c.v_exp.cpu()) if cache == "e4m3" else (None, None)
    tok, pg, sl, pos = [], [], [], []
    for i, (n, m) in enumerate(zip(new, length)):
        for j in range(n):
            idx = m - n + j
            if idx < 0:
                continue
            tok.append(lead + sum(new[:i]) + j)
            pg.append(int(b.table[i, idx // page]))
            sl.append(idx % page)
            pos.append(first + idx)
    tok, pg, sl, pos = (torch.tensor(a, dtype=torch.long) for a in (tok, pg, sl, pos))
    written[pg, sl] = True
    turned, mag = _rotated(x[tok][:, :nq + nkv], pos, hd, 1e4) if rotate else (x[tok][:, :nq + nkv],) * 2
    mag = mag.abs() if rotate else torch.zeros_like(mag)
    bits = lambda t: t.view(torch.uint8) if t.dtype == E4M3 else t
    _check_stored(b, cache, b.dt, bits(kc), ke, turned[:, nq:], mag[:, nq:], pg, sl)
    vv = x[tok][:, nq + nkv:]
    _check_stored(b, cache, b.dt, bits(vc), ve, vv, torch.zeros_like(vv), pg, sl)
    for now, old in zip((kc, vc), before):
        w = written[:, None, :].expand(now.shape[:3])
        same = now.view(torch.uint8)[~w] == old.view(torch.uint8)[~w]
        assert same.all()
    if with_q:
        got = out.double().cpu().view(b.tokens, nq, hd)[tok]
        tol = 4 * 2.0 ** -24 * mag[:, :nq]
        eps = torch.finfo(b.dt).eps
        assert torch.all((got - turned[:, :nq]).abs() <= tol + eps / 2 * (turned[:, :nq].abs() + tol) + 2.0 ** -25)
    if means:
        full = {int(p) for p, s in zip(pg, sl) if s == page - 1}
        mean = mean.cpu()
        kept = kc.double() if cache != "e4m3" else kc.double() * torch.pow(2.0, ke.double() - 127).unsqueeze(-1)
        for p in range(len(mean)):
            if p in full:
                want = kept[p].mean(1)
                assert torch.all((mean[p].double() - want).abs()
                                 <= torch.finfo(b.dt).eps / 2 * want.abs() * (1 + 1e-6) + 2.0 ** -25)
            else:
                assert torch.all(mean[p] == 9)
    return c, out


@pytest.mark.parametrize("dtype,cache,hd", LAYOUTS)
@pytest.mark.parametrize("nq,nkv,page,new,length", [
    (4, 2, 16, [1], [1]), (4, 2, 16, [1, 1, 1], [16, 17, 40]), (8, 1, 64, [1, 1], [64, 128]),
    (3, 3, 32, [5, 0, 40, 33], [5, 7, 72, 64]), (14, 2, 16, [100], [100]), (4, 4, 128, [130, 126], [256, 128]),
    (2, 1, 256, [300], [512]), (32, 8, 64, [200, 60], [200, 64]), (4, 2, 16, [3, 2], [1, 2])])
def test_append(L, dtype, cache, hd, nq, nkv, page, new, length):
    print("append", dtype, cache, hd, nq, nkv, page, new, length, flush=True)
    _append(L, nq, nkv, hd, dtype, cache, page, new, length, first=37, seed=sum(new))


@pytest.mark.parametrize("dtype,cache,hd", LAYOUTS[:6])
def test_append_forms(L, dtype, cache, hd):
    """Without means, rotation or queries; rows of no sequence; many sequences; tiny and large values."""
    print("forms", dtype, cache, hd, flush=True)
    _append(L, 4, 2, hd, dtype, cache, 16, [20, 3], [30, 3], means=False)
    _append(L, 4, 2, hd, dtype, cache, 16, [20, 3], [30, 3], rotate=False)
    _append(L, 4, 2, hd, dtype, cache, 16, [20, 3], [30, 3], with_q=False, lead=2, tail=3)
    _append(L, 4, 2, hd, dtype, cache, 16, [i % 7 for i in range(700)], [i % 7 + i % 33 for i in range(700)])
    _append(L, 4, 2, hd, dtype, cache, 64, [1] * 300, [i % 90 + 1 for i in range(300)], first=3000)
    _append(L, 4, 2, hd, dtype, cache, 16, [40], [40], size=1e-4)
    _append(L, 4, 2, hd, dtype, cache, 16, [40], [40], size=3e3)


# ---------------------------------------------------------------- choosing blocks
def _choose(b, mean, n_blocks):
    """The definition, one token at a time."""
    nkv, G = b.nkv, b.nq // b.nkv
    q = b.q.double().view(b.tokens, nkv, G, b.hd).sum(2)
    out = torch.full((b.tokens, nkv, n_blocks), 7, dtype=torch.int32)
    for i, (n, m) in enumerate(zip(b.new, b.len)):
        for j in range(n):
            t, idx = b.lead + sum(b.new[:i]) + j, m - n + j
            out[t] = -1
            if idx < 0:
                continue
            mine = idx // b.page
            for h in range(nkv):
                # (sums of exact products, exact in any order but for infinities and NaN)
                z = (q[t, h] * mean[b.table[i, :mine].long(), h].double()).sum(-1)
                z = torch.where(z.isnan(), -math.inf, z)
                best = torch.argsort(-z, stable=True)[:n_blocks - 1].tolist()  # of equal ones the first
                ids = sorted(best) + [mine]
                out[t, h, :len(ids)] = torch.tensor(ids, dtype=torch.int32)
    return out


@pytest.mark.parametrize("dtype,hd", [("f16", 64), ("f16", 128), ("bf16", 64), ("bf16", 128)])
@pytest.mark.parametrize("nq,nkv,page,new,length,n_blocks", [
    (4, 2, 16, [1, 1, 1], [5, 100, 700], 4), (8, 1, 64, [1], [4000], 16), (3, 3, 16, [5, 0, 20], [5, 30, 400], 3),
    (2, 2, 16, [2], [2100], 1), (4, 2, 32, [3], [500], 1000), (4, 1, 16, [4, 3], [2, 64], 2),
    (14, 2, 16, [1], [9000], 33), (4, 2, 16, [40, 17], [600, 333], 8), (6, 2, 16, [9], [24000], 5),
    (2, 1, 16, [5], [70000], 3),
    # many tokens of a sequence share their means
    (32, 32, 16, [40, 17], [600, 333], 8), (64, 16, 16, [70, 5, 0, 41], [800, 1, 3, 500], 5),
    (16, 16, 16, [70], [17000], 6), (8, 8, 16, [133], [33700], 40)])
def test_select(L, dtype, hd, nq, nkv, page, new, length, n_blocks):
    print("select", dtype, hd, nq, nkv, page, new, length, n_blocks, flush=True)
    b = Batch(nq, nkv, hd, dtype, dtype, page, new, length, seed=n_blocks)
    for kind in ("plain", "equal", "odd"):
        mean = torch.randn(len(b.live), nkv, hd, generator=_gen(9)).to(b.dt)
        if kind == "equal":
            mean = mean[torch.randint(0, 3, (len(b.live),), generator=_gen(10))].contiguous()
        if kind == "odd":
            mean[::5, :, 3] = NAN
            mean[1::7, :, 5] = float("inf")
            mean[2::7] = 0
        want = _choose(b, mean, n_blocks)
        ctx = _ctx(L, nq, nkv, hd)
        got = ctx.select_blocks(b.cache(L, mean.cuda()), b.q.cuda(), n_blocks, **b.args(L), max_length=max(length))
        assert torch.equal(got.cpu(), want), kind
        again = ctx.select_blocks(b.cache(L, mean.cuda()), b.q.cuda(), n_blocks, **b.args(L))
        assert torch.equal(got, again)


# ---------------------------------------------------------------- attention over blocks
BLOCKS = [
    (4, 2, 16, [1, 1], [300, 20], 5), (8, 1, 64, [1], [1000], 9), (3, 3, 16, [5, 3], [5, 200], 4),
    (2, 2, 128, [2], [600], 3), (4, 2, 16, [3], [90], 200), (20, 1, 32, [2], [200], 4), (4, 2, 16, [1], [5000], 256),
    (4, 2, 16, [40, 33], [300, 40], 5),
    # many tokens of a sequence: waves walk the blocks of several
    (64, 16, 16, [170, 165], [700, 600], 5), (64, 64, 32, [330], [900], 4), (48, 16, 64, [450], [1500], 7),
    (64, 8, 128, [330], [2000], 6), (40, 1, 256, [520], [1000], 2), (64, 16, 16, [340], [5000], 9),
    (4, 2, 16, [1] * 90, [11 * i for i in range(90)], 40), (8, 8, 16, [1] * 270, [i % 100 for i in range(270)], 3)]


@pytest.mark.parametrize("dtype,cache,hd", LAYOUTS)
@pytest.mark.parametrize("nq,nkv,page,new,length,n_blocks", BLOCKS)
def test_attend_blocks(L, dtype, cache, hd, nq, nkv, page, new, length, n_blocks):
    print("blocks", dtype, cache, hd, nq, nkv, page, new, length, n_blocks, flush=True)
    b = Batch(nq, nkv, hd, dtype, cache, page, new, length, seed=n_blocks, lead=1, tail=2)
    g = _gen(n_blocks)
    blocks = torch.full((b.tokens, nkv, n_blocks), -1, dtype=torch.int32)
    for i, (n, m) in enumerate(zip(new, length)):
        for j in range(n):
            for h in range(nkv):
                ids = torch.randperm(-(-m // page), generator=g)[:n_blocks]
                blocks[b.lead + sum(new[:i]) + j, h, :len(ids)] = ids.to(torch.int32)
    _run(L, b, blocks)
    if n_blocks > 3:  # any order, twice the same, none at all, numbers that are no block
        blocks[:, :, 1] = blocks[:, :, 0]
        blocks[:, :, 2] = 2 ** 31 - 1
        blocks[:, :, 3] = -2 ** 31
        blocks[b.lead] = -1
        _run(L, b, blocks)


@pytest.mark.parametrize("dtype,cache,hd", LAYOUTS)
@pytest.mark.parametrize("nq,nkv,new", [(8, 2, [40]), (2, 2, [3]), (64, 16, [340]), (40, 1, [530])])
def test_attend_blocks_unseen_keys_may_hold_anything(L, dtype, cache, hd, nq, nkv, new):
    """A block with infinities and NaN reaches the tokens that chose it only."""
    print("blocks unseen", dtype, cache, hd, nq, nkv, new, flush=True)
    b = Batch(nq, nkv, hd, dtype, cache, 16, new, [new[0] + 400], seed=2)
    g = _gen(3)
    n = new[0]
    blocks = torch.stack([torch.stack([torch.randperm(24, generator=g)[:5].sort()[0] for _ in range(nkv)])
                          for _ in range(n)]).to(torch.int32)
    ctx = _ctx(L, nq, nkv, hd)
    clean = b.attend(ctx, L, blocks=blocks.cuda()).view(n, nkv, -1)
    page = int(b.table[0, 7])
    if cache == "e4m3":
        b.k8[page, :, 3], b.v8[page, :, 9] = 0x7F, 0x7F
    else:
        b.k16[page, :, 3], b.v16[page, :, 9] = NAN, float("-inf")
    got = b.attend(ctx, L, blocks=blocks.cuda()).view(n, nkv, -1)
    sees = (blocks == 7).any(-1).cuda()
    assert 0 < sees.sum() < sees.numel()
    assert torch.isnan(got[sees]).all() and torch.equal(got[~sees], clean[~sees])
    if cache != "e4m3":  # a value alone
        b.k16[page, :, 3] = 0.5
        got = b.attend(ctx, L, blocks=blocks.cuda()).view(n, nkv, -1)
        assert not torch.isfinite(got[sees]).any() and torch.equal(got[~sees], clean[~sees])


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_append_choose_attend(L, cache):
    """As a program uses them: prompts appended, then tokens one by one, each behind a shared prefix or
    over chosen blocks; every step against the definition on the cache as it is."""
    nq, nkv, hd, page, steps = 4, 2, 64, 16, 5
    new0 = [70, 33, 90]
    b = Batch(nq, nkv, hd, "bf16", cache, page, [1] * 3, [n + steps for n in new0], prefix=40, seed=8)
    mean = torch.zeros(len(b.live), nkv, hd, dtype=b.dt, device="cuda")
    c = b.cache(L, mean)
    ctx = _ctx(L, nq, nkv, hd)
    g = _gen(4)

    def step(new, length):
        n = sum(new)
        q, k, v = ((torch.randn(n, h * hd, generator=g) * 1.5).to(b.dt).cuda() for h in (nq, nkv, nkv))
        start = torch.tensor([sum(new[:i]) for i in range(len(new) + 1)], dtype=torch.int32).cuda()
        a = dict(table=b.table.cuda(), length=torch.tensor(length, dtype=torch.int32).cuda(),
                 start=None if max(new) == 1 else start)
        q = ctx.cache_append(c, k, v, q=q, first=b.prefix, **a)
        behind = ctx.attend(c, q, prefix=b.prefix_pages.cuda(), prefix_length=b.prefix, max_tokens=max(new),
                            max_length=max(length), **a)
        blocks = ctx.select_blocks(c, q, 3, max_length=max(length), **a)
        over = ctx.attend(c, q, blocks=blocks, max_tokens=max(new), max_length=max(length), **a)
        # the cache as it is now
        now = Batch(nq, nkv, hd, "bf16", cache, page, new, length, prefix=b.prefix, seed=8)
        now.table, now.prefix_pages = b.table, b.prefix_pages
        now.q, now.tokens = q.cpu(), n
        if cache == "e4m3":
            now.k8, now.v8 = c.k.view(torch.uint8).cpu(), c.v.view(torch.uint8).cpu()
            now.ke, now.ve = c.k_exp.cpu(), c.v_exp.cpu()
        else:
            now.k16, now.v16 = c.k.cpu(), c.v.cpu()
        _check(now, behind, None, _reference(now))
        assert torch.equal(blocks.cpu(), _choose(now, mean.cpu(), 3))
        now.prefix = 0
        _check(now, over, None, _reference(now, blocks.cpu()))

    step(new0, new0)
    for i in range(1, steps + 1):
        step([1] * 3, [n + i for n in new0])


# ---------------------------------------------------------------- appending: places and values that do not fit
@pytest.mark.parametrize("dtype,cache,hd", LAYOUTS[:6])
def test_append_places_that_do_not_exist(L, dtype, cache, hd):
    """Tokens before the sequence, past the table, in a page that is none, at a position past max_seq."""
    print("places", dtype, cache, hd, flush=True)
    nq, nkv, page = 4, 2, 16
    b = Batch(nq, nkv, hd, dtype, cache, page, [6, 40, 30], [6, 70, 30], spare=0)
    c = b.cache(L)
    old = [t.view(torch.uint8).clone() for t in (c.k, c.v)]
    qkv = torch.randn(b.tokens, (nq + 2 * nkv) * hd, generator=_gen(1)).to(b.dt).cuda()
    q, k, v = qkv.split((nq * hd, nkv * hd, nkv * hd), 1)
    a = b.args(L)
    a["length"] = torch.tensor([3, 10 ** 6, 30], dtype=torch.int32).cuda()
    a["table"] = a["table"].clone()
    a["table"][2, 1] = 2 ** 31 - 1
    ctx = _ctx(L, nq, nkv, hd, max_seq=20)
    out = ctx.cache_append(c, k, v, q=q, first=5, **a).view(b.tokens, -1)
    torch.cuda.synchronize()
    written = torch.zeros(b.live.shape, dtype=torch.bool)
    written[int(b.table[0, 0]), :3] = True
    written[int(b.table[2, 0]), :16] = True
    for now, was in zip((c.k, c.v), old):
        w = written[:, None, :].expand(now.shape[:3]).cuda()
        assert torch.equal(now.view(torch.uint8)[~w], was[~w])
    # keys of index 15 and on, at position 20 and on, are NaN, and so are queries; values are as they are
    bits = c.k.view(torch.uint8) if cache == "e4m3" else c.k
    p2 = bits[int(b.table[2, 0])]
    assert ((p2[:, 15] & 0x7F) == 0x7F).all() if cache == "e4m3" else torch.isnan(p2[:, 15]).all()
    assert not (((p2[:, 14] & 0x7F) == 0x7F).any() if cache == "e4m3" else torch.isnan(p2[:, 14]).any())
    pos = [5 - 3 + i for i in range(6)] + [10 ** 6] * 40 + [5 + i for i in range(30)]
    nan = torch.tensor([not 0 <= x < 20 for x in pos])
    assert torch.equal(torch.isnan(out).all(1).cpu(), nan) and torch.isfinite(out[~nan.cuda()]).all()


def test_append_codes_of_odd_heads(L):
    """Zeros, the least and the largest values, borders of the scale, infinities and NaN."""
    nkv, hd = 2, 64
    for dtype in ("f16", "bf16"):
        rows = [0.0, 448.0, 449.0, 448.0 * 2 ** -20, 1e-7, 61440.0, 65504.0, float("inf"), NAN, 3e38 if dtype == "bf16" else 1.0,
                1e-38 if dtype == "bf16" else 6e-8]
        b = Batch(2, nkv, hd, dtype, "e4m3", 16, [len(rows)], [len(rows)])
        x = torch.randn(len(rows), nkv * hd, generator=_gen(2)) * 1e-3
        top = torch.tensor(rows).to(b.dt)
        x = (x.clamp(-1, 1) * top.float().nan_to_num(1, 1)[:, None]).to(b.dt)
        x[:, 5] = top
        x[:, hd + 7] = -top
        c = b.cache(L)
        ctx = _ctx(L, 2, nkv, hd)
        ctx.cache_append(c, x.cuda(), x.cuda(), rotate=False, **b.args(L, starts=True))
        page = int(b.table[0, 0])
        for code, exp in ((c.k, c.k_exp), (c.v, c.v_exp)):
            code, exp = code[page].double().cpu(), exp[page].double().cpu()
            for i, r in enumerate(rows):
                y = x[i].double().view(nkv, hd)
                if not math.isfinite(r):
                    assert torch.isnan(code[:, i]).all()
                    continue
                if dtype == "f16":
                    y = y.clamp(-61440, 61440)
                # the definition: the least exponent that fits
                amax = y.abs().amax(-1)
                for h in range(nkv):
                    e = -126
                    while amax[h] > 448 * 2.0 ** e:
                        e += 1
                    assert exp[h, i] == e + 127, (dtype, r)
                    v = y[h] * 2.0 ** -e
                    step = torch.pow(2.0, torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
                    assert torch.equal(code[h, i], torch.round(v / step) * step), (dtype, r)


@pytest.mark.parametrize("dtype,cache", [("f16", "f16"), ("bf16", "e4m3")])
def test_append_strides_and_in_place(L, dtype, cache):
    nq, nkv, hd = 4, 2, 64
    b = Batch(nq, nkv, hd, dtype, cache, 16, [20, 3], [30, 3])
    x = torch.randn(b.tokens, (nq + 2 * nkv) * hd + 5, generator=_gen(3)).to(b.dt).cuda()
    cols = (nq * hd, nkv * hd, nkv * hd)
    q, k, v = x[:, 3:-2].split(cols, 1)
    ctx = _ctx(L, nq, nkv, hd)
    caches = [b.cache(L) for _ in range(2)]
    want = ctx.cache_append(caches[0], k.contiguous(), v.contiguous(), q=q.contiguous(), **b.args(L))
    before = x.clone()
    got = ctx.cache_append(caches[1], k, v, q=q, q_out=q, **b.args(L))
    assert got.data_ptr() == q.data_ptr() and torch.equal(q, want)
    before[:, 3:3 + nq * hd] = want
    assert torch.equal(x, before)
    for n in ("k", "v"):
        assert torch.equal(getattr(caches[0], n).view(torch.uint8), getattr(caches[1], n).view(torch.uint8))


# ---------------------------------------------------------------- sizes
@pytest.mark.parametrize("cache", ["f16", "e4m3"])
def test_offsets_past_32_bits(L, cache):
    """Pages more than 4 GiB (and 2^32 elements) into the cache."""
    nq, nkv, hd, page = 8, 8, 128, 64
    pool = 70000 if cache == "e4m3" else 36000
    dt = E4M3 if cache == "e4m3" else torch.float16
    print("far", cache, flush=True)
    k, v = (torch.zeros(pool, nkv, page, hd, dtype=torch.uint8 if cache == "e4m3" else dt, device="cuda").view(dt)
            for _ in range(2))
    exps = [torch.full((pool, nkv, page), 127, dtype=torch.uint8, device="cuda") for _ in range(2)] if cache == "e4m3" else []
    mean = torch.zeros(pool, nkv, hd, dtype=torch.float16, device="cuda")
    far = L.PagedCache(k, v, *exps, k_mean=mean) if exps else L.PagedCache(k, v, k_mean=mean)
    small = Batch(nq, nkv, hd, "f16", cache, page, [150], [150], spare=0)
    near_mean = torch.zeros(len(small.live), nkv, hd, dtype=torch.float16, device="cuda")
    near = small.cache(L, near_mean)
    ctx = _ctx(L, nq, nkv, hd)
    q, kk, vv = (torch.randn(150, n * hd, generator=_gen(i)).half().cuda() for i, n in enumerate((nq, nkv, nkv)))
    a = small.args(L)
    b = {**a, "table": torch.tensor([[pool - 1, pool - 3, pool - 2]], dtype=torch.int32).cuda()}
    res = []
    for c, args in ((near, a), (far, b)):
        x = ctx.cache_append(c, kk, vv, q=q, **args)
        blocks = ctx.select_blocks(c, x, 2, **args)
        last = dict(table=args["table"], length=args["length"])
        res.append((x, blocks, ctx.attend(c, x, **args), ctx.attend(c, x, blocks=blocks, **args),
                    ctx.attend(c, x[-1:], **last), ctx.attend(c, x[-1:], prefix=args["table"][0], prefix_length=150,
                                                             **{**last, "length": last["length"] * 0})))
    for x, y in zip(*res):
        assert torch.equal(x, y)


def test_sizes_of_nothing(L):
    ctx = _ctx(L, 4, 2, 64)
    b = Batch(4, 2, 64, "f16", "f16", 16, [1], [5])
    c = b.cache(L, torch.zeros(len(b.live), 2, 64, dtype=torch.float16, device="cuda"))
    none = dict(table=torch.zeros(0, 3, dtype=torch.int32, device="cuda"),
                length=torch.zeros(0, dtype=torch.int32, device="cuda"))
    q, kv = (torch.zeros(0, n, dtype=torch.float16, device="cuda") for n in (256, 128))
    assert ctx.attend(c, q, **none).shape == (0, 256)
    assert ctx.select_blocks(c, q, 4, **none).shape == (0, 2, 4)
    assert ctx.cache_append(c, kv, kv, q=q, **none).shape == (0, 256)
    # a table without columns: only the prefix is there to see
    one = dict(table=torch.zeros(1, 0, dtype=torch.int32, device="cuda"),
               length=torch.zeros(1, dtype=torch.int32, device="cuda"))
    want = ctx.attend(c, b.q.cuda(), prefix=b.table[0, :1].cuda(), prefix_length=5, **one)
    assert torch.equal(want, b.attend(ctx, L))


# ---------------------------------------------------------------- graphs, streams, contexts
def _step(ctx, c, x, args, prefix, n):
    q = ctx.cache_append(c, x[1], x[2], q=x[0], first=40, **args)
    blocks = ctx.select_blocks(c, q, 3, max_length=700, **args)
    return (q, blocks, ctx.attend(c, q, max_tokens=n, max_length=700, prefix=prefix, prefix_length=40, **args),
            ctx.attend(c, q, max_tokens=n, max_length=700, blocks=blocks, **args),
            ctx.attend(c, q, max_tokens=n, max_length=700, **args))


@pytest.mark.parametrize("cache", ["f16", "e4m3"])
@pytest.mark.parametrize("new", [[1, 1, 1], [30, 7, 44]])
def test_captured(L, cache, new):
    """Two graphs of a whole step, replayed in turn with eager calls between, follow what the tables,
    lengths and tokens hold then."""
    nq, nkv, hd = 8, 2, 64
    stream = torch.cuda.Stream()
    ctx = L.Context(Shape(nq, nkv, hd), device=0, stream=stream.cuda_stream, max_seq=4096)
    b = Batch(nq, nkv, hd, "f16", cache, 16, new, [700, 650, 690], prefix=40, seed=5)
    with torch.cuda.stream(stream):
        mean = torch.zeros(len(b.live), nkv, hd, dtype=torch.float16, device="cuda")
        c = b.cache(L, mean)
        kept = [t for t in (c.k, c.v, c.k_exp, c.v_exp, c.k_mean) if t is not None]
        args = b.args(L, starts=max(new) > 1)
        prefix = b.prefix_pages.cuda()
        x = [torch.randn(b.tokens, h * hd, device="cuda").half() for h in (nq, nkv, nkv)]

        def eager():
            return [t.clone() for t in _step(ctx, c, x, args, prefix, max(new))]

        eager()
        stream.synchronize()
        graphs = []
        for _ in range(2):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=stream):
                out = _step(ctx, c, x, args, prefix, max(new))
            graphs.append((g, out))
        for i in range(6):
            for t in x:
                t.normal_()
            args["length"].copy_(torch.tensor([n - 16 * i for n in b.len], dtype=torch.int32))
            state = [t.clone() for t in kept]
            want = eager()
            after = [t.clone() for t in kept]
            for t, s in zip(kept, state):
                t.copy_(s)
            g, out = graphs[i % 2]
            g.replay()
            stream.synchronize()
            for got, w in zip(out, want):
                assert torch.equal(got, w)
            for t, w in zip(kept, after):
                assert torch.equal(t.view(torch.uint8), w.view(torch.uint8))


def test_two_contexts_at_once(L):
    """Calls on two streams, interleaved: each as if alone."""
    nq, nkv, hd = 8, 2, 64
    streams = [torch.cuda.Stream() for _ in range(2)]
    ctxs = [L.Context(Shape(nq, nkv, hd), device=0, stream=s.cuda_stream) for s in streams]
    batches = [Batch(nq, nkv, hd, "f16", "f16", 16, n, [900, 300], prefix=100, seed=i)
               for i, n in enumerate(([1, 1], [40, 9]))]
    alone = [b.attend(_ctx(L, nq, nkv, hd), L) for b in batches]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i].append(batches[i].attend(ctxs[i], L))
    torch.cuda.synchronize()
    for i in range(2):
        for x in got[i]:
            assert torch.equal(x, alone[i])
    with pytest.raises(ValueError):  # another stream than the ctx's
        batches[0].attend(ctxs[0], L)


def test_profiled(L):
    ctx = _ctx(L, 4, 2, 64)
    b = Batch(4, 2, 64, "f16", "f16", 16, [1, 1], [90, 40], prefix=20)
    mean = torch.zeros(len(b.live), 2, 64, dtype=torch.float16, device="cuda")
    c = b.cache(L, mean)
    ctx.set_profiling(1)
    kv = torch.zeros(2, 128, dtype=torch.float16, device="cuda")
    ctx.cache_append(c, kv, kv, **b.args(L))
    b.attend(ctx, L, cache=c)
    blocks = ctx.select_blocks(c, b.q.cuda(), 2, **b.args(L))
    ctx.attend(c, b.q.cuda(), blocks=blocks, **b.args(L))
    st = ctx.kernel_stats()
    for name in ("cache_append", "attend", "select_blocks", "attend_blocks"):
        assert st[name]["launches"] == 1 and st[name]["ms"] > 0
    ctx.set_profiling(0)


def test_results_are_repeated(L):
    """The same call gives the same bits."""
    for new, prefix in (([1] * 40, 3000), ([20, 50], 100), ([1], 0)):
        b = Batch(8, 2, 128, "f16", "e4m3", 32, new, [2000 + i for i in range(len(new))], prefix, seed=4)
        ctx = _ctx(L, 8, 2, 128)
        c = b.cache(L)
        want = b.attend(ctx, L, cache=c)
        for _ in range(3):
            assert torch.equal(b.attend(ctx, L, cache=c), want)
