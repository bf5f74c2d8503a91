"""The paged cache's operators where their sizes, values and uses are out of the ordinary; batches, the definition in
64 bits and its tolerances are test_gpu_paged's."""
import copy
import math

import pytest
import torch

from tests.test_gpu_paged import E4M3, NAN, Batch, L, Shape, _check, _ctx, _gen, _reference  # noqa: F401

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------- choosing blocks: several launches
def test_select_of_more_threads_than_a_launch(L):  # noqa: F811
    """4.3 million tokens, each a workgroup of 1024 threads: sequences in the first launch, across the border of
    the two, and one whose tokens come before its keys."""
    n, hd, page, pages = 4300000, 64, 16, 5000
    border = (2 ** 32 - 1) // 1024
    start = [2, 60, border - 40, border + 50, n - 3]
    length = [pages * page, 0, pages * page - 1000, 5]
    print("select", n, start, length, flush=True)
    ctx = _ctx(L, 1, 1, hd)
    g = _gen(1)
    q = torch.zeros(n, hd, dtype=torch.float16, device="cuda")
    table = torch.stack([torch.randperm(pages, generator=g) for _ in range(4)]).to(torch.int32).cuda()
    mean = torch.randn(pages, 1, hd, generator=g).half().cuda()
    k = torch.zeros(pages, 1, page, hd, dtype=torch.float16, device="cuda")
    cache = L.PagedCache(k, k, k_mean=mean)
    lengths = torch.tensor(length, dtype=torch.int32, device="cuda")
    out = torch.full((n, 1, 3), 7, dtype=torch.int32, device="cuda")
    for i in (0, 2):
        q[start[i]:start[i + 1]] = torch.randn(start[i + 1] - start[i], hd, generator=g).half().cuda()
    ctx.select_blocks(cache, q, 3, table=table, length=lengths, max_length=pages * page, out=out,
                      start=torch.tensor(start, dtype=torch.int32, device="cuda"))
    for i in (0, 2):
        a, b = start[i], start[i + 1]
        alone = ctx.select_blocks(cache, q[a:b], 3, table=table[i:i + 1], length=lengths[i:i + 1],
                                  start=torch.tensor([0, b - a], dtype=torch.int32, device="cuda"))
        assert torch.equal(out[a:b], alone) and (alone >= 0).all()
    assert torch.all(out[start[1]:start[2]] == -1)
    # 5 keys: the last five tokens have a block, their own, and no other
    assert torch.all(out[start[3]:n - 3 - 5] == -1)
    assert torch.equal(out[n - 8:n - 3, 0].cpu(), torch.tensor([[0, -1, -1]] * 5, dtype=torch.int32))
    assert torch.all(out[:2] == 7) and torch.all(out[n - 3:] == 7)


# ---------------------------------------------------------------- attention: scores far from zero
FAR = [([1, 1], [300, 200], 0, 0), ([1, 1, 1], [5000, 70, 1], 0, 0), ([30, 40], [300, 200], 0, 0), ([70], [3000], 0, 0),
       ([1] * 16, [20] * 16, 20000, 0), ([1, 1], [300, 200], 0, 4), ([330], [900], 0, 5)]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("new,length,prefix,n_blocks", FAR)
def test_attend_scores_far_from_zero(L, dtype, new, length, prefix, n_blocks):  # noqa: F811
    """One key's score, of up to 2^34 in fp16 and 2^70 in bf16, is past every other's by far: the result is its
    value, to the bit, and lse its score to fp32's rounding.  A score of 2^30 is itself known to 2^6 only, which is no
    reason for its weight to be 2^64 or none."""
    print("far", dtype, new, length, prefix, n_blocks, flush=True)
    nq, nkv, hd = (64, 16, 64) if n_blocks == 5 else (8, 2, 128)
    b = Batch(nq, nkv, hd, dtype, dtype, 16, new, length, prefix, seed=len(new))
    g = _gen(2)
    wrong = []
    for bits in (18, 22, 25, 28, 30, 33) + ((34,) if dtype == "f16" else (36, 50, 70)):  # (fp16: queries of 41,000)
        for sign in (1, -1):
            # scores of about 2^bits, in the exponential's units: the best sign * s, the others below it
            near = 2.0 ** ((bits - 7 + 2.5) / 2)
            b.q = (near * (1 + torch.rand(b.tokens, nq, 1, generator=g) / 2)).expand(-1, -1, hd).reshape(b.tokens, -1).to(b.dt)
            live = b.live[:, None, :].expand(b.k16.shape[:3])
            b.k16[live] = (0.25 if sign > 0 else -1.5) * near
            pages = b.prefix_pages[:1] if prefix else b.table[:, 0]
            b.k16[pages.long(), :, 0] = sign * near
            blocks = None
            if n_blocks:
                blocks = torch.arange(n_blocks, dtype=torch.int32).expand(b.tokens, nkv, n_blocks).contiguous().cuda()
            lse = torch.full((b.tokens, nq), 7.0, device="cuda")
            out = b.attend(_ctx(L, nq, nkv, hd), L, lse=lse, blocks=blocks).view(b.tokens, nq, hd).cpu()
            seq = torch.repeat_interleave(torch.arange(len(new)), torch.tensor(new))
            at = pages.long()[seq] if not prefix else pages.long().expand(b.tokens)
            want = b.v16[at, :, 0].repeat_interleave(nq // nkv, 1)
            score = (b.q.double().view(b.tokens, nq, hd) * b.k16[at, :, 0].double().repeat_interleave(nq // nkv, 1)).sum(-1)
            score = score * hd ** -0.5
            # the products' sum, the scale's two roundings, the sum's, its logarithm's base
            ok = torch.equal(out, want) and ((lse.double().cpu() - score).abs() <= (hd + 8) * 2.0 ** -23 * score.abs()).all()
            if not ok:
                wrong.append((bits * sign, out[:, 0, 0].isnan().sum().item(), (out != want).sum().item()))
    assert not wrong, wrong


# ---------------------------------------------------------------- attention: weights in fp32's precision
# (nq, nkv, hd, page, new, length, prefix, blocks): every kernel, and parts that are joined
EVERY = [(8, 2, 128, 64, [1], [500], 0, 0), (8, 2, 64, 16, [1] * 40, [200 + i for i in range(40)], 0, 0),
         (8, 2, 128, 32, [1, 1], [5000, 300], 0, 0), (8, 2, 64, 16, [1] * 64, [20] * 64, 3300, 0),
         (4, 2, 128, 64, [60, 41], [300, 200], 30, 0), (2, 1, 64, 32, [70], [3000], 0, 0),
         (8, 2, 64, 16, [1, 1], [400, 300], 0, 6), (64, 16, 64, 16, [340], [900], 0, 8)]


@pytest.mark.parametrize("dtype,cache", [("f16", "f16"), ("bf16", "bf16"), ("f16", "e4m3"), ("bf16", "e4m3")])
@pytest.mark.parametrize("nq,nkv,hd,page,new,length,prefix,n_blocks", EVERY)
def test_attend_is_as_exact_as_its_type(L, dtype, cache, nq, nkv, hd, page, new, length, prefix, n_blocks):  # noqa: F811
    """The error is that of rounding the result once.  Errors of independent steps add as squares: what is held in
    fp32 (2^-23 of a score of up to 40, some tens of them), and weights to 2^-16, are at most 1/20 of the root mean
    square of the result's rounding (2^-12 and 2^-9 / sqrt(3)), 1.00125 times together; weights of the type's own
    precision make it 1.25 times."""
    print("exact", dtype, cache, nq, nkv, hd, page, new, length, prefix, n_blocks, flush=True)
    b = Batch(nq, nkv, hd, dtype, cache, page, new, length, prefix, seed=7, q_size=1.0)
    blocks = None
    if n_blocks:
        g = _gen(3)
        blocks = torch.stack([torch.randperm(min(length) // page, generator=g)[:n_blocks].sort()[0]
                              for _ in range(b.tokens * nkv)]).view(b.tokens, nkv, n_blocks).to(torch.int32)
    want = _reference(b, blocks)[0]
    got = b.attend(_ctx(L, nq, nkv, hd), L, blocks=None if blocks is None else blocks.cuda()).double().cpu()
    off = lambda x: (x - want).square().mean().sqrt().item()
    assert off(got) <= 1.02 * off(want.to(b.dt).double())


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("new,length,prefix,n_blocks,nq,nkv", [
    ([1], [30000], 0, 0, 4, 1), ([1] * 3, [30000] * 3, 0, 0, 4, 1), ([40], [30000], 0, 0, 4, 1), ([1] * 64, [0] * 64, 30000, 0, 8, 2),
    ([1], [16384], 0, 1024, 4, 1), ([340], [16384], 0, 1024, 64, 16)])
def test_attend_many_keys_of_little_weight(L, dtype, new, length, prefix, n_blocks, nq, nkv):  # noqa: F811
    """One key of weight 1 whose value is zero, and thousands of weight 2^-26 with a value of one: all that the
    result has comes from these."""
    print("tail", dtype, new, length, prefix, n_blocks, flush=True)
    hd, page = 64, 16
    b = Batch(nq, nkv, hd, dtype, dtype, page, new, length, prefix, seed=1)
    b.q[:] = 1.0
    live = b.live[:, None, :].expand(b.k16.shape[:3])
    drop = 26 * math.log(2)
    low = torch.tensor(-drop / hd / hd ** -0.5).to(b.dt)
    b.k16[live], b.v16[live] = low, 1.0
    pages = b.prefix_pages[:1].long() if prefix else b.table[:, 0].long()
    b.k16[pages, :, 0], b.v16[pages, :, 0] = 0.0, 0.0
    blocks = None
    if n_blocks:
        blocks = torch.arange(n_blocks, dtype=torch.int32).expand(b.tokens, nkv, n_blocks).contiguous().cuda()
    lse = torch.full((b.tokens, nq), 7.0, device="cuda")
    out = b.attend(_ctx(L, nq, nkv, hd), L, lse=lse, blocks=blocks).double().cpu().view(b.tokens, nq, hd)
    w = math.exp(low.double().item() * hd * hd ** -0.5)
    for t, (i, j) in enumerate((i, j) for i, n in enumerate(new) for j in range(n)):
        tail = (prefix or length[i] - new[i] + j + 1) - 1
        want = tail * w / (1 + tail * w)
        # a score of 18: 64 exact products of 0.28, four roundings, the exponential; the weights; sums of equal terms
        tol = 64 * 18 * 2.0 ** -23 + 4 * 18 * 2.0 ** -23 + 2.0 ** -21 + 2.0 ** -16 + 2 * (tail + 64) * 2.0 ** -23
        if dtype == "f16":  # a weight is the nearest in steps of 2^-24, the largest at least 2^7
            tol += 2.0 ** -32 / 2.0 ** -26
        eps = torch.finfo(b.dt).eps / 2
        assert ((out[t] - want).abs() <= want * tol + eps * want * (1 + tol)).all()
        # (the sum of the weights is 1 and more, and as a sum of fp32 terms known to N 2^-23 of that)
        assert ((lse[t].double().cpu() - math.log1p(tail * w)).abs() <= tail * w * tol + (tail + 64) * 2.0 ** -23).all()


# ---------------------------------------------------------------- attention: tokens without keys
@pytest.mark.parametrize("dtype,cache,hd", [("f16", "f16", 64), ("bf16", "bf16", 128), ("f16", "e4m3", 128), ("bf16", "e4m3", 64)])
@pytest.mark.parametrize("new,length,prefix", [([1, 1, 1], [0, 20, 0], 0), ([3, 5], [1, 0], 0), ([40, 60, 2], [10, 0, 2], 0),
                                               ([2, 1, 4], [5000, 0, 1], 0), ([70, 9], [3000, 4], 0), ([3, 1], [1, 0], 5)])
def test_attend_tokens_before_their_sequence(L, dtype, cache, hd, new, length, prefix):  # noqa: F811
    """Each that sees no key gets zeros and minus infinity, and no other does."""
    print("before", dtype, cache, hd, new, length, prefix, flush=True)
    b = Batch(4, 2, hd, dtype, cache, 16, new, length, prefix, seed=5)
    lse = torch.full((b.tokens, 4), 7.0, device="cuda")
    out = b.attend(_ctx(L, 4, 2, hd), L, lse=lse)
    none = torch.tensor([prefix == 0 and m - n + j < 0 for n, m in zip(new, length) for j in range(n)]).cuda()
    assert none.any() == (prefix == 0)
    assert torch.all(out[none] == 0) and torch.all(lse[none] == -float("inf"))
    assert torch.all(out[~none].abs().sum(1) > 0) and torch.isfinite(lse[~none]).all()


# ---------------------------------------------------------------- calls with a workspace
# (nq, nkv, hd, page, new, length, prefix, blocks): splits of few vectors; a prefix on its own, few vectors and
# tiles; splits of tiles; splits of a walk; splits of chosen blocks
WITH_PARTS = [(8, 2, 64, 16, [1, 1], [9000, 3000], 0, 0), (4, 2, 128, 64, [1] * 8, [40] * 8, 26000, 0),
              (8, 2, 64, 16, [1] * 40, [20 + i for i in range(40)], 5300, 0), (2, 1, 64, 32, [70], [3000], 0, 0),
              (64, 16, 64, 16, [340], [5000], 0, 9), (4, 2, 64, 16, [1], [5000], 0, 256)]


class Call:
    """One attention call with every tensor on the device."""

    def __init__(self, L, ctx, nq, nkv, hd, page, new, length, prefix, n_blocks, seed):  # noqa: F811
        b = Batch(nq, nkv, hd, "f16", "f16", page, new, length, prefix, seed=seed)
        self.ctx, self.cache, self.q = ctx, b.cache(L), b.q.cuda()
        self.args = b.args(L, max_tokens=max(new), max_length=max(length))
        if prefix:
            self.args.update(prefix=b.prefix_pages.cuda(), prefix_length=prefix)
        if n_blocks:
            g = _gen(seed)
            self.args["blocks"] = torch.stack([torch.randperm(max(length) // page, generator=g)[:n_blocks].sort()[0]
                                               for _ in range(b.tokens * nkv)]).view(b.tokens, nkv, n_blocks).to(torch.int32).cuda()
        sizes = []

        def workspace(n):
            sizes.append(n)
            return torch.empty(n, dtype=torch.uint8, device="cuda")

        a = self.args
        L.lmop_attend(ctx.ctx, ctx.heads, self.cache, self.q, torch.empty_like(self.q), a["table"], a["length"], a["start"],
                      a["max_tokens"], a["max_length"], a.get("prefix"), prefix, a.get("blocks"), workspace=workspace)
        assert len(sizes) == 1 and sizes[0] > 0

    def __call__(self):
        return self.ctx.attend(self.cache, self.q, **self.args)


@pytest.mark.parametrize("nq,nkv,hd,page,new,length,prefix,n_blocks", WITH_PARTS)
def test_two_streams_with_workspaces(L, nq, nkv, hd, page, new, length, prefix, n_blocks):  # noqa: F811
    """Calls of two contexts under way at once, each with its parts in a workspace of its own."""
    print("streams", nq, nkv, hd, page, new[:3], length[:3], prefix, n_blocks, flush=True)
    calls, want = [], []
    for i in range(2):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            calls.append((stream, Call(L, L.Context(Shape(nq, nkv, hd), device=0, stream=stream.cuda_stream, max_seq=64),
                                       nq, nkv, hd, page, new, length, prefix, n_blocks, seed=i)))
            want.append(calls[i][1]())
        torch.cuda.synchronize()
    assert not torch.equal(*want)
    got = [[], []]
    for _ in range(30):
        for i, (stream, call) in enumerate(calls):
            with torch.cuda.stream(stream):
                got[i].append(call())
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(x, want[i]) for x in got[i])


@pytest.mark.parametrize("nq,nkv,hd,page,new,length,prefix,n_blocks", WITH_PARTS)
def test_captured_with_workspaces(L, nq, nkv, hd, page, new, length, prefix, n_blocks):  # noqa: F811
    """Two graphs of a call and its joining launch, replayed in turn with eager calls between."""
    print("graphs", nq, nkv, hd, page, new[:3], length[:3], prefix, n_blocks, flush=True)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        call = Call(L, L.Context(Shape(nq, nkv, hd), device=0, stream=stream.cuda_stream, max_seq=64), nq, nkv, hd, page,
                    new, length, prefix, n_blocks, seed=3)
        stream.synchronize()
        graphs = []
        for _ in range(2):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=stream):
                out = call()
            graphs.append((g, out))
        for i in range(6):
            call.q.normal_()
            want = call().clone()
            g, out = graphs[i % 2]
            out.zero_()
            g.replay()
            again = call()
            stream.synchronize()
            assert torch.equal(out, want) and torch.equal(again, want)


# ---------------------------------------------------------------- attention: values near the type's end
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("new,length,prefix,n_blocks,nq,nkv", [
    ([1], [600], 0, 0, 8, 2), ([1] * 70, [600] * 70, 0, 0, 8, 8), ([60, 41], [700, 690], 0, 0, 4, 2), ([1] * 64, [0] * 64, 3300, 0, 8, 2),
    ([1], [640], 0, 40, 8, 2), ([340], [980], 0, 40, 64, 16)])
def test_attend_large_values(L, dtype, new, length, prefix, n_blocks, nq, nkv):  # noqa: F811
    """Values of 2^127 (fp16: 65504) of two keys, the second of 2^7.9 times the first one's weight and 256 keys on, so
    that the wave that holds both does not move its reference: the result is that value, as it is with weights of at
    most one."""
    print("large", dtype, new[:3], length[:3], prefix, n_blocks, flush=True)
    hd = 128
    b = Batch(nq, nkv, hd, dtype, dtype, 16, new, length, prefix, seed=1)
    top = 65504.0 if dtype == "f16" else 2.0 ** 127
    b.q[:] = 1.0
    live = b.live[:, None, :].expand(b.k16.shape[:3])
    unit = 0.6931471805599453 / hd * hd ** 0.5  # a key of so much: a power of two in weight
    b.k16[live], b.v16[live] = -300 * unit, top
    for i in range(len(new)):
        pages = b.prefix_pages.long() if prefix else b.table[i].long()
        for key, size in ((10, 0.0), (266, 7.9)):
            b.k16[pages[key // 16], :, key % 16] = size * unit
    blocks = None
    if n_blocks:
        blocks = torch.arange(n_blocks, dtype=torch.int32).expand(b.tokens, nkv, n_blocks).contiguous().cuda()
    out = b.attend(_ctx(L, nq, nkv, hd), L, blocks=blocks)
    assert torch.all(out.float() == torch.tensor(top).to(b.dt).float())


# ---------------------------------------------------------------- infinities among values: their neighbours
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("nq,nkv,hd,page,new,length,n_blocks", [
    (2, 2, 64, 16, [9, 3], [40, 20], 0), (4, 1, 128, 32, [4], [300], 0), (4, 2, 128, 16, [60, 41], [300, 90], 0),
    (64, 16, 64, 16, [340], [900], 8)])
def test_attend_neighbours_of_infinite_values(L, dtype, nq, nkv, hd, page, new, length, n_blocks):  # noqa: F811
    """A value that is infinite or NaN, of a key that some tokens see and some do not, says nothing about the key's
    other dimensions: their results stay as they are, to the bit, in every token."""
    print("neighbours", dtype, nq, nkv, hd, page, new, length, n_blocks, flush=True)
    b = Batch(nq, nkv, hd, dtype, dtype, page, new, length, seed=9)
    key = length[0] - 2  # of the last two tokens
    blocks = None
    if n_blocks:
        key = 5 * page + 3
        g = _gen(3)
        blocks = torch.stack([torch.randperm(min(length) // page, generator=g)[:n_blocks].sort()[0]
                              for _ in range(b.tokens * nkv)]).view(b.tokens, nkv, n_blocks).to(torch.int32).cuda()
    ctx = _ctx(L, nq, nkv, hd)
    clean = b.attend(ctx, L, blocks=blocks).view(b.tokens, nq, hd)
    odd = {2: float("inf"), 9: float("-inf"), hd - 1: NAN}
    for d, x in odd.items():
        b.v16[int(b.table[0, key // page]), :, key % page, d] = x
    got = b.attend(ctx, L, blocks=blocks).view(b.tokens, nq, hd)
    others = [d for d in range(hd) if d not in odd]
    assert torch.isfinite(clean).all() and torch.equal(got[..., others], clean[..., others])
    sees = (blocks == 5).any(-1).repeat_interleave(nq // nkv, 1) if n_blocks else \
        (torch.arange(b.tokens, device="cuda") >= new[0] - 2)[:, None].expand(-1, nq) & \
        (torch.arange(b.tokens, device="cuda") < new[0])[:, None]
    assert torch.equal(torch.isfinite(got).all(-1), ~sees)


# ---------------------------------------------------------------- values of 8-bit pages
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("tokens", [1, 20])
def test_every_code_and_exponent(L, dtype, tokens):  # noqa: F811
    """A token that sees one key gets its value: the code times the power of two, as the nearest of the tokens' type."""
    dt, nkv, hd, page = torch.float16 if dtype == "f16" else torch.bfloat16, 2, 128, 16
    n = 254
    codes = torch.arange(256, dtype=torch.uint8).view(1, nkv, 1, hd).expand(n, nkv, page, hd).contiguous()
    exps = torch.arange(1, 255, dtype=torch.uint8).view(n, 1, 1).expand(n, nkv, page).contiguous()
    k = torch.zeros(n, nkv, page, hd, dtype=torch.uint8)
    cache = L.PagedCache(k.view(E4M3).cuda(), codes.view(E4M3).cuda(), torch.full_like(exps, 127).cuda(), exps.cuda())
    ctx = _ctx(L, nkv, nkv, hd)
    out = ctx.attend(cache, torch.ones(n * tokens, nkv * hd, dtype=dt, device="cuda"),
                     table=torch.arange(n, dtype=torch.int32, device="cuda")[:, None], max_tokens=tokens, max_length=1,
                     length=torch.ones(n, dtype=torch.int32, device="cuda"),
                     start=torch.arange(n + 1, dtype=torch.int32, device="cuda") * tokens)
    got = out.view(n, tokens, 256)[:, -1].cpu().double()
    value = codes[:, :, 0].reshape(n, 256).view(E4M3).double() * torch.pow(2.0, exps[:, :1, 0].double() - 127)
    want = value.to(dt).double()
    # (bf16: fp32 sums of weights of 2^-8 keep values from 2^-118 on)
    least = 0 if dtype == "f16" else 2.0 ** -118
    same = (got == want) | (got.isnan() & (want.isnan() | want.isinf())) | (value.abs() < least) & (got.abs() <= least)
    assert same.all(), [(i, hex(j), value[i, j].item(), got[i, j].item()) for i, j in (~same).nonzero()[:8].tolist()]
    if tokens > 1:
        assert torch.all(out.view(n, tokens, 256)[:, :-1] == 0)


# ---------------------------------------------------------------- infinities among values that are seen
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("nq,nkv,hd,page,new,length,prefix,n_blocks", EVERY)
def test_attend_infinite_values(L, dtype, nq, nkv, hd, page, new, length, prefix, n_blocks):  # noqa: F811
    """A positive weight times infinity is infinity, of its sign: in that dimension, for the tokens that see the key, and
    with both signs or a NaN it is NaN.  No other result changes by a bit."""
    print("inf", dtype, nq, nkv, hd, page, new[:3], length[:3], prefix, n_blocks, flush=True)
    b = Batch(nq, nkv, hd, dtype, dtype, page, new, length, prefix, seed=7, q_size=1.0)
    blocks = None
    if n_blocks:
        blocks = torch.arange(n_blocks, dtype=torch.int32).expand(b.tokens, nkv, n_blocks).contiguous().cuda()
    ctx = _ctx(L, nq, nkv, hd)
    clean = b.attend(ctx, L, blocks=blocks).view(b.tokens, nkv, nq // nkv, hd)
    assert torch.isfinite(clean).all()
    inf = float("inf")
    want = clean.clone()
    seq = torch.repeat_interleave(torch.arange(len(new)), torch.tensor(new)).cuda()
    for where, pages, n, sees in ([(0, b.prefix_pages, prefix, torch.ones_like(seq, dtype=torch.bool))] if prefix else []) + \
            [(1, b.table[0], length[0] - new[0], seq == 0)]:
        if n < 8:
            continue
        for key, d, x in ((1, 3 + where, inf), (4, 17 + where, -inf), (2, 40 + where, inf), (5, 40 + where, -inf), (3, 50 + where, NAN)):
            b.v16[int(pages[key // page]), nkv - 1, key % page, d] = x
            at = want[sees][:, -1, :, d]
            want[:, -1, :, d] = torch.where(sees[:, None], want[:, -1, :, d] + x, want[:, -1, :, d])
            assert at.numel()
    got = b.attend(ctx, L, blocks=blocks).view(want.shape)
    same = (got == want) | (got.isnan() & want.isnan())
    assert not torch.isfinite(want).all()
    assert same.all(), [(i, got[tuple(i)].item(), want[tuple(i)].item()) for i in (~same).nonzero()[:6].tolist()]


@pytest.mark.parametrize("dtype,cache,hd", [("f16", "f16", 64), ("bf16", "bf16", 128), ("f16", "e4m3", 128), ("bf16", "e4m3", 64)])
@pytest.mark.parametrize("nq,nkv,new,length,prefix", [
    (4, 2, [3, 1], [1, 0], 37), (7, 1, [8], [5], 7), (4, 2, [40, 60, 2], [10, 0, 2], 100), (4, 4, [2, 3] * 30, [0, 9] * 30, 3000),
    (8, 1, [38, 13], [35, 15], 5000), (16, 2, [2, 1, 2], [0, 5, 2], 130)])
def test_attend_tokens_before_their_sequence_see_the_prefix(L, dtype, cache, hd, nq, nkv, new, length, prefix):  # noqa: F811
    """All of it, whatever their index; every other token its own keys too."""
    print("before, prefix", dtype, cache, hd, nq, nkv, new[:4], length[:4], prefix, flush=True)
    b = Batch(nq, nkv, hd, dtype, cache, 16, new, length, prefix, seed=6)
    index = torch.tensor([m - n + j for n, m in zip(new, length) for j in range(n)])
    early = (index < 0).nonzero()[:, 0]
    lse = torch.full((b.tokens, nq), 7.0, device="cuda")
    out = b.attend(_ctx(L, nq, nkv, hd), L, lse=lse)
    alone = copy.copy(b)  # the same cache, each such token a sequence without keys
    alone.new, alone.len, alone.q, alone.tokens = [1] * len(early), [0] * len(early), b.q[early], len(early)
    alone.table = b.table[:1].expand(len(early), -1)
    _check(alone, out[early.cuda()], lse[early.cuda()], _reference(alone))
    ref = [x.clone() for x in _reference(b)]
    ref[1][early] = NAN  # (left out by _check)
    _check(b, out, lse, ref)
