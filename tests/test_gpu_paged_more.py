"""The paged cache's operators where their sizes, values and uses are out of the ordinary; batches, the definition in
64 bits and its tolerances are test_gpu_paged's."""
import pytest
import torch

from tests.test_gpu_paged import Batch, L, _ctx, _gen  # noqa: F401

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
