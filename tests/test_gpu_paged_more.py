"""The paged cache's operators where their sizes, values and uses are out of the ordinary; batches, the definition in
64 bits and its tolerances are test_gpu_paged's."""
import pytest
import torch

from tests.test_gpu_paged import L, _ctx, _gen  # noqa: F401

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
