"""Making a Context: its rotary table, and the time that takes."""
import time

import pytest
import torch

from tests.test_gpu_paged import L, Shape, _ctx  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hd,theta,max_seq", [(128, 1e4, 65536), (64, 1e6, 131072), (128, 5e5, 300)])
def test_rotary_table(L, hd, theta, max_seq):  # noqa: F811
    """Heads (1, 0) of every position come out as (cos, sin), rounded to fp32 (2^-24 of at most one) and to the type."""
    ctx = _ctx(L, 1, 1, hd, max_seq=max_seq, theta=theta)
    half = hd // 2
    angle = torch.arange(max_seq, dtype=torch.float64)[:, None] * theta ** (-2.0 * torch.arange(half, dtype=torch.float64) / hd)
    x = torch.zeros(max_seq, hd, dtype=torch.float16, device="cuda")
    x[:, :half] = 1
    pos = torch.arange(max_seq, dtype=torch.int32, device="cuda")
    for kind in (torch.float16, torch.bfloat16):
        got = ctx.qk_norm_rope(x.to(kind), pos=pos).double().cpu()
        want = torch.cat((angle.cos(), angle.sin()), 1)
        step = torch.finfo(kind).eps / 2
        assert ((got - want).abs() <= step * want.abs() + 2.0 ** -23 + (2.0 ** -25 if kind is torch.float16 else 0)).all()
    # the next position has none
    assert ctx.qk_norm_rope(x[:1], pos=pos[:1] + max_seq).isnan().all()


def test_a_context_is_made_in_little_time(L):  # noqa: F811
    """65,536 positions of heads of 128: a table of 34 MB.  On a CPU thread it took 60 to 116 ms."""
    took = []
    for _ in range(6):
        torch.cuda.synchronize()
        t = time.perf_counter()
        ctx = L.Context(Shape(32, 8, 128), device=0, stream=torch.cuda.current_stream().cuda_stream, max_seq=65536)
        took.append(time.perf_counter() - t)
        ctx.close()
    print("made in", [f"{x * 1e3:.2f} ms" for x in took], flush=True)
    assert min(took) < 0.01
