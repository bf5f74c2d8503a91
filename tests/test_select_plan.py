"""How a choice of blocks is divided, on the host: every launch of every call that the library accepts is one
that HIP makes, and every token is in one of them."""
import ctypes as C
import random
import shutil
import subprocess

import pytest

from paper_2606_31808_amd import build
from paper_2606_31808_amd import lmop as L
from tests.test_operator_refusals import UNS, _call, _paged, ctx  # noqa: F401

SRC = """
#include "select_plan.h"
using namespace lmop;
extern "C" void plan(int n_seqs, int n_tokens, int max_length, int page, int nkv, int hd, int starts, long long* out) {
  const SelectPlan p = plan_select(SelectSizes{n_seqs, n_tokens, max_length, page, nkv, hd, starts != 0});
  out[0] = p.pages, out[1] = p.tile, out[2] = p.waves, out[3] = p.items, out[4] = p.each;
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    if not shutil.which("g++"):
        pytest.skip("no g++")
    d = tmp_path_factory.mktemp("plan")
    (d / "r.cpp").write_text(SRC)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-shared", "-fPIC", f"-I{build.CSRC}", str(d / "r.cpp"), "-o",
                    str(d / "r.so")], check=True)
    lib = C.CDLL(str(d / "r.so"))

    def f(*sizes):
        out = (C.c_longlong * 5)()
        lib.plan(*(int(x) for x in sizes), out)
        return tuple(out)

    return f


def _check(plan, n_seqs, n_tokens, max_length, page, nkv, hd, starts):
    pages, tile, waves, items, each = plan(n_seqs, n_tokens, max_length, page, nkv, hd, starts)
    assert pages == max(1, -(-max_length // page))
    assert 1 <= each <= items < 2 ** 31
    assert each * nkv * 64 * waves < 2 ** 32
    assert items == (n_tokens // tile + n_seqs if tile else n_tokens)
    assert (tile or 1) * pages <= 16384 and (waves == 16 or tile or pages <= 4 * 64 // (hd // 8) * 8)
    return -(-items // each), tile


def test_long_contexts_of_many_tokens_are_several_launches(plan):
    """Accepted calls that one launch of 1024 threads a workgroup could not take."""
    assert _check(plan, 1, 1300000, 16384 * 16, 16, 4, 64, True) == (2, 0)
    assert _check(plan, 1, 140000, 8750 * 16, 16, 32, 128, True) == (2, 0)
    assert _check(plan, 1, 4300000, 5000 * 16, 16, 1, 64, True) == (2, 0)
    assert _check(plan, 1, 1300000, 16, 16, 4, 64, True) == (1, 16)
    assert _check(plan, 32, 32, 32000, 64, 8, 128, False) == (1, 0)


def test_what_is_accepted_can_be_launched(plan):
    rng = random.Random(3)
    several = 0
    for _ in range(20000):
        nkv, group = rng.choice((1, 2, 4, 8, 32)), rng.choice((1, 2, 4, 8))
        page, hd = rng.choice((16, 32, 64, 128, 256)), rng.choice((64, 128))
        n_seqs = int(2 ** rng.uniform(0, 22))
        n_tokens = int(rng.choice((2 ** rng.uniform(0, 23), 2 ** 24 / (group + 2) / nkv * rng.uniform(0.7, 1))))
        starts = rng.random() < 0.8
        if not starts:
            n_tokens = n_seqs
        # what the library takes
        if (n_tokens + 2 * n_seqs) * (group + 2) * nkv > 2 ** 24:
            continue
        max_length = rng.choice((0, int(2 ** rng.uniform(0, 14) * page)))
        several += _check(plan, n_seqs, n_tokens, max_length, page, nkv, hd, starts)[0] > 1
    assert several > 10


@pytest.mark.parametrize("tokens,kv,refused", [(1300000, 4, False), (1398099, 4, False), (1398100, 4, True)])
def test_library_takes_them(ctx, tokens, kv, refused):  # noqa: F811
    """The first and the last call of one sequence, of the ctx's 4 + 4 heads, that are accepted."""
    assert ctx.heads[1] == kv
    a = _paged(ctx, "lmop_select_blocks", batch_n_tokens=tokens, batch_n_seqs=1, max_length=16384 * 16)
    assert _call(ctx, "lmop_select_blocks", a) == UNS
    assert ("too many for one call" in L._lib.lmop_last_error(ctx.ctx).decode()) == refused
