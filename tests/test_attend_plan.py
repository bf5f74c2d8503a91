"""How attention over a paged cache is divided, on the host: the sizes that the GPU tests run take every
kernel, every key is walked once, and workspaces are as large as the parts."""
import ctypes as C
import itertools
import random
import shutil
import subprocess

import pytest

from paper_2606_31808_amd import build
from tests import test_gpu_paged as gpu

SRC = """
#include "attend_plan.h"
using namespace lmop;
struct Out { int few, waves, tiles, splits, chunk, per_seq; };
static Out of(const AttendLaunch& l) { return Out{l.few, l.waves, l.tiles, l.splits, l.chunk, l.per_seq}; }
extern "C" int plan(int n_seqs, int n_tokens, int max_tokens, int max_length, int prefix, int n_blocks, int page,
                    int nq, int nkv, int hd, int starts, Out* own, Out* pre, unsigned long long* bytes) {
  AttendSizes s{n_seqs, n_tokens, max_tokens, max_length, prefix, n_blocks, page, nq, nkv, hd, starts != 0};
  const AttendPlan p = plan_attend(s);
  *own = of(p.own), *pre = of(p.prefix), *bytes = attend_workspace(p, s);
  return p.parts;
}
extern "C" void constants(int* c) {
  c[0] = kFewVectors, c[1] = kTileVectors, c[2] = kTileKeys, c[3] = kMaxEntries, c[4] = kWalkVectors, c[5] = kWalkWindow;
}
"""


class Out(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("few", "waves", "tiles", "splits", "chunk", "per_seq")]


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    if not shutil.which("g++"):
        pytest.skip("no g++")
    d = tmp_path_factory.mktemp("plan")
    (d / "r.cpp").write_text(SRC)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-shared", "-fPIC", f"-I{build.CSRC}", str(d / "r.cpp"), "-o",
                    str(d / "r.so")], check=True)
    return C.CDLL(str(d / "r.so"))


def _plan(lib, n_seqs, n_tokens, max_tokens, max_length, prefix, n_blocks, page, nq, nkv, hd, starts):
    own, pre, size = Out(), Out(), C.c_ulonglong()
    parts = lib.plan(n_seqs, n_tokens, max_tokens, max_length, prefix, n_blocks, page, nq, nkv, hd, int(starts),
                     C.byref(own), C.byref(pre), C.byref(size))
    return parts, own, pre, size.value


def _kind(parts, own, pre, n_blocks):
    name = ("blocks " if n_blocks else "") + (f"few {own.waves}" if own.few else "walk" if n_blocks else "tile")
    if pre.tiles:
        name += " + " + ("few" if pre.few else "tile")
    return name


def test_gpu_sizes_take_every_kernel(lib):
    kinds, joined = set(), set()
    cases = [(nq, nkv, page, [1] * len(ln), ln, pre, 0) for nq, nkv, page, ln, pre in gpu.SINGLE + gpu.LONG + gpu.MANY]
    cases += [(nq, nkv, page, new, ln, pre, 0) for nq, nkv, page, new, ln, pre in gpu.SEVERAL]
    cases += [(nq, nkv, page, new, ln, 0, nb) for nq, nkv, page, new, ln, nb in gpu.BLOCKS]
    for nq, nkv, page, new, length, prefix, nb in cases:
        starts = max(new) != 1 or min(new) != 1
        p = _plan(lib, len(new), sum(new), max(new), max(length), prefix, nb, page, nq, nkv, 64, starts)
        kinds.add(_kind(*p[:3], nb))
        joined.add((p[0] > 0, p[1].few))
    assert kinds == {"few 1", "few 4", "few 8", "tile", "few 4 + few", "few 4 + tile", "few 1 + tile", "few 1 + few",
                     "blocks few 1", "blocks few 4", "blocks few 8", "blocks walk"}
    assert joined == set(itertools.product((False, True), (0, 1)))


def test_every_key_is_walked_once(lib):
    c = (C.c_int * 6)()
    lib.constants(c)
    few, tile, keys, entries, walk, window = c
    rng = random.Random(1)
    for _ in range(3000):
        nkv = rng.choice((1, 2, 8))
        group, page = rng.choice((1, 2, 3, 4, 7, 16, 40)), rng.choice((16, 32, 64, 128, 256))
        n_seqs = int(2 ** rng.uniform(0, 12))
        max_tokens = rng.choice((1, 1, 2, int(2 ** rng.uniform(0, 10))))
        starts = max_tokens > 1 or rng.random() < 0.3
        new = [rng.randint(0, max_tokens) for _ in range(n_seqs)] if starts else [1] * n_seqs
        n_tokens = sum(new) + (rng.randint(0, 5) if starts else 0)
        if max(new) == 0 or max_tokens > n_tokens:
            continue
        length = rng.choice((0, int(2 ** rng.uniform(0, 20))))
        prefix = rng.choice((0, 0, int(2 ** rng.uniform(0, 16))))
        nb = rng.choice((0, 0, rng.randint(1, 1024)))
        if nb:
            prefix = 0
        parts, own, pre, size = _plan(lib, n_seqs, n_tokens, max_tokens, length, prefix, nb, page, group * nkv, nkv, 64, starts)
        # the parts and the workspace
        n = own.splits + (pre.splits if pre.tiles else 0)
        assert parts == (n if n > 1 else 0)
        assert size == parts * n_tokens * group * nkv * (64 + 2) * 4
        # the keys: splits of chunks cover them, and none starts past them
        pages = -(-length // page)
        for launch, shared, mine in ((own, 0 if pre.tiles else prefix, True), (pre, prefix, False)):
            if not launch.tiles:
                continue
            if nb and not launch.few:
                steps = -(-pages // window)
            elif nb:
                steps = nb
            elif launch.few:
                steps = -(-shared // page) + (pages if mine else 0)
            else:
                steps = -(-shared // keys) + (-(-length // keys) if mine else 0)
            steps = max(steps, 1)
            assert launch.splits * launch.chunk >= steps > (launch.splits - 1) * launch.chunk
            if launch.few:
                assert launch.chunk <= entries
        # the vectors: every tile that a sequence needs is there
        of = walk if nb and not own.few else few if own.few else tile
        if nb and own.few:
            assert own.per_seq * of >= group and own.tiles == n_tokens * own.per_seq
        elif own.per_seq:
            assert own.per_seq * of >= max_tokens * group and own.tiles == n_seqs * own.per_seq
        else:
            at = 0
            for s, k in enumerate(new):
                base, after = at * group // of + s, (at + k) * group // of + s + 1
                assert after - base >= -(-k * group // of) and after <= own.tiles
                at += k
        if pre.tiles:
            assert pre.tiles * (few if pre.few else tile) >= n_tokens * group
            assert own.few and own.waves in (1, 4)  # they share a launch of four waves a workgroup
