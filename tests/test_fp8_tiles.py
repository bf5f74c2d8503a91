"""The block-scaled FP8 product's rule on the host: the sizes that the GPU tests
run take every kernel it offers, and it is never far from the fastest one."""
import ctypes as C
import os
import re
import shutil
import subprocess

import pytest
import torch

from paper_2606_31808_amd import build
from tests import test_gpu_operators as gpu

SRC = """
#include "fp8_tiles.h"
extern "C" int pick(int f32, int m, int n, int k) { return lmop::pick_fp8_kernel(f32, m, n, k); }
extern "C" int kernels() { return lmop::kNumFp8Kernels; }
"""


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    if not shutil.which("g++"):
        pytest.skip("no g++")
    d = tmp_path_factory.mktemp("rule")
    (d / "r.cpp").write_text(SRC)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", f"-I{build.CSRC}",
                    str(d / "r.cpp"), "-o", str(d / "r.so")], check=True)
    return C.CDLL(str(d / "r.so"))


@pytest.mark.parametrize("f32", [0, 1])
def test_gpu_sizes_take_every_kernel(rule, f32):
    taken = {rule.pick(f32, m, n, k) for m, n, k in gpu.SIZES + gpu.LARGE}
    assert taken == set(range(f32, rule.kernels()))  # the largest tile is for 16-bit results


# us by kernel: 0 256x256, 1 128x256, 2 64x128, 3 64x64, 4 32x64, 5 and 6 few tokens
MEASURED = [
    (0, 1, 6144, 4096, {3: 12.4, 5: 8.5, 6: 10.2}),
    (0, 16, 6144, 4096, {3: 12.9, 4: 11.8, 5: 11.7, 6: 12.7}),
    (0, 24, 6144, 4096, {3: 13.1, 4: 12.1, 6: 14.6}),
    (0, 64, 6144, 4096, {2: 20.3, 3: 14.6, 4: 12.3}),
    (0, 256, 6144, 4096, {2: 19.9, 3: 21.9, 4: 26.1}),
    (0, 1, 4096, 14336, {3: 35.8, 5: 12.9, 6: 15.5}),
    (0, 16, 4096, 14336, {3: 37.7, 4: 32.3, 5: 18.6, 6: 20.0}),
    (1, 24, 4096, 14336, {3: 53.2, 4: 49.8, 6: 24.5}),
    (0, 128, 4096, 14336, {2: 59.9, 3: 42.3, 4: 32.8}),
    (0, 256, 4096, 14336, {2: 58.7, 3: 42.8, 4: 50.8}),
    (0, 1, 28672, 4096, {3: 26.8, 5: 22.7, 6: 29.5}),
    (0, 16, 28672, 4096, {2: 28.6, 3: 27.2, 4: 26.6, 5: 35.6}),
    (0, 128, 28672, 4096, {2: 41.2, 3: 46.6, 4: 57.8}),
    (0, 24, 2048, 2048, {3: 7.2, 4: 7.0, 6: 5.1}),
    (0, 64, 768, 6272, {2: 22.0, 3: 16.2, 4: 15.2, 6: 11.8}),
    (1, 64, 768, 6272, {2: 36.0, 3: 24.5, 4: 22.9, 6: 12.3}),
    (0, 64, 2048, 4096, {2: 15.3, 3: 11.5, 4: 10.9, 6: 8.4}),
    (1, 64, 2048, 4096, {2: 24.9, 3: 17.3, 4: 16.2, 6: 8.8}),
    (0, 48, 1536, 14336, {2: 57.4, 3: 40.1, 4: 32.2, 6: 23.3}),
    (0, 48, 4096, 4096, {2: 18.7, 3: 13.4, 4: 11.6, 6: 14.3}),
    (1, 48, 4096, 4096, {2: 26.0, 3: 17.8, 4: 16.8, 6: 14.6}),
    (0, 128, 768, 4096, {2: 15.3, 3: 11.5, 4: 10.9, 6: 8.3}),
    (1, 128, 768, 4096, {2: 24.9, 3: 17.3, 4: 16.2, 6: 8.7}),
    (0, 128, 2048, 2048, {2: 9.1, 3: 7.2, 4: 7.0, 6: 8.3}),
    (0, 512, 4096, 4096, {0: 60.1, 1: 35.5, 2: 19.4, 3: 21.2}),
    (1, 256, 4096, 4096, {1: 53.4, 2: 26.6, 3: 18.4, 4: 24.0}),
    (1, 512, 4096, 4096, {1: 54.2, 2: 27.4, 3: 27.3, 4: 43.9}),
    (0, 2047, 4096, 4096, {0: 62.5, 1: 41.7, 2: 57.6, 3: 72.7}),
    (1, 2047, 4096, 4096, {1: 62.5, 2: 81.0, 3: 95.8}),
    (1, 16384, 4096, 14336, {1: 1526.0, 2: 1926.0, 3: 2363.0}),
    (0, 4096, 16384, 2048, {0: 123.0, 1: 146.0}),
    (0, 16384, 4096, 14336, {0: 772.0, 1: 902.0, 2: 1266.0}),
    (0, 16384, 28672, 4096, {0: 1645.0, 1: 1868.0, 2: 2600.8}),
]


@pytest.mark.parametrize("f32,m,n,k,us", MEASURED)
def test_pick_is_near_the_fastest(rule, f32, m, n, k, us):
    pick = rule.pick(f32, m, n, k)
    assert pick in us, pick
    assert us[pick] <= 1.1 * min(us.values())


def test_rule_is_defined_at_the_limits(rule):
    for f32 in (0, 1):
        for m, n, k in ((1, 1, 1), (2 ** 30, 16, 1), (16, 2 ** 30, 1), (1, 1, 2 ** 23),
                        (2 ** 19, 2 ** 19, 2 ** 23)):
            assert f32 <= rule.pick(f32, m, n, k) < rule.kernels()


def test_helpers_keep_the_wait_state(tmp_path):
    """The masked 4-byte load has an instruction between its write of M0 and the load."""
    if not os.path.exists(build.HIPCC):
        pytest.skip("no hipcc")
    src, out = tmp_path / "p.hip", tmp_path / "p.s"
    src.write_text('#include "lds_dma4.h"\nusing namespace lmop;\nextern "C" __global__ void probe('
                   "const char* a, unsigned off, unsigned lds, unsigned long m) {\n"
                   "  g2l4_m0_mask(a, off * threadIdx.x, lds, m);\n}\n")
    subprocess.run([build.HIPCC, *build.FLAGS, "-x", "hip", "--offload-device-only", "-S", str(src),
                    "-o", str(out)], check=True, capture_output=True)
    lines = [l.split(";")[0].strip() for l in out.read_text().splitlines()]
    lines = [l for l in lines if l and not l.startswith(".")]
    at = next(i for i, l in enumerate(lines) if l.startswith("global_load_lds_dword "))
    assert re.match(r"s_\w+ m0,", lines[at - 2]) and not re.match(r"s_\w+ m0,", lines[at - 1])
    assert lines[at + 1].startswith("s_mov_b64 exec, -1")


LIMITS = """
#include "fp8_tiles.h"
extern "C" int pick(int f32, int m, int n, int k) { return lmop::pick_fp8_kernel(f32, m, n, k); }
extern "C" int rows(int kernel, int m, int n) { return lmop::fp8_rows(kernel, m, n); }
extern "C" void group(int kernel, int* out) {
  const lmop::Fp8Group g = lmop::fp8_group(kernel);
  out[0] = g.bm, out[1] = g.bn, out[2] = g.threads;
}
"""


def test_every_launch_is_one_that_hip_makes(tmp_path):
    """The launches of a call have fewer than 2^32 threads each and whole tiles, for the kernel
    that the rule picks, at sizes up to the accepted limits (2^30 tiles of 16 x 16)."""
    if not shutil.which("g++"):
        pytest.skip("no g++")
    (tmp_path / "l.cpp").write_text(LIMITS)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", f"-I{build.CSRC}",
                    str(tmp_path / "l.cpp"), "-o", str(tmp_path / "l.so")], check=True)
    lib, out = C.CDLL(str(tmp_path / "l.so")), (C.c_int * 3)()
    ends = [2 ** i + d for i in range(30) for d in (-1, 0, 1)] + [2 ** 30 - 1, 2 ** 30]
    ends = sorted({x for x in ends if x > 0})
    several = 0
    for f32 in (0, 1):
        for k in (1, 128, 4096, 14336, 2 ** 23):
            for n in ends:
                # every order of magnitude of tokens that is accepted beside n columns
                most = min(2 ** 30, (2 ** 30 // -(-n // 16)) * 16)
                for m in {1, 16, 17, 32, 33, 64, 300, 2000, most // 3, most - 1, most}:
                    if not 0 < m <= most:
                        continue
                    kernel = lib.pick(f32, m, n, k)
                    lib.group(kernel, out)
                    bm, bn, threads = out
                    rows = lib.rows(kernel, m, n)
                    assert 0 < rows <= m and (rows == m or rows % bm == 0), (m, n, k, kernel)
                    assert -(-rows // bm) * -(-n // bn) * threads < 2 ** 32, (m, n, k, kernel)
                    # what fits is one launch
                    assert rows == m or -(-m // bm) * -(-n // bn) * threads >= 2 ** 32
                    several += rows != m
    assert several


@pytest.mark.parametrize("big", [False, True])
def test_what_the_cut_of_products_costs(big):
    """The 8-bit instruction's cut (which a GPU test pins to the bit) on unit-normal tokens and
    weights, and with a feature in a hundred ten times as large.  Of eight products seven lose
    up to u = 2^-13 of the largest p, of either sign: 7 u off at most, and u / sqrt(3) each in
    the root mean square if what is cut off is spread evenly."""
    g, (m, n, k) = torch.Generator().manual_seed(7), (48, 128, 1024)
    x = torch.randn(m, k, generator=g)
    if big:
        x *= torch.where(torch.rand(k, generator=g) < 0.01, 10.0, 1.0)
    groups = x.view(m, -1, gpu.G)
    sa = groups.abs().amax(-1) / 448
    a = (groups / sa[..., None]).view(m, k).to(gpu.F8)
    w = torch.randn(n, k, generator=g).view(n, -1, gpu.G)
    sb = (w.abs().amax((0, 2)) / 448)[None]
    b = (w / sb[..., None]).view(n, k).to(gpu.F8)
    off = gpu._cut_product(a, sa, b, sb)[0].double()
    whole, _, largest = gpu._ref_matmul(a, sa, b, sb)
    off -= whole
    assert torch.all(off.abs() <= 7 * 2.0 ** -13 * largest)
    p = [t.float().double().abs().view(t.shape[0], -1, 8).amax(-1) * s.double().repeat_interleave(16, 1)
         for t, s in ((a, sa), (b, sb))]
    rms = (7 / 3) ** 0.5 * 2.0 ** -13 * ((p[0] ** 2) @ (p[1] ** 2).t()).sum() ** 0.5
    print(f"off by {off.norm() / whole.norm():.2e} of the norm, bound {rms / whole.norm():.2e}")
    assert 1e-5 * whole.norm() < off.norm() <= rms
