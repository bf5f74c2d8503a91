"""Keys that change lanes through a wave's own LDS: the hardware keeps such accesses in order, the compiler
only where a fence says so.  This reads the intermediate code of every instance of the hand-over, before any
optimisation."""
import os
import re
import subprocess

import pytest

from paper_2606_31808_amd import build


@pytest.fixture(scope="module")
def functions(tmp_path_factory):
    if not os.path.exists(build.HIPCC):
        pytest.skip("no hipcc")
    out = tmp_path_factory.mktemp("ir") / "paged_attention.ll"
    subprocess.run([build.HIPCC, *build.FLAGS, "-x", "hip", "--offload-device-only", "-O1", "-Xclang", "-disable-llvm-passes",
                    "-emit-llvm", "-S", os.path.join(build.CSRC, "paged_attention.hip"), "-o", str(out)],
                   check=True, capture_output=True)
    return dict(re.findall(r"^define [^@]*@(\w+)\([^\n]*\{\n(.*?)^\}", out.read_text(), re.M | re.S))


def test_the_order_is_a_fence(functions):
    body = [b for n, b in functions.items() if "wave_order" in n]
    assert len(body) == 1
    assert 'fence syncscope("wavefront") acq_rel' in body[0] and "llvm.amdgcn.wave.barrier" in body[0]


def test_hand_over_is_ordered(functions):
    """Both sides of the writes: behind the reads of the chunk before, ahead of this one's."""
    hand_overs = {n: b for n, b in functions.items() if "stash_keys" in n}
    assert len(hand_overs) == 16  # two types, two kinds of pages, two head sizes, 16 and 32 vectors
    for name, body in hand_overs.items():
        calls = re.findall(r"call [^@\n]*@(\w+)\(", body)
        order = [i for i, c in enumerate(calls) if "wave_order" in c]
        writes = [i for i, c in enumerate(calls) if "key_at" in c]
        assert writes and len(order) == 2 and order[0] < writes[0] and writes[-1] < order[1], name
