"""The order of the LDS accesses by which the lanes of a wave pass data to each other without a barrier
(csrc/lamp_cache_prefix.h), in the compiler's intermediate code: one lane's stores and another's loads are ordered
only by a fence between them."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2609_39361_amd import build as B

FORMS = [(64, 64, 1), (64, 64, 2), (64, 64, 4), (128, 64, 1), (128, 64, 2), (128, 64, 4), (256, 32, 1), (256, 32, 2)]

SOURCE = '#include "lamp_cache_prefix.h"\nnamespace lamp {\n' + "".join(
    "__global__ __launch_bounds__(256, 2) void form_%d_%d_%d(SharedAttnParams p)\n{\n"
    "    __shared__ PrefixShared<%d, %d> sh;\n    cache_prefix<%d, %d, %d>(p, (int)blockIdx.x, sh);\n}\n"
    % (d, kt, n, d, kt, d, kt, n) for d, kt, n in FORMS) + "}\n"


def _unordered(events):
    """Whether a load follows a store, or a store a load, without a fence between; events of a loop's body, repeated."""
    before = set()
    for e in events + events:
        if e == "fence":
            before = set()
        else:
            if {"load": "store", "store": "load"}[e] in before:
                return True
            before.add(e)
    return False


def test_the_rule():
    assert _unordered(["store", "load"]) and _unordered(["store", "fence", "load"]) and _unordered(["fence", "store", "store", "load", "fence"])
    assert not _unordered(["store", "store", "fence", "load", "fence"]) and not _unordered(["fence", "store", "fence", "load"])


@pytest.mark.skipif(not (os.path.exists(B.HIPCC) or shutil.which(B.HIPCC)), reason="no hipcc")
def test_lanes_of_a_wave_see_what_the_others_stored(tmp_path):
    src, ir = tmp_path / "forms.hip", tmp_path / "forms.ll"
    src.write_text(SOURCE)
    subprocess.run([B.HIPCC, "--offload-arch=" + B.ARCH, "-O2", "-std=c++17", "-ffp-contract=off", "-I", os.path.join(B.ROOT, "include"),
                    "-I", B.CSRC, "--cuda-device-only", "-emit-llvm", "-S", str(src), "-o", str(ir)], check=True, capture_output=True)
    bodies = re.findall(r"^define [^\n]*form_(\d+)_(\d+)_(\d+)[^\n]*\{\n(.*?)^\}", ir.read_text(), re.S | re.M)
    assert sorted(tuple(int(x) for x in b[:3]) for b in bodies) == FORMS
    for *name, body in bodies:
        # between barriers of the workgroup: the part with the tiles' loop
        parts = []
        for part in re.split(r"@llvm\.amdgcn\.s\.barrier", body):
            events = []
            for line in part.splitlines():
                if re.search(r"\bfence syncscope\(\"wavefront\"\)", line):
                    events.append("fence")
                m = re.search(r"\b(store|load) <4 x i32>.*addrspace\(3\)", line)
                if m:
                    events.append(m.group(1))
            parts.append(events)
        loop = max(parts, key=lambda e: e.count("load"))
        d, kt, _ = (int(x) for x in name)
        assert loop.count("store") == 2 * (kt * d // 1024) and loop.count("load") >= loop.count("store"), name
        assert not _unordered(loop), name
