"""The serving operators' binding and argument checks at their edges, on the
CPU (nothing is launched)."""
import ctypes
import os
import subprocess
import sys

import pytest
import torch

from paper_2609_39361_amd import lamp

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.skipif(not os.path.exists(lamp.LIB_PATH), reason="liblamp.so not built")


@pytest.mark.parametrize("shape", [(0, 64), (4, 0), (0, 0)])
def test_an_empty_rope_table_is_refused(shape):
    """(An empty tensor has no address, which the library takes as "not rotated".)"""
    with pytest.raises(ValueError, match="rope"):
        lamp._rope(torch.empty(shape), -1)
    with pytest.raises(ValueError, match="rope"):
        lamp._rope(torch.ones(4, 64)[:shape[0], :shape[1]].contiguous(), -1)
    assert lamp._rope(None, -1) == (None, 0, 0)


def test_workspace_size_of_tables_without_columns():
    """attn_cache accepts them, so the size says what such a call needs: the plan of more than 256 sequences."""
    size = lamp.attn_cache_workspace_size
    assert size(256, 256, 4, 1, 64, 16, 0) == 0 and size(3, 2, 4, 1, 64, 16, 0) == 0
    assert size(300, 300, 4, 1, 64, 16, 0) == size(300, 300, 4, 1, 64, 16, 1) > 0
    assert size(300, 300, 4, 1, 64, 16, -1) == 0


@pytest.mark.parametrize("eps,ok", [(1e39, False), (1e308, False), (1e-50, False), (0.0, True), (1e-45, True), (3.4e38, True)])
def test_eps_is_an_fp32_number(eps, ok):
    """The kernels hold it in fp32: one that is infinite there would make every row 0, one that vanishes zero rows NaN.
    (No tokens: the checks alone.)"""
    rows, L, P = lamp._ROWS3.pack(*(4096, 512, 128, 64, 2) * 3), lamp.lib(), ctypes.c_void_p
    rc = [L.lamp_qk_norm_rope(rows, rows, 1, 0, 64, 0, None, None, 0, None, 0, 0, None, eps, None),
          L.lamp_kv_append(None, None, 0, 128, 64, 128, 64, lamp._CACHE.pack(4096, 4096, 4096, 4096, 4, 2, 64, 64),
                           lamp._BATCH.pack(4096, 4, 4096, 4096, 2, 0, 4), P(4096), 0, None, 0, 0, eps, None)]
    assert rc == ([0, 0] if ok else [1, 1])
    assert ok or "eps" in L.lamp_last_error().decode()


def test_the_binding_imports_with_a_torch_without_a_gpu_build():
    """Whose torch._C has none of the calls behind the current stream and device; with one, the public calls do."""
    code = """
import torch
for name in ("_cuda_getCurrentRawStream", "_cuda_getDevice"):
    if hasattr(torch._C, name):
        delattr(torch._C, name)
from paper_2609_39361_amd import lamp
assert lamp.rope_table(4, 16, device="cpu").shape == (4, 16)
assert lamp._current_device is torch.cuda.current_device
class Stream:
    cuda_stream = 7
torch.cuda.current_stream = lambda dev: Stream
assert lamp._raw_stream(0) == 7
"""
    subprocess.run([sys.executable, "-c", code], check=True, cwd=ROOT)


def test_workspace_size_of_a_chunk_among_many_tokens():
    """A long chunk beside many single tokens is held by the form for many rows, whose partial outputs the workspace has,
    though the batch has few rows a sequence on average; single tokens and short tables need none of them."""
    size = lamp.attn_cache_workspace_size
    few = 1024 * 16 * 130 * 4 + 2048 * 40   # (1024 partial outputs of 16 rows, d + 2 numbers each, and what names them)
    for S, chunk, Hq in ((128, 385, 32), (64, 961, 8), (300, 400, 32)):
        rows = (S - 1 + chunk) * (Hq // 8)
        units = (rows // 256 + min(S, rows // 65)) * 8 + 256   # (more than 64 rows each; 256 fill the device)
        assert size(S - 1 + chunk, S, Hq, 8, 128, 64, 470) > min(units, 512) * 256 * 130 * 4
        assert size(S, S, Hq, 8, 128, 64, 470) < few           # (one token each)
        assert size(S - 1 + chunk, S, Hq, 8, 128, 64, 8) < few
    assert size(4 * 32, 32, 32, 8, 128, 64, 16) < few          # (four tokens each)
