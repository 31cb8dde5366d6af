"""The serving operators' argument checks (before any device call) and the
64-bit definitions the GPU tests use, on the CPU."""
import ctypes
import math
import os

import pytest
import torch

import serveref as R
from paper_2609_39361_amd import lamp

P = ctypes.c_void_p
OK, INVALID, UNSUPPORTED = 0, 1, 2

pytestmark = pytest.mark.skipif(not os.path.exists(lamp.LIB_PATH), reason="liblamp.so not built")


def _err():
    return lamp.lib().lamp_last_error().decode()


def _rows(q=(4096, 512, 128, 64, 4), k=(4096, 512, 128, 64, 2), v=(4096, 512, 128, 64, 2)):
    return lamp._ROWS3.pack(*q, *k, *v)


def _norm(rin=None, rout=None, B=1, N=3, d=64, f32=0, qw=4096, kw=4096, bits=0, rope=4096, npos=8, rot=64, pos=None, eps=1e-6):
    return lamp.lib().lamp_qk_norm_rope(rin or _rows(), rout or _rows(), B, N, d, f32, P(qw), P(kw), bits, P(rope), npos, rot,
                                        pos, eps, None)


def test_norm_rope_refusals():
    assert lamp.lib().lamp_qk_norm_rope(None, None, 1, 1, 64, 0, None, None, 0, None, 0, 0, None, 1e-6, None) == INVALID
    assert _norm(d=96) == UNSUPPORTED and "96" in _err()
    assert _norm(B=-1) == INVALID
    for rot in (0, -16, 8, 24, 80):
        assert _norm(rot=rot) == INVALID and "rot" in _err()
    assert _norm(npos=0) == INVALID and "npos" in _err()
    assert _norm(rope=4100) == INVALID and "16 bytes" in _err()
    assert _norm(qw=4098) == INVALID and "gains" in _err()
    assert _norm(bits=4) == INVALID and "gain_f32" in _err()
    for eps in (-1.0, math.inf, math.nan):
        assert _norm(eps=eps) == INVALID and "eps" in _err()
    assert _norm(rin=_rows(q=(0, 512, 128, 64, 4))) == INVALID and "null" in _err()
    assert _norm(rin=_rows(q=(4104, 512, 128, 64, 4))) == INVALID and "q: rows" in _err()
    assert _norm(rin=_rows(k=(4096, 512, 132, 64, 2))) == INVALID and "k: rows" in _err()
    assert _norm(rout=_rows(v=(4096, 512, 128, 60, 2))) == INVALID and "v: rows" in _err()
    assert _norm(rout=_rows(q=(4096, 512, 128, 0, 4))) == INVALID and "share" in _err()
    assert _norm(rout=_rows(k=(4096, 512, 0, 64, 2))) == INVALID and "share" in _err()
    assert _norm(rin=_rows(k=(4096, 512, 128, 64, 3))) == INVALID and "heads" in _err()
    assert _norm(B=1 << 13, N=1 << 13) == UNSUPPORTED
    # nothing to do
    assert _norm(B=0) == OK and _norm(N=0) == OK
    z = _rows((0, 0, 0, 0, 0), (0, 0, 0, 0, 0), (0, 0, 0, 0, 0))
    assert _norm(rin=z, rout=z) == OK


def _cache(k=4096, v=4096, ks=4096, vs=4096, pages=4, H=2, page=64, d=64):
    return lamp._CACHE.pack(k, v, ks, vs, pages, H, page, d)


def _batch(table=4096, stride=4, kv=4096, st=4096, S=2, T=5, width=4):
    return lamp._BATCH.pack(table, stride, kv, st, S, T, width)


def _append(c=None, b=None, k=4096, v=4096, f32=0, strides=(128, 64, 128, 64), w=4096, rope=4096, npos=8, rot=64, eps=1e-6):
    return lamp.lib().lamp_kv_append(P(k), P(v), f32, *strides, c or _cache(), b or _batch(), P(w), 0,
                                     P(rope), npos, rot, eps, None)


def _attn(c=None, b=None, q=4096, strides=(256, 64), Hq=4, causal=1, window=0, scale=0.125, o=4096, lse=4096, ws=None, n=0):
    return lamp.lib().lamp_attn_cache(P(q), *strides, Hq, c or _cache(), b or _batch(), causal, window,
                                      scale, P(o), P(lse), ws, n, None)


@pytest.mark.parametrize("call", [_append, _attn])
def test_cache_and_batch_refusals(call):
    assert call(c=_cache(d=80)) == UNSUPPORTED
    for page in (0, 8, 48, 512, -64):
        assert call(c=_cache(page=page)) == UNSUPPORTED and "page" in _err()
    assert call(c=_cache(pages=0)) == INVALID
    assert call(c=_cache(H=0)) == INVALID
    assert call(c=_cache(H=70000), b=_batch(S=1)) == UNSUPPORTED
    for part in ("k", "v", "ks", "vs"):
        assert call(c=_cache(**{part: 0})) == INVALID and "null" in _err()
    assert call(c=_cache(k=4104)) == INVALID and call(c=_cache(v=4100)) == INVALID
    assert call(b=_batch(S=-1)) == INVALID and call(b=_batch(T=-1)) == INVALID and call(b=_batch(width=-1)) == INVALID
    assert call(b=_batch(st=0)) == INVALID and "q_start" in _err()   # T != S
    assert call(b=_batch(table=0)) == INVALID and call(b=_batch(kv=0)) == INVALID
    assert call(b=_batch(T=(1 << 23) + 1)) == UNSUPPORTED
    assert call(b=_batch(S=1 << 22)) == UNSUPPORTED
    assert call(b=_batch(S=(1 << 19) + 1)) == UNSUPPORTED and "S*Hkv" in _err()   # (2 heads)
    assert call(b=_batch(width=(1 << 24) + 1)) == UNSUPPORTED
    assert call(b=_batch(S=0, st=0, T=0)) == OK and call(b=_batch(T=0)) == OK


def test_append_refusals():
    assert _append(k=0) == INVALID and _append(v=4100) == INVALID
    assert _append(strides=(128, 60, 128, 64)) == INVALID and "k: rows" in _err()
    assert _append(strides=(128, 64, 100, 64)) == INVALID and "v: rows" in _err()
    assert _append(w=4100) == INVALID and "gain" in _err()
    assert _append(rot=72) == INVALID and _append(rot=40) == INVALID and _append(eps=-1.0) == INVALID


def test_attention_refusals():
    assert _attn(Hq=3) == INVALID and "multiple" in _err()
    assert _attn(Hq=0) == INVALID
    assert _attn(causal=2) == INVALID and _attn(window=-1) == INVALID
    assert _attn(causal=0, window=4) == INVALID and "window" in _err()
    assert _attn(scale=math.inf) == INVALID and _attn(scale=math.nan) == INVALID
    assert _attn(scale=1e39) == INVALID and _attn(scale=-3e38) == INVALID   # (times log2 e, in fp32)
    assert _attn(q=0) == INVALID and _attn(o=0) == INVALID and _attn(lse=0) == INVALID and _attn(o=4104) == INVALID
    assert _attn(strides=(250, 64)) == INVALID and "q: rows" in _err()
    assert _attn(b=_batch(T=1 << 22), Hq=64) == UNSUPPORTED


def test_attention_workspace_size():
    size = lamp.attn_cache_workspace_size
    assert size(1, 1, 32, 8, 128, 64, 4) == 0          # one piece at most
    assert size(1, 1, 32, 8, 128, 64, 7) == 0 and size(1, 1, 32, 8, 128, 64, 8) > 0   # (4 tiles of 64 keys a piece at least)
    assert size(0, 1, 32, 8, 128, 64, 500) == 0 and size(1, 1, 3, 2, 128, 64, 500) == 0
    assert size(1, 1, 32, 8, 96, 64, 500) == 0 and size(1, 1, 32, 8, 128, 48, 500) == 0
    assert size(1, 1, 32, 8, 128, 256, 1 << 23) == 0
    # more than 256 sequences: where each starts in the plan (8 bytes a sequence; one form here), each part from a multiple of 256
    assert size(256, 256, 32, 8, 128, 64, 1) == 0
    assert size(257, 257, 32, 8, 128, 64, 1) == 256 + 256 * math.ceil(257 * 8 / 256)
    # bounded whatever the batch: at most 512 partial outputs of 256 rows and 1024 of 16, each of d + 2 numbers, what names them, and the plan
    assert size(1 << 20, 1 << 10, 64, 8, 256, 256, 1 << 12) <= (512 * 256 + 1024 * 16) * 258 * 4 + 1536 * 32 + 8 * 256 + 2 * 8 * 1024


def test_binding_refuses_cpu_tensors():
    x = torch.zeros(2, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        lamp.qk_norm_rope(x)
    cache = lamp.kv_cache(2, 2, 64, 16, device="cpu")
    assert cache.k.shape == (2, 2, 16, 64) and cache.v.shape == (2, 2, 64, 16) and cache.k.dtype == torch.float8_e4m3fn
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError):
        lamp.kv_append(x, x, cache, i[:, None], i)
    with pytest.raises(ValueError):
        lamp.attn_cache(x, cache, i[:, None], i)


def test_rope_table():
    t = lamp.rope_table(10, 64, 1e4, device="cpu")
    assert t.shape == (10, 64) and t.dtype == torch.float32
    for p, i in ((0, 0), (9, 0), (7, 31)):
        a = p * 1e4 ** (-2.0 * i / 64)
        assert abs(float(t[p, i]) - math.cos(a)) < 1e-7 and abs(float(t[p, 32 + i]) - math.sin(a)) < 1e-7


def test_reference_e4m3_and_scale():
    codes = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    assert torch.equal(R.e4m3(codes), codes)
    mid = (codes[1:] + codes[:-1]) / 2
    even = torch.where(torch.arange(126) % 2 == 0, codes[:-1], codes[1:])
    assert torch.equal(R.e4m3(mid), even)
    for x, s in ((448.0, 1.0), (448.1, 2.0), (1.0, 2.0 ** -8), (0.0, 2.0 ** -100), (1.75, 2.0 ** -8), (1.76, 2.0 ** -7)):
        assert R.need_scale(torch.tensor([x, math.nan, -math.inf])) == s


def test_reference_attention_of_one_key():
    g = torch.Generator().manual_seed(0)
    parts = R.random_cache(2, 1, 16, 64, g)
    q = torch.randn(1, 2, 64, generator=g)
    ref = R.Cache(*parts)
    o, lse, _, _ = R.attention(q, ref, torch.tensor([[1]]), [1], [0, 1], 16)
    assert torch.allclose(o[0, 0], ref.v[1, 0, :, 0] * ref.vs[1, 0])
    assert torch.allclose(lse[0, 1], (q[0, 1].double() * ref.k[1, 0, 0]).sum() * ref.ks[1, 0] / 8)
