"""The argument checks of the operators of long contexts and changing batches
(before any device call), and the plain arithmetic the GPU tests use, on the CPU."""
import math
import os

import pytest
import torch

import longref as Q
from paper_2609_39361_amd import lamp
from test_serve_host import INVALID, OK, P, UNSUPPORTED, _batch, _cache, _err

pytestmark = pytest.mark.skipif(not os.path.exists(lamp.LIB_PATH), reason="liblamp.so not built")


def _bounds(c=None, b=None, bounds=4096):
    return lamp.lib().lamp_kv_bounds(c or _cache(), b or _batch(), P(bounds), None)


def _select(c=None, b=None, q=4096, strides=(256, 64), Hq=4, bounds=4096, budget=4, first=1, last=2, out=4096, ws=None, n=0):
    return lamp.lib().lamp_select_pages(P(q), *strides, Hq, c or _cache(), b or _batch(), P(bounds), budget, first, last, P(out), ws, n, None)


def _pages(c=None, b=None, q=4096, strides=(256, 64), Hq=4, places=4096, budget=4, scale=0.125, o=4096, lse=4096, ws=None, n=0):
    return lamp.lib().lamp_attn_pages(P(q), *strides, Hq, c or _cache(), b or _batch(), P(places), budget, scale, P(o), P(lse), ws, n, None)


def _shared(c=None, b=None, q=4096, strides=(256, 64), Hq=4, prefix=4096, start=4096, groups=1, scale=0.125, o=4096, lse=4096, ws=None, n=0):
    return lamp.lib().lamp_attn_shared(P(q), *strides, Hq, c or _cache(), b or _batch(), P(prefix), P(start), groups, scale, P(o), P(lse), ws, n,
                                       None)


def _advance(lens=4096, add=4096, prefix=4096, table=4096, stride=4, S=3, width=4, page=64, T=9, ring=4096, pages=8, state=4096, kv=4096, st=4096,
             pos=4096, out=4096):
    return lamp.lib().lamp_kv_advance(P(lens), P(add), P(prefix), P(table), stride, S, width, page, T, P(ring), pages, P(state), P(kv), P(st),
                                      P(pos), P(out), None)


@pytest.mark.parametrize("call", [_bounds, _select, _pages, _shared])
def test_cache_and_batch_refusals(call):
    assert call(c=_cache(d=80)) == UNSUPPORTED
    for page in (0, 8, 48, 512, -64):
        assert call(c=_cache(page=page)) == UNSUPPORTED and "page" in _err()
    assert call(c=_cache(pages=0)) == INVALID and call(c=_cache(H=0)) == INVALID
    for part in ("k", "v", "ks", "vs"):
        assert call(c=_cache(**{part: 0})) == INVALID and "null" in _err()
    assert call(c=_cache(k=4104)) == INVALID
    assert call(b=_batch(S=-1)) == INVALID and call(b=_batch(T=-1)) == INVALID and call(b=_batch(width=-1)) == INVALID
    assert call(b=_batch(st=0)) == INVALID and "q_start" in _err()
    assert call(b=_batch(table=0)) == INVALID and call(b=_batch(kv=0)) == INVALID
    assert call(b=_batch(T=(1 << 23) + 1)) == UNSUPPORTED
    assert call(b=_batch(S=(1 << 19) + 1)) == UNSUPPORTED
    assert call(b=_batch(width=(1 << 24) + 1)) == UNSUPPORTED
    assert call(b=_batch(S=0, st=0, T=0)) == OK and call(b=_batch(T=0)) == OK


@pytest.mark.parametrize("call", [_select, _pages, _shared])
def test_query_refusals(call):
    assert call(Hq=3) == INVALID and "multiple" in _err()
    assert call(Hq=0) == INVALID and call(q=0) == INVALID and call(q=4100) == INVALID
    assert call(strides=(250, 64)) == INVALID and "q: rows" in _err()
    assert call(b=_batch(T=1 << 22), Hq=64) == UNSUPPORTED


@pytest.mark.parametrize("call", [_pages, _shared])
def test_attention_refusals(call):
    for scale in (math.inf, math.nan, 1e39):
        assert call(scale=scale) == INVALID and "scale" in _err()
    assert call(o=0) == INVALID and call(lse=0) == INVALID and call(o=4104) == INVALID


def test_bounds_and_select_refusals():
    assert _bounds(bounds=0) == INVALID and _bounds(bounds=4100) == INVALID and "bounds" in _err()
    assert _select(bounds=0) == INVALID and _select(bounds=4100) == INVALID and _select(out=0) == INVALID
    for budget, first, last in ((0, 0, 0), (-1, 0, 0), (4, -1, 0), (4, 0, -1), (4, 3, 2), (2, 2 ** 31 - 1, 2 ** 31 - 1)):
        assert _select(budget=budget, first=first, last=last) == INVALID and "budget" in _err()
    assert _select(budget=(1 << 20) + 1) == UNSUPPORTED
    assert _select(b=_batch(T=(1 << 22) + 1)) == UNSUPPORTED and "T above" in _err()
    assert _select(b=_batch(T=1 << 22, width=1 << 20)) == UNSUPPORTED and "T*Hkv*width" in _err()
    assert _select(b=_batch(width=5000), budget=4, ws=P(4096), n=8) == 6          # (too small a workspace)
    assert _select(b=_batch(width=5000), budget=4, ws=P(4100), n=1 << 20) == INVALID and "256" in _err()


def test_pages_and_shared_refusals():
    assert _pages(places=0) == INVALID and "places" in _err()
    assert _pages(budget=0) == INVALID and _pages(budget=-3) == INVALID
    assert _pages(budget=(1 << 20) + 1) == UNSUPPORTED
    assert _pages(b=_batch(T=(1 << 12) + 1), budget=1 << 20) == UNSUPPORTED   # (2^24 + 4096)
    assert _pages(b=_batch(T=1 << 12), budget=1 << 20) == UNSUPPORTED and _pages(b=_batch(T=1 << 22), budget=1) == UNSUPPORTED   # (2^24)
    assert _pages(budget=64, ws=P(4096), n=8) == 6
    assert _shared(prefix=0) == INVALID and _shared(start=0) == INVALID
    assert _shared(groups=0) == INVALID and _shared(groups=3) == INVALID and "groups" in _err()   # (of 2 sequences)
    assert _shared(b=_batch(T=(1 << 21) + 1)) == UNSUPPORTED
    assert _shared(ws=P(4096), n=8) == 6


def test_advance_refusals():
    for name in ("lens", "add", "table", "ring", "state", "kv", "st", "pos", "out"):
        assert _advance(**{name: 0}) == INVALID and "null" in _err()
    assert _advance(S=-1) == INVALID and _advance(width=-1) == INVALID and _advance(T=-1) == INVALID and _advance(pages=0) == INVALID
    for page in (0, 8, 48, 512, -16):
        assert _advance(page=page) == UNSUPPORTED and "page" in _err()
    assert _advance(S=(1 << 20) + 1) == UNSUPPORTED and _advance(T=(1 << 23) + 1) == UNSUPPORTED
    assert _advance(width=(1 << 24) + 1) == UNSUPPORTED
    assert _advance(stride=3) == INVALID and _advance(stride=0) == INVALID and "share" in _err()


def test_workspace_sizes():
    size = lamp.select_pages_workspace_size
    assert size(3, 1, 8, 2, 64, 10, 10) == 0 and size(0, 1, 8, 2, 64, 10, 4) == 0 and size(3, 1, 7, 2, 64, 10, 4) == 0
    # scores in LDS, but for rows too long for it, or for a workgroup each
    assert size(3, 1, 8, 2, 64, 10, 4) == 0 and size(300, 300, 8, 2, 128, 512, 4) == 0 and size(300, 300, 8, 2, 64, 1024, 4) == 0
    assert size(300, 300, 8, 2, 128, 513, 4) == 300 * 2 * 513 * 4 and size(1, 1, 8, 2, 128, 513, 4) == 2 * 513 * 4
    assert size(2000, 300, 8, 2, 128, 1024, 4) == 0 and size(2000, 300, 8, 2, 128, 1025, 4) == 2000 * 2 * 1025 * 4
    assert size(1 << 23, 1 << 20, 1, 1, 64, 1 << 20, 4) == 0
    size = lamp.attn_pages_workspace_size
    assert size(2, 4, 3, 64, 16, 4) == 0 and size(1, 4, 2, 80, 16, 4) == 0 and size(1, 4, 2, 64, 24, 4) == 0
    assert size(1, 4, 2, 64, 16, 16) == 0 and size(1, 4, 2, 64, 16, 64) > 0   # (4 tiles of 64 keys a part at least)
    assert size(1, 4, 2, 64, 16, 5000) > 0 and size(1 << 24, 4, 2, 64, 16, 1) == 0
    assert size((1 << 21) - 1, 4, 2, 64, 16, 1025) > 0 and size(1 << 21, 4, 2, 64, 16, 1025) == 0   # (2^24)
    size = lamp.attn_shared_workspace_size
    assert size(1, 1, 2, 4, 2, 64, 16, 4) == 0 and size(1, 1, 0, 4, 2, 64, 16, 4) == 0 and size(1, 1, 1, 4, 2, 64, 16, 4) > 0
    assert size(1 << 22, 1, 1, 4, 2, 64, 16, 4) == 0
    # long tables of many tokens fit the sizes the kernels count in
    assert size(1 << 18, 1 << 10, 1 << 9, 32, 8, 128, 64, 1 << 14) > 0


def test_binding_refusals():
    z = torch.zeros(2, 3, dtype=torch.int32)
    with pytest.raises(ValueError):
        lamp.kv_advance(lamp.kv_pool(4, device="cpu"), z, z[0], z[0], 16, 4)
    with pytest.raises(ValueError):
        lamp.kv_bounds(lamp.kv_cache(2, 1, 64, 16, device="cpu"), None, z, z[0], 2)
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    cache = lamp.kv_cache(2, 1, 64, 16, device="cpu")
    for call in (lambda q: lamp.select_pages(q, cache, None, z, z[0], 4), lambda q: lamp.attn_pages(q, cache, z, z[0], None),
                 lambda q: lamp.attn_shared(q, cache, z, z[0], z[0], z[0])):
        for x in (q, q[0], None):
            with pytest.raises(ValueError):
                call(x)


def test_the_plain_step():
    """Pages are taken in order and given back in order; the ring closes."""
    table = torch.tensor([[4, -1, -1], [1, 2, -1], [-1, -1, -1]], dtype=torch.int32)
    ring = torch.tensor([5, -9, -9, 0, 3], dtype=torch.int32)   # free: 0, 3, 5
    kv, st, pos, state, t, r = Q.advance([16, 20, 0], [1, -1, 17], None, table, 16, 20, ring, [3, 3, 0, 0])
    assert kv == [17, 0, 17] and st == [0, 1, 1, 18] and pos == [16] + list(range(17)) + [0, 0]
    assert t.tolist() == [[4, 0, -1], [1, 2, -1], [3, 5, -1]]
    assert r.tolist() == [5, 1, 2, 0, 3] and state == [1, 2, 3, 0]


def test_the_plain_scores_bound_the_logits():
    """A page's score is at least every product of the rounded query with its keys, in its units."""
    g = torch.Generator().manual_seed(3)
    k = (torch.randn(16, 64, generator=g) * 100).clamp(-448, 448).to(torch.float8_e4m3fn).double()
    q = torch.randn(3, 64, generator=g).to(torch.bfloat16)
    rng = torch.stack([torch.ceil(k.amax(0) / 4), torch.floor(k.amin(0) / 4)]).to(torch.int8)
    x, e = Q.rounded(q)
    assert int(x.abs().max()) in range(64, 128) and float((q.double() - x * 2.0 ** e).abs().max()) <= 2.0 ** (e - 1)
    top = float(Q.scores(q, rng[None], torch.ones(1))[0])
    assert 4 * top >= float((x.double() @ k.T).max()) and top < 2 ** 23
