"""Values at the edges of what the operators of long contexts and changing batches are told: table entries, scales,
sizes."""
import pytest
import torch

from test_gpu_long import _cache_of_scales, _check_select, _i32, _lists, _run_pages, _run_shared, _select_case, _shared_case
from test_gpu_serve import L, _attn_case, _device_cache, _run_attn  # noqa: F401

pytestmark = pytest.mark.gpu

NO_PAGE = [-1, 10 ** 6, 2 ** 31 - 1, -2 ** 31]


@pytest.mark.parametrize("entry", NO_PAGE)
@pytest.mark.parametrize("d,page", [(64, 16), (128, 64), (256, 32)])
def test_attn_cache_every_missing_entry(L, entry, d, page):  # noqa: F811
    """Rows that see a place whose entry is no page are NaN, whatever the entry: single tokens, chunks, and (300 tokens) a
    prompt in the form for many rows."""
    for lens in ([(700, 1), (60, 3)], [(700, 300), (300, 40)]):
        q, parts, table, kv, starts = _attn_case(L, lens, 4, 2, d, page, seed=d)
        table[0, 2] = entry
        for window in (0, 100):
            got = _run_attn(L, q, parts, table, kv, starts, page, 4, window=window)
            assert torch.isnan(got[0][0]).all() == (window == 0) and torch.isfinite(got[0][starts[1]:].float()).all()


@pytest.mark.parametrize("entry", NO_PAGE)
@pytest.mark.parametrize("d,page", [(64, 16), (128, 64), (256, 32)])
def test_attn_pages_every_missing_entry(L, entry, d, page):  # noqa: F811
    q, parts, table, kv, starts = _attn_case(L, [(700, 2), (900, 1)], 4, 2, d, page, seed=d)
    table[0, 2] = entry
    places = _lists(table, kv, starts, 2, page, 5, 1)
    places[0, 0] = torch.tensor([0, 2, 5, -1, -1])
    places[1, 1] = torch.tensor([1, 3, 2, 6, 9])
    places[0, 1, places[0, 1] == 2] = 1
    got = _run_pages(L, (q, parts, table, kv, starts), page, 4, places)
    assert torch.isnan(got[0][0, :2]).all() and torch.isnan(got[0][1, 2:]).all()
    assert torch.isfinite(got[0][0, 2:].float()).all() and torch.isfinite(got[0][2].float()).all()


@pytest.mark.parametrize("entry", NO_PAGE)
@pytest.mark.parametrize("d,page", [(64, 16), (128, 64), (256, 32)])
def test_attn_shared_every_missing_entry(L, entry, d, page):  # noqa: F811
    """Of a prefix, and of one sequence's own keys; in the forms for few rows, for prefixes, and for many rows."""
    for groups in ([(256, [(100, 1), (30, 2)]), (64, [(70, 1)])], [(256, [(100, 260), (30, 2)]), (64, [(70, 1)])]):
        q, parts, table, kv, starts, prefix, gs = _shared_case(groups, 4, 1, d, page, seed=d)
        for places in ((range(2), 128 // page), ((1,), 256 // page)):
            hole = table.clone()
            for s in places[0]:
                hole[s, places[1]] = entry
            got = _run_shared(L, (q, parts, hole, kv, starts, prefix, gs), page)
            assert torch.isnan(got[0][starts[1]:starts[2]]).all() and torch.isfinite(got[0][starts[2]:].float()).all()
            assert torch.isnan(got[0][0]).all() == (len(places[0]) == 2)


@pytest.mark.parametrize("lo,hi", [(100, 120), (-149, -110), (-149, 128), (120, 128)])
@pytest.mark.parametrize("Hq,H,d,keys", [(4, 2, 64, 6000), (1, 1, 256, 4000), (40, 2, 64, 3000), (8, 1, 128, 30000), (34, 1, 128, 17000)])
def test_select_scales_of_the_whole_range(L, Hq, H, d, keys, lo, hi):  # noqa: F811
    """Scores pass fp32's largest number, and its smallest normal one, in order all the same; in one launch and in two."""
    q, rng, ks, table, kv, starts = _select_case([(keys, 2), (keys // 3, 1)], Hq, H, d, 16, hi - lo)
    g = torch.Generator().manual_seed(hi)
    ks = (2.0 ** torch.randint(lo, hi, ks.shape, generator=g).double()).float()
    assert bool((ks > 0).all()) and bool(torch.isfinite(ks).all())
    q[0] *= 0.01
    for budget in (5, 40):
        _check_select(L, (q, rng, ks, table, kv, starts), 16, budget, 1, 1)


def test_sizes_beyond_a_c_int_are_refused(L):  # noqa: F811
    """Not taken by their low 32 bits."""
    q, rng, ks, table, kv, starts = _select_case([(500, 2)], 4, 2, 64, 16, 3)
    cache = _cache_of_scales(L, ks, 16, 64)
    args = (q.cuda(), cache, rng.cuda(), table.cuda(), _i32(kv))
    out = torch.full((2, 2, 6), -2, dtype=torch.int32, device="cuda")
    for big in (2 ** 32, 2 ** 32 + 1, -2 ** 32, 2 ** 31, -2 ** 31 - 1, 2 ** 64 + 1):
        for kw in (dict(first=big), dict(last=big)):
            with pytest.raises(ValueError):
                L.select_pages(*args, 6, _i32(starts), out=out, **kw)
        with pytest.raises(ValueError):
            L.select_pages(*args, big, _i32(starts))
    assert bool((out == -2).all())
    pool, t, n = L.kv_pool(8), torch.full((2, 4), -1, dtype=torch.int32, device="cuda"), _i32([0, 0])
    for page, tokens in ((2 ** 32 + 16, 4), (16, 2 ** 32 + 4), (-2 ** 32 + 16, 4)):
        with pytest.raises(ValueError):
            L.kv_advance(pool, t, n, _i32([1, 1]), page, tokens, None, (n, _i32([0] * 3), _i32([0] * 4), pool.state))
    assert pool.state.tolist() == [0, 8, 0, 0] and bool((t == -1).all()) and n.tolist() == [0, 0]
    bounds = L.kv_page_bounds(cache)
    with pytest.raises(ValueError):
        L.kv_bounds(cache, bounds, table.cuda(), _i32(kv), 2 ** 32 + 2, _i32(starts))


@pytest.mark.parametrize("d,page", [(64, 256), (128, 64), (256, 16)])
def test_attn_pages_of_the_longest_sequences(L, d, page):  # noqa: F811
    """Entries of a list that hold no keys hold none of a sequence as long as a table reaches (2^30 keys, of a few pages)."""
    q, parts, table, kv, starts = _attn_case(L, [(40 * page, 3)], 4, 2, d, page, seed=d)
    width = 2 ** 30 // page
    long = table[0, torch.arange(width) % 40].unsqueeze(0).contiguous()
    places = torch.full((3, 2, 7), -1, dtype=torch.int32)
    places[0, :, 3] = width - 1
    places[1, 0, :6] = torch.tensor([-1, 5, 2 ** 31 - 1, width - 1, width, width - 2])
    places[1, 1, 6] = 0
    places[2, :, 1:5:2] = torch.tensor([width // 2 + 3, width - 1])
    got = _run_pages(L, (q, parts, long, [2 ** 30], [0, 3]), page, 4, places)
    assert torch.isfinite(got[0].float()).all() and torch.isfinite(got[1]).all()


def test_caches_whose_offsets_pass_32_bits(L):  # noqa: F811
    """The pages of small cases at the end of a cache of 4.6 GB of keys: ranges, selection, attention over places and over a
    shared prefix are those of the small cache."""
    page, H, d, many = 64, 8, 128, 70000
    q, parts, table, kv, starts, prefix, gs = _shared_case([(320, [(100, 2), (30, 1)]), (0, [(700, 1), (5, 90)])], 16, H, d, page, seed=3)
    small = _device_cache(L, parts)
    n = parts[0].shape[0]
    assert (many - n) * H * page * d > 2 ** 32
    big = L.kv_cache(many, H, d, page)
    for x, y in zip(big, small):
        x[many - n:] = y
    far = torch.where(table >= 0, table + many - n, table).cuda()
    args = _i32(kv), _i32(starts)
    got = []
    for cache, tab in ((small, table.cuda()), (big, far)):
        rng = L.kv_bounds(cache, L.kv_page_bounds(cache), tab, args[0], starts[-1], args[1])
        rng = L.kv_bounds(cache, rng, tab, args[0], sum(kv), _i32([0, *torch.tensor(kv).cumsum(0).tolist()]))   # (every key as new)
        places = L.select_pages(q.cuda(), cache, rng, tab, args[0], 4, args[1])
        got.append((rng[-n:], places, *L.attn_pages(q.cuda(), cache, tab, args[0], places, args[1]),
                    *L.attn_shared(q.cuda(), cache, tab, args[0], _i32(prefix), _i32(gs), args[1])))
    assert bool(got[0][0].any()) and bool((got[0][1] >= 0).any())
    for x, y in zip(*got):
        assert torch.equal(x, y)
    _run_shared(L, (q, parts, table, kv, starts, prefix, gs), page)
