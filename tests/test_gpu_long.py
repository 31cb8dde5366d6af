"""The operators of long contexts and changing batches on the GPU against plain
arithmetic (longref.py): steps planned on the device, the ranges of pages, the
pages that are selected, the attention over them, and over shared prefixes."""
import math

import pytest
import torch

import longref as Q
import serveref as R
from test_gpu_serve import L, NAN_CODES, _attn_case, _device_cache, _gen, _i32  # noqa: F401

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------- steps

def _pool_case(lens, add, prefix, page, spare, seed, width=None):
    """Tables of `lens` keys (the first prefix // page places the same in all) and a pool of what is left and `spare` more."""
    g = _gen(seed)
    held = [-(-n // page) for n in lens]
    kept = max(prefix or [0]) // page
    need = [max(0, -(-(n + max(0, a)) // page) - h) for n, a, h in zip(lens, add, held)]
    pages = sum(held) + sum(need) + spare + kept
    order = torch.randperm(pages, generator=g).int()
    width = width or max([h + n for h, n in zip(held, need)] + [0]) + 1
    table = torch.full((len(lens), width), -1, dtype=torch.int32)
    at = kept
    for s, h in enumerate(held):
        own = min(h, prefix[s] // page if prefix else 0)
        table[s, :own] = order[:own]
        table[s, own:h] = order[at:at + h - own]
        at += h - own
    head, free = int(torch.randint(0, pages, (1,), generator=g)), order[at:]
    ring = torch.full((pages,), -9, dtype=torch.int32)
    ring[(head + torch.arange(len(free))) % pages] = free
    return table, ring, [head, len(free), 0, 0]


def _check_step(L, lens, add, prefix, page, T, table, ring, state, in_place=False):  # noqa: F811
    want = Q.advance(lens, add, prefix, table, page, T, ring, state)
    td, rd, sd, ld = table.cuda(), ring.cuda(), _i32(state), _i32(lens)
    out = (ld, _i32([-3] * (len(lens) + 1)), _i32([-3] * T), sd) if in_place else None
    kv, st, pos, pool = L.kv_advance(L.KVPool(rd, sd), td, ld, _i32(add), page, T, None if prefix is None else _i32(prefix), out)
    for got, exp, what in ((kv, want[0], "kv_lens"), (st, want[1], "q_start"), (pos, want[2], "positions"), (pool.state, want[3], "state")):
        assert got.tolist() == list(exp), what
    assert torch.equal(td.cpu(), want[4]) and torch.equal(rd.cpu(), want[5])
    if in_place:
        assert kv.data_ptr() == ld.data_ptr() and pool.state.data_ptr() == sd.data_ptr()
    return want


STEPS = [
    # lens, add, prefix, page
    ([0], [1], None, 16),
    ([0], [0], None, 64),
    ([16, 15, 17, 0, 31], [1, 1, 1, 1, 2], None, 16),
    ([100, 64, 0, 7, 128], [-1, 200, 33, 0, -5], None, 64),
    ([64, 64, 70, 200, 64], [1, -1, -1, -1, 0], [64, 64, 64, 64, 64], 32),
    ([300, 0, 10], [-1, 3000, 1], [40, 0, 300], 16),
    ([256, 1000], [20000, -2], None, 256),
]


@pytest.mark.parametrize("i", range(len(STEPS)))
@pytest.mark.parametrize("in_place", [False, True])
def test_advance(L, i, in_place):  # noqa: F811
    lens, add, prefix, page = STEPS[i]
    T = sum(max(0, a) for a in add)
    case = _pool_case(lens, add, prefix, page, 3, i)
    for more in (0, 5):
        assert _check_step(L, lens, add, prefix, page, T + more, *case, in_place=in_place)[3][3] == 0


@pytest.mark.parametrize("S,T", [(1000, 8192), (1024, 8193), (1025, 20000), (5000, 40000), (2049, 9000)])
def test_advance_many(L, S, T):  # noqa: F811
    """More sequences than the workgroup has threads, tokens within one launch and beyond it."""
    g = _gen(S)
    lens = torch.randint(0, 300, (S,), generator=g).tolist()
    add = torch.randint(-1, 5, (S,), generator=g).tolist()
    add[S // 2] = 3000
    prefix = [32 * (s % 3) for s in range(S)]
    lens = [max(n, p) for n, p in zip(lens, prefix)]
    assert _check_step(L, lens, add, prefix, 16, T, *_pool_case(lens, add, prefix, 16, 7, S))[3][3] == 0


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("S,longest,new,T", [(700, 20000, 40, 30000), (1500, 6000, 3, 3000), (4500, 900, 60, 200000), (3, 40, 20000, 60001)])
def test_advance_by_several_workgroups(L, S, longest, new, T, in_place):  # noqa: F811
    """Many entries and positions, in one launch or (in place) two; steps that are not admitted among them."""
    g = _gen(S + longest)
    lens = torch.randint(0, longest, (S,), generator=g).tolist()
    add = torch.where(torch.rand(S, generator=g) < 0.2, -1, torch.randint(0, new, (S,), generator=g)).tolist()
    prefix = [32 * (s % 3) for s in range(S)]
    lens = [max(n, p) for n, p in zip(lens, prefix)]
    table, ring, state = _pool_case(lens, add, prefix, 16, 7, S)
    want = _check_step(L, lens, add, prefix, 16, T, table, ring, state, in_place=in_place)
    assert want[3][3] == 0 and want[1][-1] > 0
    short = [state[0], want[3][2] - 1, 0, 0]
    assert _check_step(L, lens, add, prefix, 16, T, table, ring, short, in_place=in_place)[3][3] == 1


def test_advance_captured_in_place_by_several_workgroups(L):  # noqa: F811
    """A captured step in place goes on from step to step as the plain one does, until one is not admitted."""
    S, page, T, g = 600, 16, 20000, _gen(9)
    lens, pages = torch.randint(0, 3000, (S,), generator=g).tolist(), 130000
    table = torch.full((S, 1000), -1, dtype=torch.int32)
    order, at = torch.randperm(pages, generator=g).int(), 0
    for s, n in enumerate(lens):
        held = -(-n // page)
        table[s, :held] = order[at:at + held]
        at += held
    ring, state = torch.cat([order[at:], torch.full((at,), -9, dtype=torch.int32)]), [0, pages - at, 0, 0]
    rd, sd, td, ld, ad = ring.cuda(), _i32(state), table.cuda(), _i32(lens), _i32([0] * S)
    out = (ld, _i32([0] * (S + 1)), _i32([0] * T), sd)
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        L.kv_advance(L.KVPool(rd, sd), td, ld, ad, page, T, None, out)
    seen = set()
    for step in range(6):
        add = torch.where(torch.rand(S, generator=g) < 0.2, -1, torch.randint(0, 60 if step < 5 else 200, (S,), generator=g)).int()
        ad.copy_(add)
        graph.replay()
        torch.cuda.synchronize()
        lens, starts, positions, state, table, ring = Q.advance(lens, add.tolist(), None, table, page, T, ring, state)
        for got, want in zip(out, (lens, starts, positions, state)):
            assert got.tolist() == list(want)
        assert torch.equal(td.cpu(), table) and torch.equal(rd.cpu(), ring)
        seen.add(state[3])
    assert seen == {0, 4}


def test_advance_refuses_steps(L):  # noqa: F811
    """Too few free pages, tokens, places: nothing is added, sequences leave all the same; too many pages going back: none."""
    lens, add = [40, 20, 100, 0], [30, -1, 1, 16]
    table, ring, state = _pool_case(lens, add, None, 16, 0, 1)
    assert _check_step(L, lens, add, None, 16, 47, table, ring, state)[3][3] == 0      # (all of the pool's pages)
    short = [state[0], state[1] - 1, 0, 0]
    for T in (47, 9000):
        assert _check_step(L, lens, add, None, 16, T, table, ring, short)[3][3] == 1
    assert _check_step(L, lens, add, None, 16, 46, table, ring, state)[3][3] == 4
    assert _check_step(L, lens, add, None, 16, 46, table[:, :6].contiguous(), ring, short)[3][3] == 7
    full = [state[0], len(ring) - 1, 0, 0]
    assert _check_step(L, lens, add, None, 16, 47, table, ring, full)[3][3] == 8
    for S, T in ((0, 0), (0, 5), (2, 0)):
        _check_step(L, [16] * S, [0] * S, None, 16, T, table[:S], ring, state)


def test_advance_of_values_that_break_their_rules(L):  # noqa: F811
    """Wild lengths, prefixes, pool states: no access outside the arrays (guards around them stay)."""
    S, width, pages, T = 40, 5, 30, 64
    g = _gen(3)
    for i in range(6):
        big = torch.randint(-2 ** 31, 2 ** 31 - 1, (4, S), generator=g).int()
        small = torch.randint(-3, 90, (4, S), generator=g).int()
        lens, add, prefix = (torch.where(torch.rand(S, generator=g) < 0.1 * (i % 3), big[k], small[k]) for k in range(3))
        buf = [torch.full((n + 64,), 5, dtype=torch.int32, device="cuda") for n in (S * width, pages, S, S + 1, T, 4)]
        inner = [b[32:-32] for b in buf]
        inner[0].copy_(torch.randint(-9, 40, (S * width,), generator=g))
        state = torch.tensor([[5, 20, 0, 0], [-7, 99, 0, 0], [2 ** 31 - 1, 2 ** 31 - 1, 0, 0], [-2 ** 31, -5, 0, 0]][i % 4], dtype=torch.int32).cuda()
        L.kv_advance(L.KVPool(inner[1], state), inner[0].view(S, width), lens.cuda(), add.cuda(), 16, T, prefix.cuda(), tuple(inner[2:]))
        for b in buf:
            assert bool((b[:32] == 5).all()) and bool((b[-32:] == 5).all())
        st = inner[3].tolist()
        assert st[0] == 0 and st == sorted(st) and st[-1] <= T


# ---------------------------------------------------------------- the ranges of pages

@pytest.mark.parametrize("lens,H,d,page", [
    ([(0, 1)], 1, 64, 16),
    ([(15, 1), (16, 1), (17, 1), (0, 33), (0, 0), (5, 0)], 3, 128, 16),
    ([(63, 2), (64, 64), (10, 200), (200, 1)], 2, 256, 64),
    ([(300, 500), (0, 256)], 2, 128, 256),
    ([(100, 28), (1, 127), (128, 0)], 5, 64, 128),
    ([(i % 70, 1 + i % 3) for i in range(150)], 1, 128, 32),
])
def test_bounds(L, lens, H, d, page):  # noqa: F811
    g = _gen(d + page)
    pages, table, kv, starts = R.layout(lens, page, seed=page)
    parts = R.random_cache(pages, H, page, d, g)
    codes = parts[0].view(torch.uint8)
    # every code, NaN among them; a channel of NaN alone; slots behind the keys full of the largest
    codes.copy_(torch.randint(0, 256, codes.shape, generator=g))
    codes[:, :, :, 3] = NAN_CODES[1]
    for s, n in enumerate(kv):
        if n % page:
            codes[int(table[s, n // page]), :, n % page:] = 0x7E
    before = torch.randint(-112, 113, (pages, H, 2, d), generator=g).to(torch.int8)
    got = L.kv_bounds(_device_cache(L, parts), before.cuda(), table.cuda(), _i32(kv), starts[-1] + 3, _i32(starts))
    assert torch.equal(got.cpu(), Q.bounds(R.Cache(*parts), before, table, kv, starts, page))


def test_bounds_of_missing_pages_and_one_token_each(L):  # noqa: F811
    g = _gen(5)
    parts = R.random_cache(6, 2, 16, 64, g)
    table = torch.tensor([[1, -1, 2], [99, 0, -7], [3, 4, 5]], dtype=torch.int32)
    before = torch.full((6, 2, 2, 64), 9, dtype=torch.int8)
    ref = R.Cache(*parts)
    for kv, starts in (([40, 20, 60], [0, 40, 60, 80]), ([1, 2, -3], [0, 1, 5, 6])):
        got = L.kv_bounds(_device_cache(L, parts), before.cuda(), table.cuda(), _i32(kv), starts[-1], _i32(starts))
        assert torch.equal(got.cpu(), Q.bounds(ref, before, table, kv, starts, 16))
    got = L.kv_bounds(_device_cache(L, parts), before.cuda(), table.cuda(), _i32([33, 17, 48]), 3)
    assert torch.equal(got.cpu(), Q.bounds(ref, before, table, [33, 17, 48], [0, 1, 2, 3], 16))
    assert L.kv_page_bounds(_device_cache(L, parts)).shape == (6, 2, 2, 64)


# ---------------------------------------------------------------- selecting

def _select_case(lens, Hq, H, d, page, seed, trailing=0):
    g = _gen(seed)
    pages, table, kv, starts = R.layout(lens, page, seed=seed)
    T = starts[-1] + trailing
    hi = torch.randint(-20, 113, (pages, H, d), generator=g)
    lo = torch.minimum(hi, torch.randint(-112, 21, (pages, H, d), generator=g))
    rng = torch.stack([hi, lo], 2).to(torch.int8)
    ks = torch.ldexp(torch.ones(pages, H), torch.randint(-2, 3, (pages, H), generator=g) - 6)
    q = (torch.randn(T, Hq, d, generator=g) * torch.exp(2 * torch.randn(T, Hq, 1, generator=g))).to(torch.bfloat16)
    return q, rng, ks, table, kv, starts


def _cache_of_scales(L, ks, page, d):  # noqa: F811
    c = L.kv_cache(ks.shape[0], ks.shape[1], d, page)
    return c._replace(k_scale=ks.cuda())


def _check_select(L, case, page, budget, first, last, trailing=0, **kw):  # noqa: F811
    q, rng, ks, table, kv, starts = case
    want = Q.select(q, rng, ks, table, kv, starts, page, budget, first, last)
    out = torch.full(want.shape, -2, dtype=torch.int32, device="cuda")
    got = L.select_pages(q.cuda(), _cache_of_scales(L, ks, page, q.shape[2]), rng.cuda(), table.cuda(), _i32(kv), budget, _i32(starts),
                         first=first, last=last, out=out, **kw)
    assert got.data_ptr() == out.data_ptr() and torch.equal(got.cpu(), want)
    return want


@pytest.mark.parametrize("lens,Hq,H,d,page,budget,first,last", [
    ([(0, 1)], 1, 1, 64, 16, 1, 0, 0),
    ([(500, 1)], 4, 1, 64, 16, 5, 1, 2),
    ([(700, 1), (3, 1), (1023, 1), (1024, 1)], 8, 2, 128, 16, 7, 0, 0),
    ([(900, 3), (0, 0), (5, 0), (129, 17), (0, 40)], 6, 2, 128, 32, 4, 2, 2),
    ([(2000, 9)], 16, 1, 256, 16, 20, 1, 0),
    ([(3000, 5)], 34, 2, 64, 16, 50, 0, 1),
    ([(5000, 2), (100, 30)], 40, 1, 128, 16, 64, 1, 1),
    ([(4000, 1), (300, 66)], 5, 5, 256, 64, 9, 1, 2),
    ([(20010, 1)], 32, 8, 128, 64, 64, 1, 2),
    ([(i * 37 % 900, 1) for i in range(90)], 4, 2, 64, 16, 12, 1, 1),
    ([(9000, 2)], 2, 1, 64, 16, 300, 3, 5),
])
def test_select(L, lens, Hq, H, d, page, budget, first, last):  # noqa: F811
    _check_select(L, _select_case(lens, Hq, H, d, page, d + page), page, budget, first, last)


@pytest.mark.parametrize("lens,Hq,H,d,budget", [
    ([(195000, 1)], 2, 1, 64, 100),                                        # a row too long for one workgroup
    ([(150000, 1)] + [(30 + i, 1) for i in range(129)], 4, 2, 64, 60),     # among many short ones
    ([(150000, 2)] + [(30 + i, 1) for i in range(29)], 2, 1, 128, 60),
    ([(195000, 1)] + [(30 + i % 50, 1) for i in range(257)], 2, 1, 256, 60),
    ([(40, 1)] * 3 + [(40000, 14)], 1, 1, 64, 33),                         # 14 tokens of a sequence
    ([(2500, 40), (900, 7)], 3, 3, 64, 20),
    ([(15900, 30)], 32, 32, 64, 70),                                       # a chunk of tokens with rows as long as one workgroup takes
    ([(8000, 1), (8191, 1), (16368, 1)], 8, 8, 64, 9),                     # single tokens of rows up to that length
    ([(8000, 1), (8191, 1), (16384, 1)], 8, 8, 64, 9),                     # and beyond it
])
def test_select_long(L, lens, Hq, H, d, budget):  # noqa: F811
    _check_select(L, _select_case(lens, Hq, H, d, 16, 77), 16, budget, 1, 2)


def test_select_ties_zeros_and_what_is_not_finite(L):  # noqa: F811
    """Equal scores go to the lower places; zero queries and scales; NaN and infinities of the queries count as 0; missing
    pages come last, in the order of their places."""
    q, rng, ks, table, kv, starts = _select_case([(800, 6)], 4, 2, 64, 16, 9)
    rng[...] = rng[0, 0]
    ks[...] = 0.25
    ks[table[0, 5:30].long()] = 0.0
    q[1] = 0.0
    q[2, :, ::3] = math.nan
    q[2, 1, 1::3] = -math.inf
    q[3] = math.inf
    q[4] = torch.finfo(torch.bfloat16).tiny / 4
    q[5] = torch.finfo(torch.bfloat16).max * torch.where(torch.arange(64) % 2 == 0, 1.0, -1.0)
    for budget in (1, 8, 40, 50):
        _check_select(L, (q, rng, ks, table, kv, starts), 16, budget, 0, 0)
    table = table.clone()
    table[0, 7:47] = torch.tensor([-1, 10 ** 6] * 20, dtype=torch.int32)
    for budget in (3, 20):
        _check_select(L, (q, rng, ks, table, kv, starts), 16, budget, 1, 1)


def test_select_edges_of_the_rounding(L):  # noqa: F811
    """Largest magnitudes around 127 steps, halves between integers, of every exponent."""
    q, rng, ks, table, kv, starts = _select_case([(600, 40)], 2, 1, 64, 16, 10)
    x = torch.randint(-255, 256, (40, 2, 64), generator=_gen(11)).double() / 2
    x[:, :, 0] = torch.tensor([126.0, 126.5, 127.0, 127.5, 63.5])[torch.arange(40) % 5][:, None]
    e = torch.linspace(-130, 118, 40).round()
    q = (x.clamp(-127.5, 127.5) * torch.exp2(e.double())[:, None, None]).to(torch.bfloat16)
    _check_select(L, (q, rng, ks, table, kv, starts), 16, 10, 0, 0)


def test_select_tokens_behind_the_last_negative_positions_and_narrow_tables(L):  # noqa: F811
    case = _select_case([(300, 4), (0, 0), (50, 2)], 2, 1, 64, 16, 12, trailing=5)
    _check_select(L, case, 16, 3, 0, 1)
    q, rng, ks, table, kv, starts = case
    _check_select(L, (q, rng, ks, table, [2, 0, -4], starts), 16, 3, 0, 1)      # positions below 0 see nothing
    _check_select(L, (q, rng, ks, table[:, :6].contiguous(), kv, starts), 16, 3, 0, 1)
    _check_select(L, (q, rng, ks, table[:, :0].contiguous(), kv, starts), 16, 3, 0, 1)
    none = L.select_pages(q.cuda()[:0], _cache_of_scales(L, ks, 16, 64), rng.cuda(), table.cuda()[:0], _i32([]), 3, _i32([0]))
    assert none.shape == (0, 1, 3)


def test_select_without_starts_and_with_strides(L):  # noqa: F811
    q, rng, ks, table, kv, starts = _select_case([(400 + i, 1) for i in range(7)], 4, 2, 128, 16, 13)
    want = Q.select(q, rng, ks, table, kv, starts, 16, 6, 1, 2)
    wide = torch.empty(7, 12, 128, dtype=torch.bfloat16, device="cuda")
    wide[:, 2:10:2] = q.cuda()
    broad = torch.full((7, table.shape[1] + 9), -5, dtype=torch.int32, device="cuda")
    broad[:, :table.shape[1]] = table.cuda()
    got = L.select_pages(wide[:, 2:10:2], _cache_of_scales(L, ks, 16, 128), rng.cuda(), broad[:, :table.shape[1]], _i32(kv), 6)
    assert torch.equal(got.cpu(), want)


# ---------------------------------------------------------------- attention over selected pages

def _lists(table, kv, starts, H, page, budget, seed, wild=False):
    """Random distinct places of each token and head, the last among them; -1 between and behind."""
    g = _gen(seed)
    T = starts[-1]
    out = torch.full((T, H, budget), -1, dtype=torch.int32)
    for s in range(len(kv)):
        for t in range(starts[s], starts[s + 1]):
            pos = kv[s] - starts[s + 1] + t
            n = pos // page + 1 if pos >= 0 else 0
            for h in range(H):
                mine = torch.randperm(max(0, n - 1), generator=g)[:budget - 1].tolist() + ([n - 1] if n else [])
                mine = mine[-budget:]
                if wild:
                    mine = (mine[:budget - 3] + [-7, 2 ** 31 - 1, table.shape[1] + 3])[:budget]
                    at = torch.randperm(budget, generator=g)[:len(mine)]
                else:
                    mine.sort()
                    at = torch.arange(len(mine))
                out[t, h, at] = torch.tensor(mine, dtype=torch.int32)
    return out


def _run_pages(L, case, page, Hq, places, scale=None, **kw):  # noqa: F811
    q, parts, table, kv, starts = case
    o, lse, ob, lb = Q.attention_of_places(q, R.Cache(*parts), table, kv, starts, page, places, scale)
    got = L.attn_pages(q.cuda(), _device_cache(L, parts), table.cuda(), _i32(kv), places.cuda(), _i32(starts), scale=scale, **kw)
    R.near(got[0], o, ob, "o")
    R.near(got[1], lse, lb, "lse")
    return got


@pytest.mark.parametrize("lens,Hq,H,d,page,budget", [
    ([(0, 1)], 1, 1, 64, 16, 1),
    ([(100, 1)], 4, 1, 64, 16, 3),
    ([(62, 1), (63, 1), (64, 1), (500, 1), (0, 1)], 8, 2, 128, 64, 4),
    ([(300, 5), (0, 0), (5, 0), (129, 1), (0, 20)], 6, 2, 128, 32, 5),
    ([(2000, 3)], 16, 1, 256, 16, 40),
    ([(1000, 2)], 34, 2, 64, 128, 3),
    ([(3000, 1), (100, 2)], 5, 5, 256, 64, 30),
    ([(9000, 1)], 32, 8, 128, 64, 60),
    ([(700, 1)], 2, 1, 128, 256, 2),
    ([(20000, 1)], 4, 1, 64, 16, 1200),
    ([(40 * i, 1) for i in range(70)], 4, 1, 64, 16, 7),
])
def test_pages(L, lens, Hq, H, d, page, budget):  # noqa: F811
    case = _attn_case(L, lens, Hq, H, d, page, seed=d + budget)
    _run_pages(L, case, page, Hq, _lists(case[2], case[3], case[4], H, page, budget, 1))
    _run_pages(L, case, page, Hq, _lists(case[2], case[3], case[4], H, page, max(budget, 4), 2, wild=True), scale=-0.07)


def test_pages_of_all_places_is_the_whole_attention(L):  # noqa: F811
    q, parts, table, kv, starts = _attn_case(L, [(1000, 4), (37, 2)], 8, 2, 128, 32, seed=3)
    places = torch.arange(table.shape[1], dtype=torch.int32).expand(6, 2, -1).contiguous()
    args = (q.cuda(), _device_cache(L, parts), table.cuda(), _i32(kv))
    a, b = L.attn_pages(*args, places.cuda(), _i32(starts)), L.attn_cache(*args, _i32(starts))
    o, lse, ob, lb = R.attention(q, R.Cache(*parts), table, kv, starts, 32)
    for x in (a, b):
        R.near(x[0], o, ob, "o")
        R.near(x[1], lse, lb, "lse")


def test_pages_empty_lists_missing_pages_and_nan(L):  # noqa: F811
    """Rows without keys are 0 with lse -infinity; a listed place without a page makes its rows NaN, one that is not listed
    none; NaN keys and values reach the tokens that list their pages."""
    q, parts, table, kv, starts = _attn_case(L, [(400, 6), (90, 3)], 4, 2, 64, 16, seed=4)
    table[0, 3] = -1
    table[0, 9] = 10 ** 6
    parts[0].view(torch.uint8)[int(table[0, 5]), 0, 7, 11] = NAN_CODES[0]
    parts[1].view(torch.uint8)[int(table[0, 6]), 1, 12, 4] = NAN_CODES[1]
    parts[1].view(torch.uint8)[int(table[1, 5]), :, 9, 12] = NAN_CODES[0]   # position 92: the last token's alone
    places = torch.full((9, 2, 5), -1, dtype=torch.int32)
    for t, mine in enumerate(([], [3, 4], [5, 25], [6], [9], [24, 23, 7], [5], [5, 4], [5, 0])):
        places[t, :, :len(mine)] = torch.tensor(mine, dtype=torch.int32)
    got = _run_pages(L, (q, parts, table, kv, starts), 16, 4, places)
    assert not got[0][0].any() and bool((got[1][0] == -math.inf).all())


def test_pages_listed_twice_count_twice(L):  # noqa: F811
    case = _attn_case(L, [(400, 3), (1000, 1)], 4, 2, 64, 16, seed=6)
    places = torch.full((4, 2, 200), -1, dtype=torch.int32)
    for t in range(4):
        for h in range(2):
            mine = [3, 7, 3, 0, 9, 9, 9, 25 if t < 3 else 62, 3] + list(range(20)) * (8 * (t == 3))
            places[t, h, :len(mine)] = torch.tensor(mine, dtype=torch.int32)
    _run_pages(L, case, 16, 4, places)


def test_pages_tokens_behind_the_last_and_one_each(L):  # noqa: F811
    q, parts, table, kv, starts = _attn_case(L, [(300, 1), (100, 1)], 4, 2, 64, 16, seed=5, trailing=3)
    places = _lists(table, kv, starts, 2, 16, 6, 7)
    o, lse, ob, lb = Q.attention_of_places(q[:2], R.Cache(*parts), table, kv, starts, 16, places)
    padded = torch.cat([places, torch.full((3, 2, 6), 1, dtype=torch.int32)]).cuda()
    out = (torch.full((5, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((5, 4), 7.0, device="cuda"))
    L.attn_pages(q.cuda(), _device_cache(L, parts), table.cuda(), _i32(kv), padded, _i32(starts), out=out)
    assert bool((out[0][2:] == 7).all()) and bool((out[1][2:] == 7).all())
    got = L.attn_pages(q.cuda()[:2], _device_cache(L, parts), table.cuda(), _i32(kv), places.cuda())
    for x in (got, (out[0][:2], out[1][:2])):
        R.near(x[0], o, ob, "o")
        R.near(x[1], lse, lb, "lse")


# ---------------------------------------------------------------- shared prefixes

def _shared_case(groups, Hq, H, d, page, seed=1, trailing=0):
    g = _gen(seed)
    pages, table, kv, starts, prefix, gs = Q.shared_layout(groups, page, seed=seed)
    parts = R.random_cache(pages, H, page, d, g)
    free = torch.ones(pages, page, dtype=torch.bool)
    for s, n in enumerate(kv):
        for j in range(-(-n // page)):
            free[int(table[s, j]), :max(0, n - j * page)] = False
    parts[0].view(torch.uint8)[free[:, None].expand(pages, H, page)] = NAN_CODES[0]
    parts[1].view(torch.uint8).transpose(2, 3)[free[:, None].expand(pages, H, page)] = NAN_CODES[1]
    q = (torch.randn(starts[-1] + trailing, Hq, d, generator=g) * 1.5).to(torch.bfloat16)
    return q, parts, table, kv, starts, prefix, gs


def _run_shared(L, case, page, scale=None, **kw):  # noqa: F811
    q, parts, table, kv, starts, prefix, gs = case
    T = starts[-1]
    o, lse, ob, lb = R.attention(q[:T], R.Cache(*parts), table, kv, starts, page, True, 0, scale)
    got = L.attn_shared(q.cuda(), _device_cache(L, parts), table.cuda(), _i32(kv), _i32(prefix), _i32(gs), _i32(starts), scale=scale, **kw)
    R.near(got[0][:T], o, ob, "o")
    R.near(got[1][:T], lse, lb, "lse")
    return got


SHARED = [
    # [(prefix, [(own cached, new), ...]), ...], Hq, Hkv, d, page
    ([(16, [(0, 1)])], 1, 1, 64, 16),
    ([(0, [(5, 1), (0, 3)])], 4, 2, 64, 16),
    ([(64, [(0, 1), (63, 1), (1, 1)])], 8, 2, 128, 64),
    ([(300, [(3, 1), (50, 1)])], 6, 2, 128, 16),                           # (a prefix that is no whole pages)
    ([(256, [(0, 2), (10, 1)]), (0, [(70, 1)]), (32, [(1, 5)])], 3, 1, 256, 32),
    ([(1024, [(20 * i, 1) for i in range(20)])], 8, 2, 128, 64),
    ([(512, [(7, 40), (0, 100), (200, 3)])], 4, 2, 64, 64),
    ([(128, [(0, 90), (30, 70)]), (640, [(5, 1)] * 30)], 4, 1, 128, 32),
    ([(256, [(0, 1), (40, 130)])], 5, 1, 256, 256),
    ([(2048, [(100, 1)] * 6)], 32, 8, 128, 64),
    ([(48, [(i % 40, 1 + i % 2) for i in range(50)])] * 3, 2, 1, 64, 16),
    ([(160, [(0, 0), (10, 2), (0, 0)]), (16, []), (16, [(0, 0)]), (32, [(1, 1)])], 4, 2, 64, 16),
]


@pytest.mark.parametrize("i", range(len(SHARED)))
def test_shared(L, i):  # noqa: F811
    groups, Hq, H, d, page = SHARED[i]
    _run_shared(L, _shared_case(groups, Hq, H, d, page, seed=50 + i), page)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
def test_shared_both_forms_every_page(L, d, page):  # noqa: F811
    """Groups and sequences of few and of many rows, prefixes around the tiles' ends."""
    groups = [(page, [(70, 60), (page - 1, 1), (0, 1)]), (3 * page, [(1, 1)] * 40), (0, [(31, 64)])]
    _run_shared(L, _shared_case(groups, 4, 2, d, page, seed=d + page), page)


def test_shared_long(L):  # noqa: F811
    _run_shared(L, _shared_case([(8192, [(37 * i % 300, 1) for i in range(24)])], 8, 2, 128, 64, seed=70), 64)
    _run_shared(L, _shared_case([(6000, [(0, 200), (10, 150)])], 4, 1, 128, 16, seed=71), 16, scale=-0.1)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("page", [16, 32, 64])
def test_shared_scales_values_far_apart_and_growing_logits(L, d, page):  # noqa: F811
    """Logits of either sign and none; pages of values 2^140 apart and of scale 0; keys whose logits rise by hundreds along the
    prefix; in the forms for prefixes and (1100 rows) for many rows."""
    for groups in ([(320, [(10, 1), (0, 3), (70, 1)])], [(320, [(10, 250), (30, 25)])]):
        case = _shared_case(groups, 4, 1, d, page, seed=80)
        for scale in (-0.1, 0.0):
            _run_shared(L, case, page, scale=scale)
        q, parts, table, kv, starts, prefix, gs = case
        for j in range(table.shape[1]):
            for s in range(table.shape[0]):
                if int(table[s, j]) >= 0:
                    parts[3][int(table[s, j])] = [2.0 ** 70, 2.0 ** -70, 1.0, 0.0, 2.0 ** -100][j % 5]
        _run_shared(L, case, page)
        q, parts, table, kv, starts, prefix, gs = case = _shared_case(groups, 4, 1, d, page, seed=81)
        for j in range(320 // page):
            parts[2][int(table[0, j])] = 2.0 ** (-6 + 2 * ((j * page) // 64))
        _run_shared(L, case, page)


def test_shared_of_fewer_keys_than_new_tokens(L):  # noqa: F811
    """Tokens before position 0 see nothing: o = 0, lse = -infinity; in both forms."""
    q, parts, table, kv, starts, prefix, gs = _shared_case([(0, [(3, 9)]), (32, [(0, 4), (2, 1)]), (0, [(0, 300)])], 4, 1, 64, 16, seed=85)
    kv[0], kv[3] = 2, 150
    got = _run_shared(L, (q, parts, table, kv, starts, prefix, gs), 16)
    for rows in (slice(0, 7), slice(14, 164)):
        assert not got[0][rows].any() and bool((got[1][rows] == -math.inf).all())


def test_shared_of_lengths_beyond_the_table_and_of_nothing(L):  # noqa: F811
    """Rows that see keys beyond the table are NaN; no tokens, no sequences with tokens; a prefix as long as the table."""
    q, parts, table, kv, starts, prefix, gs = _shared_case([(64, [(30, 2), (3, 1)])], 4, 2, 64, 16, seed=82)
    c = _device_cache(L, parts)
    args = (_i32(prefix), _i32(gs), _i32(starts))
    o, lse = L.attn_shared(q.cuda(), c, table[:, :5].contiguous().cuda(), _i32(kv), *args)
    assert torch.isnan(o[:2]).all() and torch.isnan(lse[:2]).all() and torch.isfinite(o[2:].float()).all()
    o, lse = L.attn_shared(q.cuda()[:0], c, table.cuda(), _i32(kv), _i32(prefix), _i32(gs), _i32([0, 0, 0]))
    assert o.shape[0] == 0
    out = (torch.full((3, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((3, 4), 7.0, device="cuda"))
    L.attn_shared(q.cuda(), c, table.cuda(), _i32(kv), _i32(prefix), _i32(gs), _i32([0, 0, 0]), out=out)
    assert bool((out[0] == 7).all()) and bool((out[1] == 7).all())
    none = table[:, :0].contiguous().cuda()
    o, lse = L.attn_shared(q.cuda(), c, none, _i32(kv), *args)
    assert torch.isnan(o).all()


def test_pages_and_select_on_another_stream_while_the_first_is_busy(L):  # noqa: F811
    """Calls on two streams with their own workspaces give what they give alone."""
    cases = [_attn_case(L, [(900 + i, 1) for i in range(20)], 8, 2, 64, 16, seed=83 + k) for k in range(2)]
    work = []
    for q, parts, table, kv, starts in cases:
        places = _lists(table, kv, starts, 2, 16, 30, 5).cuda()
        cache = _device_cache(L, parts)
        rng = torch.randint(-100, 100, (cache.k.shape[0], 2, 2, 64), generator=_gen(84)).sort(2, descending=True)[0].to(torch.int8).cuda()
        work.append((q.cuda(), cache, table.cuda(), _i32(kv), places, rng.contiguous(), _i32([0, 20]), _i32([16] * 20), _i32(starts)))

    def run(q, cache, table, kv, places, rng, gs, prefix, starts):
        return (*L.attn_pages(q, cache, table, kv, places, starts), L.select_pages(q, cache, rng, table, kv, 20, starts),
                *L.attn_pages(q[:1], cache, table[:1], kv[:1], places[:1].contiguous()))

    alone = [run(*w) for w in work]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in work]
    both = [[], []]
    for _ in range(20):
        for k, s in enumerate(streams):
            with torch.cuda.stream(s):
                both[k].append(run(*work[k]))
    torch.cuda.synchronize()
    for k in range(2):
        for got in both[k]:
            for x, y in zip(got, alone[k]):
                assert torch.equal(x, y)


@pytest.mark.parametrize("n", [150, 700])
def test_shared_many_sequences(L, n):  # noqa: F811
    """More groups and sequences than a workgroup plans for itself."""
    groups = [(16 * (g % 4), [((7 * i) % 40, (i + g) % 3) for i in range(g % 5)]) for g in range(n)]
    groups[3] = (320, [(4, 90), (0, 1)])
    _run_shared(L, _shared_case(groups, 2, 1, 64, 16, seed=72), 16)


def test_shared_repeats_bit_for_bit_and_leaves_what_lies_behind(L):  # noqa: F811
    case = _shared_case([(512, [(i, 1) for i in range(30)]), (64, [(0, 50)])], 8, 2, 64, 32, seed=73, trailing=4)
    T = case[4][-1]
    out = [(torch.full((T + 4, 8, 64), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((T + 4, 8), 7.0, device="cuda")) for _ in range(2)]
    need = L.attn_shared_workspace_size(T + 4, 31, 2, 8, 2, 64, 32, case[2].shape[1])
    for o, fill in zip(out, (0, 0xFF)):
        ws = torch.full((need,), fill, dtype=torch.uint8, device="cuda")
        _run_shared(L, case, 32, out=o, workspace=ws)
        assert bool((o[0][T:] == 7).all()) and bool((o[1][T:] == 7).all())
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])


def test_shared_missing_pages_nan_and_infinite_logits(L):  # noqa: F811
    """A missing page of a prefix makes all of its group's rows NaN, one of a sequence that sequence's; NaN of a key or a
    value reaches the rows that see it; rows of -infinity are NaN with lse -infinity."""
    groups = [(96, [(5, 1), (40, 2)]), (64, [(0, 70), (20, 3)])]
    q, parts, table, kv, starts, prefix, gs = _shared_case(groups, 4, 2, 64, 16, seed=74)
    hole = table.clone()
    hole[0:2, 4] = -1
    _run_shared(L, (q, parts, hole, kv, starts, prefix, gs), 16)
    hole = table.clone()
    hole[2, 6] = 10 ** 6
    _run_shared(L, (q, parts, hole, kv, starts, prefix, gs), 16)
    parts[0].view(torch.uint8)[int(table[0, 2]), 0, 3, 1] = NAN_CODES[0]     # of the first group's prefix
    parts[1].view(torch.uint8)[int(table[2, 1]), 1, 9, 5] = NAN_CODES[1]     # of the second's
    parts[1].view(torch.uint8)[int(table[2, 5]), 0, 8, 5] = NAN_CODES[1]     # position 85: some rows of a prompt
    _run_shared(L, (q, parts, table, kv, starts, prefix, gs), 16)
    q, parts, table, kv, starts, prefix, gs = _shared_case(groups, 4, 2, 64, 16, seed=75)
    parts[0].view(torch.uint8)[..., 0] = 0x38
    q[1, 2, 0] = -math.inf
    q[0, 0, 0] = math.inf
    q[30, 1, 0] = -math.inf
    got = [t.float().cpu() for t in L.attn_shared(q.cuda(), _device_cache(L, parts), table.cuda(), _i32(kv), _i32(prefix), _i32(gs), _i32(starts))]
    low, high = torch.zeros(starts[-1], 4, dtype=torch.bool), torch.zeros(starts[-1], 4, dtype=torch.bool)
    low[1, 2] = low[30, 1] = high[0, 0] = True
    assert torch.isnan(got[0][low | high]).all() and torch.isnan(got[1][high]).all() and bool((got[1][low] == -math.inf).all())
    assert not torch.isnan(got[0][~(low | high)]).any() and torch.isfinite(got[1][~(low | high)]).all()


def test_shared_of_values_that_break_their_rules(L):  # noqa: F811
    """Wild starts, groups and prefixes of the other sequences: the first group's rows are right."""
    groups = [(32, [(10, 20), (3, 10)]), (16, [(5, 9)] * 5)]
    q, parts, table, kv, starts, prefix, gs = _shared_case(groups, 4, 2, 64, 16, seed=76)
    o, lse, ob, lb = R.attention(q, R.Cache(*parts), table, kv, starts, 16)
    wild = table.clone()
    wild[2:] = 2 ** 31 - 1
    for pre, g, k in (([2 ** 31 - 1] * 5, [0, 2, 7], [-5] * 5), ([-9] * 5, [0, 2, 2 ** 31 - 1], [2 ** 31 - 1] * 5), ([17] * 5, [0, 2, -7], [3] * 5),
                      ([48] * 5, [0, 2, 1], [2 ** 31 - 1] * 5)):
        got = L.attn_shared(q.cuda(), _device_cache(L, parts), wild.cuda(), _i32(kv[:2] + k), _i32(prefix[:2] + pre), _i32(g), _i32(starts))
        R.near(got[0][:30], o[:30], ob[:30], "o")
        R.near(got[1][:30], lse[:30], lb[:30], "lse")
    for st in ([0, 20, 30, 10, 5, 2 ** 31 - 1, -4, 75], [0, 20, 30, 30, 30, 30, 30, 2 ** 31 - 1]):
        got = L.attn_shared(q.cuda(), _device_cache(L, parts), wild.cuda(), _i32(kv), _i32(prefix), _i32(gs), _i32(st))
        n = 5 if 5 in st else 30
        R.near(got[0][:n], o[:n], ob[:n], "o")


# ---------------------------------------------------------------- together

def test_a_server_over_steps(L):  # noqa: F811
    """Prompts behind a shared prefix, then single tokens, sequences that leave and are replaced: planned, appended, ranged,
    selected and attended on the device, against the same steps in plain arithmetic; and the same captured once."""
    d, page, H, Hq, pages, S, T, budget = 64, 16, 2, 4, 60, 4, 90, 6
    g = _gen(90)
    cache, pool = L.kv_cache(pages, H, d, page), L.kv_pool(pages)
    table = torch.full((S, 12), -1, dtype=torch.int32, device="cuda")
    rng = L.kv_page_bounds(cache)
    lens = _i32([0] * S)
    # the prefix: sequence 0's first two pages, which the others then hold too
    steps = [[32, 0, 0, 0], [5, 40, 1, 17], [1, 1, 1, 1], [1, -1, 1, 1], [1, 30, 1, -1], [3, 1, 1, 0]]
    prefix = [0] * S
    ref_table, ref_ring, ref_state, ref_lens = table.cpu(), pool.ring.cpu(), pool.state.tolist(), [0] * S
    kc = R.Cache(*(t.cpu() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale)))
    ref_rng = rng.cpu()
    for i, add in enumerate(steps):
        if i == 1:   # the others begin behind the prefix
            table[1:, :2] = table[0, :2]
            lens[1:] = 32
            ref_table[1:, :2] = ref_table[0, :2]
            ref_lens = [32] * S
            prefix = [32] * S
        if i == 4:   # sequence 1 is admitted again
            lens[1] = 32
            ref_lens[1] = 32
        lens, starts, pos, pool = L.kv_advance(pool, table, lens, _i32(add), page, T, _i32(prefix))
        ref_lens, st, p, ref_state, ref_table, ref_ring = Q.advance(ref_lens, add, prefix, ref_table, page, T, ref_ring, ref_state)
        assert lens.tolist() == ref_lens and starts.tolist() == st and pos.tolist() == p and pool.state.tolist() == ref_state
        assert torch.equal(table.cpu(), ref_table) and torch.equal(pool.ring.cpu(), ref_ring) and ref_state[3] == 0
        x = torch.randn(T, Hq + 2 * H, d, generator=g).to(torch.bfloat16)
        q, k, v = x.cuda().split([Hq, H, H], 1)
        L.kv_append(k, v, cache, table, lens, starts)
        R.append(kc, x[:, Hq:Hq + H], x[:, Hq + H:], ref_table, ref_lens, st, page)
        L.kv_bounds(cache, rng, table, lens, T, starts)
        ref_rng = Q.bounds(R.Cache(*(t.cpu() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale))), ref_rng, ref_table, ref_lens, st, page)
        assert torch.equal(rng.cpu(), ref_rng), i
        n = st[-1]
        places = L.select_pages(q, cache, rng, table, lens, budget, starts, first=1, last=1)
        want = Q.select(x[:n, :Hq], ref_rng, cache.k_scale.cpu(), ref_table, ref_lens, st, page, budget, 1, 1)
        assert torch.equal(places[:n].cpu(), want), i
        now = R.Cache(*(t.cpu() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale)))
        o, lse, ob, lb = Q.attention_of_places(x[:n, :Hq], now, ref_table, ref_lens, st, page, want)
        got = L.attn_pages(q, cache, table, lens, places, starts)
        R.near(got[0][:n], o, ob, "pages %d" % i)
        o, lse, ob, lb = R.attention(x[:n, :Hq], now, ref_table, ref_lens, st, page)
        got = L.attn_shared(q, cache, table, lens, _i32(prefix), _i32([0, S]), starts)
        R.near(got[0][:n], o, ob, "shared %d" % i)
        R.near(got[1][:n], lse, lb, "shared lse %d" % i)


def test_captured_steps_follow_the_batch(L):  # noqa: F811
    """One graph of a whole step, in place, replayed over steps whose lengths, leavers and newcomers change, with eager work
    between; each replay against the eager calls from the same state."""
    d, page, H, Hq, S, T, budget = 128, 32, 2, 8, 6, 120, 4
    g = _gen(91)
    x = torch.randn(T, Hq + 2 * H, d, generator=g).to(torch.bfloat16).cuda()
    prefix, groups = _i32([0] * S), _i32([0, 3, S])

    def fresh():
        cache, pool = L.kv_cache(80, H, d, page), L.kv_pool(80)
        z = dict(device="cuda", dtype=torch.int32)
        return dict(cache=cache, pool=pool, table=torch.full((S, 20), -1, **z), lens=torch.zeros(S, **z), add=torch.zeros(S, **z),
                    starts=torch.zeros(S + 1, **z), pos=torch.zeros(T, **z), rng=L.kv_page_bounds(cache), x=x.clone(),
                    places=torch.full((T, H, budget), -1, **z),
                    out=[(torch.zeros((T, Hq, d), dtype=torch.bfloat16, device="cuda"), torch.zeros((T, Hq), device="cuda")) for _ in range(2)])

    def step(s):
        q, k, v = s["x"].split([Hq, H, H], 1)
        L.kv_advance(s["pool"], s["table"], s["lens"], s["add"], page, T, prefix, (s["lens"], s["starts"], s["pos"], s["pool"].state))
        L.kv_append(k, v, s["cache"], s["table"], s["lens"], s["starts"])
        L.kv_bounds(s["cache"], s["rng"], s["table"], s["lens"], T, s["starts"])
        L.select_pages(q, s["cache"], s["rng"], s["table"], s["lens"], budget, s["starts"], out=s["places"])
        L.attn_pages(q, s["cache"], s["table"], s["lens"], s["places"], s["starts"], out=s["out"][0])
        L.attn_shared(q, s["cache"], s["table"], s["lens"], prefix, groups, s["starts"], out=s["out"][1])

    a, b = fresh(), fresh()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(a)   # loads the code (a step of no tokens)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(a)
    for i, add in enumerate([[100, 0, 5, 1, 0, 14], [1, 90, 1, 1, 20, 1], [1] * S, [-1, 1, 1, -1, 1, 1], [60, 1, 1, 40, 1, 1], [1] * S, [0] * S]):
        y = torch.randn(x.shape, generator=g).to(torch.bfloat16).cuda()
        for s in (a, b):
            s["add"].copy_(_i32(add))
            s["x"].copy_(y)
        graph.replay()
        step(b)
        torch.cuda.synchronize()
        assert int(a["pool"].state[3]) == 0
        n = int(a["starts"][-1])
        for key in ("table", "lens", "starts", "pos", "rng"):
            assert torch.equal(a[key], b[key]), (i, key)
        assert torch.equal(a["pool"].ring, b["pool"].ring) and torch.equal(a["pool"].state, b["pool"].state)
        assert torch.equal(a["places"][:n], b["places"][:n]), i
        for u, w in zip(a["out"], b["out"]):
            assert torch.equal(u[0][:n], w[0][:n]) and torch.equal(u[1][:n], w[1][:n]), i
        torch.randn(1000, 1000, device="cuda").sum().item()
