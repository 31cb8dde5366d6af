"""The operators of long contexts and changing batches in the forms that only some batches take: each
test names the sizes from which its form runs, and holds its batch to them."""
import math
import os
import re

import pytest
import torch

import longref as Q
import serveref as R
from test_gpu_long import (_cache_of_scales, _check_select, _check_step, _gen, _i32, _pool_case, _run_shared, _select_case,
                           _shared_case)
from test_gpu_serve import L, NAN_CODES, _device_cache  # noqa: F401

pytestmark = pytest.mark.gpu

CSRC = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "paper_2609_39361_amd", "csrc")


def _constant(file, name):
    """A constant of the kernels' rules, as the source has it."""
    with open(os.path.join(CSRC, file)) as f:
        return int(re.search(r"\b%s = (\d+)\b" % name, f.read()).group(1))


# ---------------------------------------------------------------- shared prefixes

@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
def test_shared_form_for_many_rows_every_page(L, d, page):  # noqa: F811
    """A group of more rows than the form for prefixes takes, its prefix ending off the key tiles (pages of 16 and 32), and
    sequences of more than the form for few: behind that prefix, of their own alone; smaller groups beside them."""
    groups = [(3 * page, [(70, 400), (page - 1, 150), (0, 1)]), (page, [(1, 1)] * 10), (0, [(31, 64)]), (0, [(5, 2)])]
    G, many, few = 2, _constant("lamp_cache_shared.hip", "GROUP_PREFIX"), _constant("lamp_cache_shared.hip", "SHARED_FEW")
    assert 551 * G > many and 64 * G > few and 10 * G < many
    _run_shared(L, _shared_case(groups, G, 1, d, page, seed=d + page), page)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_shared_join_of_many_rows(L, d):  # noqa: F811
    """Rows in the join for many rows: of a prefix in pieces and own keys whole or in pieces, of own keys in pieces alone,
    finished already; rows that see nothing in a sequence in pieces; a missing page, NaN; tokens behind the last."""
    Hq, H, page = 8, 2, 32
    groups = [(0, [(2000, 1)]), (1984, [(5, 1), (40, 2), (700, 1)] * 2), (64, [(0, 70), (20, 3)]), (0, [(3, 1), (0, 0)]), (0, [(0, 1100)])]
    q, parts, table, kv, starts, prefix, gs = _shared_case(groups, Hq, H, d, page, seed=d, trailing=5)
    T = starts[-1]
    assert T * Hq > _constant("lamp_cache_shared.hip", "JOIN_WIDE")
    kv[-1] = 1000                                        # (the first 100 of its tokens are before position 0)
    table[2, 1984 // page] = -1                          # own keys of the second group's second sequence
    parts[1].view(torch.uint8)[int(table[1, 7]), 1, 9, 5] = NAN_CODES[1]      # a value of that group's prefix
    parts[0].view(torch.uint8)[int(table[8, 2]), 0, 3, 1] = NAN_CODES[0]      # a key that one sequence sees
    out = (torch.full((T + 5, Hq, d), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((T + 5, Hq), 7.0, device="cuda"))
    need = L.attn_shared_workspace_size(T + 5, len(kv), len(groups), Hq, H, d, page, table.shape[1])
    for fill in (0xFF, 0):
        _run_shared(L, (q, parts, table, kv, starts, prefix, gs), page, out=out, workspace=torch.full((need,), fill, dtype=torch.uint8, device="cuda"))
        assert bool((out[0][T:] == 7).all()) and bool((out[1][T:] == 7).all())
    none = slice(T - 1100, T - 1000)
    assert not out[0][none].any() and bool((out[1][none] == -math.inf).all()) and torch.isfinite(out[1][T - 1000:T]).all()


# ---------------------------------------------------------------- selecting

def _two_launches(L, case, budget):  # noqa: F811
    q, rng, _, table, kv, _ = case
    return L.select_pages_workspace_size(q.shape[0], len(kv), q.shape[1], rng.shape[1], q.shape[2], table.shape[1], budget) > 0


@pytest.mark.parametrize("d,lens,one", [
    (64, [(16383, 1), (16352, 1), (40, 1)], True),      # 1024 places, the longest row of one launch
    (64, [(16384, 1), (16352, 1), (40, 1)], False),
    (128, [(8191, 1), (8000, 1)], True),                # 512 places
    (128, [(8192, 1), (8000, 1)], False),               # rows of the second launch's smaller workgroups: 513 to 1024 places
    (128, [(16383, 1), (300, 2), (9000, 1)], False),
    (128, [(16384, 1), (300, 2), (9000, 1)], False),    # and of its larger ones
    (256, [(4095, 1), (17, 1)], True),                  # 256 places
    (256, [(4096, 1), (17, 1)], False),
    (256, [(11000, 3), (16383, 1)], False),
])
def test_select_on_both_sides_of_its_borders(L, d, lens, one):  # noqa: F811
    """Tables as wide as their longest row."""
    q, rng, ks, table, kv, starts = _select_case(lens, 4, 2, d, 16, d + len(lens))
    case = q, rng, ks, table[:, :-1].contiguous(), kv, starts
    for budget in (1, 9, 200):
        assert _two_launches(L, case, budget) != one
        _check_select(L, case, 16, budget, min(budget, 1), 0 if budget == 1 else 2)


@pytest.mark.parametrize("d,keys,G", [(128, keys, G) for keys in (9000, 30000) for G in (1, 3, 4, 8, 16, 17, 40)]
                         + [(64, 17000, 2), (64, 17000, 20), (256, 5000, 20), (256, 17000, 5)])
def test_select_in_two_launches_of_every_group_size(L, d, keys, G):  # noqa: F811
    """Groups within the matrix product's rows and beyond them, rows of up to 1024 places and of more; several tokens a tile."""
    case = _select_case([(keys, 3), (0, 2), (keys // 2, 5)], 2 * G, 2, d, 16, G)
    assert _two_launches(L, case, 30)
    _check_select(L, case, 16, 30, 1, 2)


@pytest.mark.parametrize("d,width,Hq,H,new", [
    (256, 768, 128, 128, 16),     # 16 tokens a tile: as many scores as LDS is given
    (128, 700, 128, 128, 16),
    (64, 1024, 128, 128, 40),
    (256, 1024, 256, 128, 16),    # 8 tokens a tile
])
def test_select_chunks_of_wide_tables_in_one_launch(L, d, width, Hq, H, new):  # noqa: F811
    """Chunks of tokens over rows longer than single tokens' are taken in one launch; some heads compared."""
    q, rng, ks, table, kv, starts = _select_case([(16 * width - new, new)], Hq, H, d, 16, width)
    case = q, rng, ks, table[:, :width].contiguous(), kv, starts
    assert not _two_launches(L, case, 50)
    got = L.select_pages(q.cuda(), _cache_of_scales(L, ks, 16, d), rng.cuda(), case[3].cuda(), _i32(kv), 50, _i32(starts))
    G = Hq // H
    for h in (0, H // 2, H - 1):
        want = Q.select(q[:, h * G:h * G + G], rng[:, h:h + 1], ks[:, h:h + 1], case[3], kv, starts, 16, 50, 1, 2)
        assert torch.equal(got[:, h:h + 1].cpu(), want)


# ---------------------------------------------------------------- steps

@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("S", [100, 1500])
def test_advance_around_the_second_workgroup(L, S, in_place):  # noqa: F811
    """As many tokens and table entries as one workgroup takes, and one more."""
    share, g = _constant("lamp_advance.hip", "SHARE"), _gen(S)
    width = 64 if S == 100 else 16
    lens = torch.randint(0, 16 * width - 20, (S,), generator=g).tolist()
    add = torch.where(torch.rand(S, generator=g) < 0.3, -1, torch.randint(0, 9 if S == 100 else 2, (S,), generator=g)).tolist()
    case = _pool_case(lens, add, None, 16, 7, S, width=width)
    last = share - 1 - S * width // 64
    assert 0 < last and sum(max(0, a) for a in add) <= last
    for T in (last, last + 1):
        assert _check_step(L, lens, add, None, 16, T, *case, in_place=in_place)[3][3] == 0


# ---------------------------------------------------------------- captured

def test_captured_forms_follow_lengths_that_change(L):  # noqa: F811
    """One graph of attn_shared planned by a launch of its own, with the forms for prefixes and for many rows and the join of
    many rows, of select_pages in two launches and attn_pages in pieces: replayed over batches of other lengths and groups,
    with eager work between, each replay against the eager calls."""
    page, d, H, Hq, S, groups, T = 16, 64, 2, 8, 150, 12, 900
    g = _gen(21)
    pages, width = 5000, 1100
    parts = R.random_cache(pages, H, page, d, g)
    cache = _device_cache(L, parts)
    hi = torch.randint(-20, 113, (pages, H, d), generator=g)
    rng = torch.stack([hi, torch.minimum(hi, torch.randint(-112, 21, (pages, H, d), generator=g))], 2).to(torch.int8).cuda()
    assert S + groups > _constant("lamp_cache_plan.h", "SHARED_ALONE") and T * Hq > _constant("lamp_cache_shared.hip", "JOIN_WIDE")
    assert T * (Hq // H) > _constant("lamp_cache_shared.hip", "GROUP_PREFIX")
    assert L.select_pages_workspace_size(T, S, Hq, H, d, width, 20) > 0 and L.attn_pages_workspace_size(40, Hq, H, d, page, 100) > 0
    q = torch.randn(T, Hq, d, generator=g).to(torch.bfloat16).cuda()
    lists = torch.randint(-1, 300, (40, H, 100), generator=g).int().cuda()
    z = dict(device="cuda", dtype=torch.int32)
    st = dict(table=torch.zeros((S, width), **z), kv=torch.zeros(S, **z), starts=torch.zeros(S + 1, **z), prefix=torch.zeros(S, **z),
              gs=torch.zeros(groups + 1, **z))

    def batch(seed):
        """A batch whose first group holds many rows (but for seed 1), some tokens behind the last."""
        b = _gen(seed)
        cut = sorted(torch.randperm(S - 1, generator=b)[:groups - 1].add(1).tolist())
        gs = [0, *cut, S]
        table = torch.randint(0, pages, (S, width), generator=b).int()
        new = torch.randint(0, 4, (S,), generator=b)
        new[0] = 300 if seed != 1 else 2
        prefix, own = torch.zeros(S, dtype=torch.long), torch.randint(0, 200, (S,), generator=b)
        for a, e in zip(gs, gs[1:]):
            prefix[a:e] = 16 * int(torch.randint(0, 60, (1,), generator=b))
            table[a:e, :60] = table[a, :60].clone()
        own[S - 1] = 15000
        return dict(table=table, kv=(prefix + own + new).int(), starts=torch.cat([torch.zeros(1), new.cumsum(0)]).int(), prefix=prefix.int(),
                    gs=torch.tensor(gs, dtype=torch.int32))

    def step():
        o = L.attn_shared(q, cache, st["table"], st["kv"], st["prefix"], st["gs"], st["starts"])
        return (*o, L.select_pages(q, cache, rng, st["table"], st["kv"], 20, st["starts"]),
                *L.attn_pages(q[:40], cache, st["table"][:40], st["kv"][:40], lists))

    def load(seed):
        for k, v in batch(seed).items():
            st[k].copy_(v)

    load(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for seed in (1, 2, 0, 3, 1):
        load(seed)
        graph.replay()
        want = step()
        torch.cuda.synchronize()
        n = int(st["starts"][-1])
        assert 300 <= n < T or seed == 1
        for x, y in zip(held[:3], want[:3]):
            assert torch.equal(x[:n], y[:n]), seed
        for x, y in zip(held[3:], want[3:]):
            assert torch.equal(x, y), seed
        torch.randn(1000, 1000, device="cuda").sum().item()
    b = batch(2)
    load(2)
    o, lse, ob, lb = R.attention(q[:int(b["starts"][-1])].cpu(), R.Cache(*parts), b["table"], b["kv"].tolist(), b["starts"].tolist(), page)
    graph.replay()
    R.near(held[0][:len(o)], o, ob, "o")
    R.near(held[1][:len(o)], lse, lb, "lse")
