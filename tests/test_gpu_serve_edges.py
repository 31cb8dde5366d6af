"""The serving operators on the GPU where their definitions have no finite
value, or where the host's plan of a batch changes, against plain 64-bit
arithmetic (serveref.py)."""
import math

import pytest
import torch

import serveref as R
from test_gpu_serve import L, NAN_CODES, _attn_case, _device_cache, _gen, _i32, _run_attn, _same_cache  # noqa: F401

pytestmark = pytest.mark.gpu


# (cached, new) lengths, Hq, Hkv, d, page, window, scale: each form alone, in pieces, both beside each other
INFINITE = [
    ([(40, 1), (0, 1)], 4, 1, 128, 64, 0, None),
    ([(30, 5)], 4, 2, 64, 16, 0, -0.2),
    ([(3000, 1)], 8, 2, 128, 64, 0, None),
    ([(2500, 3)], 4, 1, 256, 32, 900, None),
    ([(100, 200)], 4, 2, 128, 64, 0, None),
    ([(50, 150)], 2, 1, 256, 16, 70, -0.2),
    ([(4000, 300)], 4, 1, 64, 64, 0, None),
    ([(700, 150), (30, 1), (900, 4)], 4, 2, 128, 32, 0, None),
]


@pytest.mark.parametrize("i", range(len(INFINITE)))
def test_attention_of_infinite_logits(L, i):  # noqa: F811
    """Rows whose logits are all -infinity have no softmax (0/0): o is NaN and lse -infinity, unlike rows that see no
    key (o = 0).  Logits of +infinity: NaN.  Neither reaches another row."""
    lens, Hq, H, d, page, window, scale = INFINITE[i]
    q, parts, table, kv, starts = _attn_case(L, lens, Hq, H, d, page, seed=40 + i)
    parts[0].view(torch.uint8)[..., 0] = 0x38          # every key's channel 0 is 1
    T, sign = starts[-1], -1.0 if scale and scale < 0 else 1.0
    rows = torch.arange(T * Hq).view(T, Hq)
    low, high = rows % 5 == 1, rows % 5 == 3            # (each in every row tile)
    clean = q.clone()
    clean[low | high] = 0.0
    q[..., 0][low] = -math.inf * sign
    q[..., 0][high] = math.inf * sign
    kw = dict(window=window, scale=scale)
    o, lse, ob, lb = R.attention(clean, R.Cache(*parts), table, kv, starts, page, True, window, scale)
    got = [t.cpu() for t in L.attn_cache(q.cuda(), _device_cache(L, parts), table.cuda(), _i32(kv), _i32(starts), **kw)]
    rest = ~(low | high)
    R.near(got[0][rest], o[rest], ob[rest], "o")
    R.near(got[1][rest], lse[rest], lb[rest], "lse")
    assert torch.isnan(got[0][high]).all() and torch.isnan(got[1][high]).all()
    assert torch.isnan(got[0][low]).all(), "rows of -infinity: o"
    assert bool((got[1][low] == -math.inf).all()), "rows of -infinity: lse"


def test_empty_rope_tables_are_refused(L):  # noqa: F811
    """By every entry point that takes one (they came back unrotated)."""
    k = torch.zeros(3, 2, 64, dtype=torch.bfloat16, device="cuda")
    cache, table = L.kv_cache(6, 2, 64, 16), torch.zeros(3, 2, dtype=torch.int32, device="cuda")
    for rope in (L.rope_table(0, 64), L.rope_table(4, 64)[:0], L.rope_table(4, 64)[:, :0].contiguous()):
        with pytest.raises(ValueError):
            L.qk_norm_rope(k, rope=rope)
        with pytest.raises(ValueError):
            L.kv_append(k, k, cache, table, _i32([1, 1, 1]), rope=rope)


def test_tables_without_columns_of_many_sequences(L):  # noqa: F811
    """Planned by a launch of its own, in the caller's workspace: the size it is told is what the call needs; captured and
    replayed with other lengths."""
    S, Hq, d, page = 300, 4, 64, 16
    cache, none = L.kv_cache(2, 1, d, page), torch.empty(S, 0, dtype=torch.int32, device="cuda")
    q = torch.randn(S, Hq, d, generator=_gen(50)).to(torch.bfloat16).cuda()
    need = L.attn_cache_workspace_size(S, S, Hq, 1, d, page, 0)
    kv = _i32([0] * S)
    with pytest.raises(L.LampError):
        L.attn_cache(q, cache, none, kv, workspace=torch.zeros(need - 1, dtype=torch.uint8, device="cuda"))
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    out = (torch.full((S, Hq, d), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((S, Hq), 7.0, device="cuda"))

    def check(lens):
        seen = torch.tensor(lens) > 0   # (a key that the table does not hold)
        assert torch.isnan(out[0].cpu()[seen]).all() and torch.isnan(out[1].cpu()[seen]).all()
        assert not out[0].cpu()[~seen].any() and bool((out[1].cpu()[~seen] == -math.inf).all())
    L.attn_cache(q, cache, none, kv, out=out, workspace=ws)
    check([0] * S)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L.attn_cache(q, cache, none, kv, out=out)
    for i in range(3):
        lens = [(s + i) % 3 for s in range(S)]
        kv.copy_(_i32(lens))
        graph.replay()
        check(lens)
        torch.randn(1000, 1000, device="cuda").sum().item()


def test_attention_windows_beyond_32_bits(L):  # noqa: F811
    """A window that no C int holds is one that hides nothing, not its low 32 bits."""
    q, parts, table, kv, starts = _attn_case(L, [(90, 4), (20, 1)], 4, 2, 64, 16, seed=51)
    args = (q.cuda(), _device_cache(L, parts), table.cuda(), _i32(kv), _i32(starts))
    want = L.attn_cache(*args)
    for window in (2 ** 31, 2 ** 32 + 3, 2 ** 40, 2 ** 64 + 1):
        for a, b in zip(L.attn_cache(*args, window=window), want):
            assert torch.equal(a, b), window
    for window in (-2 ** 32 + 3, -2 ** 31 - 1):
        with pytest.raises(L.LampError):
            L.attn_cache(*args, window=window)


def test_an_empty_workspace_is_no_workspace(L):  # noqa: F811
    """One without bytes is refused where the call needs some (its address is null, which the library takes as its own
    shared workspace) and taken where it needs none."""
    q, parts, table, kv, starts = _attn_case(L, [(2000, 1), (20, 1)], 4, 2, 64, 16, seed=52)
    args = (q.cuda(), _device_cache(L, parts), table.cuda(), _i32(kv), _i32(starts))
    assert L.attn_cache_workspace_size(2, 2, 4, 2, 64, 16, table.shape[1]) > 0
    none = torch.empty(0, dtype=torch.uint8, device="cuda")
    with pytest.raises(ValueError):
        L.attn_cache(*args, workspace=none)
    short = (args[0], args[1], args[2][:, :8], _i32([100, 21]), args[4])
    assert L.attn_cache_workspace_size(2, 2, 4, 2, 64, 16, 8) == 0
    for a, b in zip(L.attn_cache(*short, workspace=none), L.attn_cache(*short)):
        assert torch.equal(a, b)


def _wide(table, width):
    """The table in one of `width` columns, of which the others hold -1."""
    wide = torch.full((table.shape[0], width), -1, dtype=torch.int32)
    wide[:, :table.shape[1]] = table
    return wide


# lengths, Hq, Hkv, d, page, columns: a chunk among sequences so short that they have 16 rows or fewer on average, in a table of
# so many keys that it takes the form for many rows in a launch of its own; planned by each wave and by a launch
CHUNKS = [
    ([(i * 37 % 500, 1) for i in range(60)] + [(900, 150), (0, 1)], 4, 1, 128, 64, 900),
    ([(300, 120)] + [(i * 41 % 300, 1) for i in range(150)], 8, 2, 64, 16, 9000),
    ([(i * 29 % 200, 1 + i % 2) for i in range(280)] + [(1500, 90), (0, 200)], 8, 2, 128, 32, 2000),
    ([(5, 0), (2000, 100)] + [(i * 31 % 400, 1) for i in range(64)], 4, 2, 256, 128, 400),
    ([(i % 9, 1 + i % 3) for i in range(90)] + [(3, 1)], 8, 2, 64, 16, 9000),     # (no long one after all)
]


def _chunk_case(L, i, seed):  # noqa: F811
    lens, Hq, H, d, page, width = CHUNKS[i]
    q, parts, table, kv, starts = _attn_case(L, lens, Hq, H, d, page, seed=seed)
    G, S, T = Hq // H, len(lens), starts[-1]
    assert T * G <= 16 * S and 64 < (T - S + 1) * G
    assert (T - S + 1) * G * width * page * H * d >= 1 << 32   # (the host's rule)
    return q, parts, _wide(table, width), kv, starts, page, Hq


@pytest.mark.parametrize("window", [0, 100])
@pytest.mark.parametrize("i", range(len(CHUNKS)))
def test_attention_of_a_chunk_among_many_tokens(L, i, window):  # noqa: F811
    """Each sequence in the form it takes, and bit-equal repeats."""
    q, parts, table, kv, starts, page, Hq = _chunk_case(L, i, 60 + i)
    got = _run_attn(L, q, parts, table, kv, starts, page, Hq, window=window)
    again = L.attn_cache(q.cuda(), _device_cache(L, parts), table.cuda(), _i32(kv), _i32(starts), window=window)
    for a, b in zip(got, again):
        assert torch.equal(a, b)
