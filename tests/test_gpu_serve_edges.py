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


# more than 256 sequences (planned by a launch) whose rows take both forms in one launch, some in pieces in each
PLANNED = ([(i * 37 % 600, 1) for i in range(125)] + [(i * 29 % 500, 40 + i * 53 % 260) for i in range(50)] + [(2500, 1), (3000, 90), (7, 0)]
           + [(i * 31 % 300, 1 + i % 3) for i in range(130)])


@pytest.mark.parametrize("Hq,H,d,page,window,causal", [(4, 1, 64, 16, 0, True), (4, 2, 128, 64, 0, True), (2, 1, 256, 32, 130, True),
                                                       (2, 1, 128, 16, 0, False)])
def test_attention_planned_in_both_forms(L, Hq, H, d, page, window, causal):  # noqa: F811
    q, parts, table, kv, starts = _attn_case(L, PLANNED, Hq, H, d, page, seed=70 + d + page, trailing=3)
    n = starts[-1]
    assert len(kv) > 256 and n * (Hq // H) > 16 * len(kv)
    ref, rl, ob, lb = R.attention(q[:n], R.Cache(*parts), table, kv, starts, page, causal, window)
    out = (torch.full((n + 3, Hq, d), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((n + 3, Hq), 7.0, device="cuda"))
    args = (q.cuda(), _device_cache(L, parts), table.cuda(), _i32(kv), _i32(starts), causal, window)
    L.attn_cache(*args, out=out)
    R.near(out[0][:n], ref, ob, "o")
    R.near(out[1][:n], rl, lb, "lse")
    assert bool((out[0][n:] == 7).all()) and bool((out[1][n:] == 7).all())
    need = L.attn_cache_workspace_size(n + 3, len(kv), Hq, H, d, page, table.shape[1])
    for a, b in zip(L.attn_cache(*args, workspace=torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")), out):
        assert torch.equal(a[:n], b[:n])


def test_captured_plan_of_both_forms_follows_the_lengths(L):  # noqa: F811
    """More than 256 sequences, captured once and replayed while chunks, pieces and single tokens change places."""
    S, T = 300, 4000
    q, parts, table, _, _ = _attn_case(L, [(900, T // S)] * S, 4, 1, 64, 16, seed=80, poison=False)
    q = torch.cat([q, q])[:T]
    c, td, qd = _device_cache(L, parts), table.cuda(), q.cuda()
    steps = []
    for i in range(4):
        n = [(7 * s + i) % 3 for s in range(S)]
        for s in range(i, S, 23):
            n[s] += 40 + 37 * ((s + i) % 5)
        kv = [min(900 + T // S, (s * 53 * (i + 1)) % 880 + n[s]) for s in range(S)]
        st = [0]
        for x in n:
            st.append(min(T, st[-1] + x))
        steps.append((_i32(kv), _i32(st)))
    kv, st = steps[0][0].clone(), steps[0][1].clone()
    out = (torch.zeros((T, 4, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((T, 4), device="cuda"))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        L.attn_cache(qd, c, td, kv, st, out=out)   # loads the code
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L.attn_cache(qd, c, td, kv, st, out=out)
    for i, (a, b) in enumerate(steps + steps[:2]):
        kv.copy_(a)
        st.copy_(b)
        graph.replay()
        n = int(b[-1])
        want = L.attn_cache(qd, c, td, a, b)
        assert torch.equal(out[0][:n], want[0][:n]) and torch.equal(out[1][:n], want[1][:n]), "replay %d" % i
        ref, rl, ob, lb = R.attention(q[:n, :2], R.Cache(*parts), table, a.tolist(), b.tolist(), 16) if i == 1 else (None,) * 4
        if ref is not None:
            R.near(out[0][:n, :2], ref, ob, "o")
            R.near(out[1][:n, :2], rl, lb, "lse")
        torch.randn(1000, 1000, device="cuda").sum().item()


@pytest.mark.parametrize("new,width", [(20, 7), (7, 40000)])
def test_planned_tables_of_both_forms_that_break_their_rules(L, new, width):  # noqa: F811
    """Starts that decrease, pass T or are negative, endless lengths and wild entries behind a good first sequence: its rows
    are right (every index taken from the tables is bounded).  In one launch of both forms, and (the wide table) in two."""
    more = 300
    lens = [(40, 50)] + [(9, new)] * more
    q, parts, table, kv, starts = _attn_case(L, lens, 2, 1, 64, 16, seed=81)
    T = starts[-1]
    assert (T * 2 > 16 * (more + 1)) == (width == 7)
    table = _wide(table, width)
    o, lse, ob, lb = R.attention(q[:50], R.Cache(*parts), table[:1], kv[:1], starts[:2], 16)
    wild = table.clone()
    wild[1:, :6] = torch.tensor([-(2 ** 31), 2 ** 31 - 1, 12345678, -5, 99, 7], dtype=torch.int32)
    st = _i32(starts)
    for s in (st.flip(0), torch.where(torch.arange(more + 2, device="cuda") % 2 == 0, st, 2 ** 31 - 1), torch.full_like(st, -(2 ** 31))):
        s = s.to(torch.int32)
        s[0], s[1] = 0, 50
        s[2:] = s[2:].clamp(min=50)   # (rows from 50 on may be several sequences')
        for rest in (2 ** 31 - 1, -5):
            got = L.attn_cache(q.cuda(), _device_cache(L, parts), wild.cuda(), _i32([90] + [rest] * more), s)
            R.near(got[0][:50], o, ob, "o")
            R.near(got[1][:50], lse, lb, "lse")


@pytest.mark.parametrize("page", [32, 64, 128])
@pytest.mark.parametrize("n,Hq,d,window", [(1, 4, 128, 0), (6, 2, 256, 9), (120, 4, 128, 0), (120, 4, 128, 50), (90, 2, 256, 0), (150, 1, 64, 70)])
def test_attention_nan_in_long_pages_reaches_only_rows_that_see_it(L, page, n, Hq, d, window):  # noqa: F811
    """NaN keys, values and queries where a page holds whole key tiles of the form for many rows."""
    q, parts, table, kv, starts = _attn_case(L, [(50, n)], Hq, 1, d, page, seed=90)
    kc, vc = parts[0].view(torch.uint8), parts[1].view(torch.uint8)
    for back, chan in ((1, 3), (n // 2 + 1, 40), (n + 20, 41)):
        j = kv[0] - back
        vc[int(table[0, j // page]), 0, chan, j % page] = NAN_CODES[back % 2]
    if n > 1:
        j = kv[0] - 2
        kc[int(table[0, j // page]), 0, j % page, 5] = NAN_CODES[0]
    q[0, 0, 0] = math.nan
    _run_attn(L, q, parts, table, kv, starts, page, Hq, window=window)


@pytest.mark.parametrize("n,d,page", [(1, 128, 64), (9, 64, 128), (200, 128, 64), (200, 64, 128), (200, 128, 256), (150, 256, 64)])
def test_attention_missing_long_pages(L, n, d, page):  # noqa: F811
    """As with short ones: NaN for the rows that see a missing page, and for no other."""
    q, parts, table, kv, starts = _attn_case(L, [(600, n), (40, 1)], 4, 1, d, page, seed=91)
    table[0, 1] = -1
    table[0, (kv[0] - 1) // page] = parts[0].shape[0]
    for window in (0, 20, 150):
        _run_attn(L, q, parts, table, kv, starts, page, 4, window=window)


@pytest.mark.parametrize("d,rot", [(64, 64), (128, 64), (256, 256)])
def test_norm_rope_tokens_in_fp32(L, d, rot):  # noqa: F811
    """[T,H,d] in fp32, slices of a fused projection, by given positions; gains of either type; values rounded with them."""
    g = _gen(d + rot)
    T, Hq, Hkv = 9, 6, 2
    x = torch.randn(T, Hq + 2 * Hkv, d, generator=g) * torch.exp(torch.randn(T, 1, 1, generator=g))
    w = [(1 + 0.3 * torch.randn(d, generator=g)).to(t) for t in (torch.float32, torch.bfloat16)]
    table = L.rope_table(5000, rot, 1e6, device="cpu")
    pos = torch.tensor([4999, 0, 5, 5, 5000, -1, 1234, 4998, 17], dtype=torch.int32)
    q, k, v = x.cuda().split([Hq, Hkv, Hkv], dim=1)
    got = L.qk_norm_rope(q, k, v, w[0].cuda(), w[1].cuda(), table.cuda(), pos.cuda(), eps=1e-5)
    for h in range(Hq + Hkv):
        want, err = R.norm_rope(x[:, h], w[0] if h < Hq else w[1], table, pos.long(), 1e-5)
        y = got[0][:, h] if h < Hq else got[1][:, h - Hq]
        R.near(y, want, R.BF16 * want.abs() + 1.01 * err + 1e-38, "head %d" % h)
    assert torch.equal(got[2].cpu(), x[:, Hq + Hkv:].to(torch.bfloat16))


@pytest.mark.parametrize("S,width", [(64, 9000), (290, 9000)])
def test_captured_chunk_that_comes_and_goes(L, S, width):  # noqa: F811
    """One capture of the two launches replayed with a chunk in the first, another or no sequence."""
    T, Hq, d, page = 3 * S, 4, 64, 16
    q, parts, table, _, _ = _attn_case(L, [(600, 3)] * S, Hq, 1, d, page, seed=82, poison=False)
    assert T * Hq <= 16 * S and (T - S + 1) * Hq * width * page * d >= 1 << 32
    c, td, qd = _device_cache(L, parts), _wide(table, width).cuda(), q.cuda()
    steps = []
    for at in (0, 17, None, S - 1, 0):
        n = [1 + (s == at) * 120 for s in range(S)]
        kv = [min(603, (s * 53) % 480 + n[s]) for s in range(S)]
        st = [0]
        for x in n:
            st.append(st[-1] + x)
        steps.append((_i32(kv), _i32(st)))
    kv, st = steps[0][0].clone(), steps[0][1].clone()
    out = (torch.zeros((T, Hq, d), dtype=torch.bfloat16, device="cuda"), torch.zeros((T, Hq), device="cuda"))
    L.attn_cache(qd, c, td, kv, st, out=out)   # loads the code
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L.attn_cache(qd, c, td, kv, st, out=out)
    for i, (a, b) in enumerate(steps):
        kv.copy_(a)
        st.copy_(b)
        graph.replay()
        n = int(b[-1])
        ref, rl, ob, lb = R.attention(q[:n], R.Cache(*parts), table, a.tolist(), b.tolist(), page)
        R.near(out[0][:n], ref, ob, "o")
        R.near(out[1][:n], rl, lb, "lse")
        for x, y in zip(L.attn_cache(qd, c, td, a, b), out):
            assert torch.equal(x[:n], y[:n]), "replay %d" % i
        torch.randn(1000, 1000, device="cuda").sum().item()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_norm_rope_at_the_ends_of_fp32(L, dtype):  # noqa: F811
    """Rows whose squares fp32 still holds are normed; one whose sum of squares passes 2^128 comes out 0."""
    x = torch.randn(4, 2, 64, generator=_gen(95)).to(dtype)
    x[0] *= 2.0 ** 58
    x[1] *= 2.0 ** 100
    x[2] *= 2.0 ** -60
    w = torch.ones(64)
    y = L.qk_norm_rope(x.cuda(), q_weight=w.cuda(), eps=0.0)[0]
    for t in (0, 2, 3):
        want, err = R.norm_rope(x[t], w, None, None, 0.0)
        R.near(y[t], want, R.BF16 * want.abs() + 1.01 * err, "row %d" % t)
    assert not y[1].any()
