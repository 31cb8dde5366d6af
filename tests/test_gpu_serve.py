"""The serving operators on the GPU against plain 64-bit arithmetic
(serveref.py): the per-head norms with the rotation, appending to the 8-bit
paged cache, the attention over it, and the three as a server runs them."""
import math

import pytest
import torch

import serveref as R

pytestmark = pytest.mark.gpu

NAN_CODES = (0x7F, 0xFF)


@pytest.fixture(scope="module")
def L():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_39361_amd import lamp
    lamp.lib()
    return lamp


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


# ---------------------------------------------------------------- norms and rotation

@pytest.mark.parametrize("B,N,Hq,Hkv,d,rot,dtype", [
    (1, 1, 1, 1, 64, 64, torch.bfloat16),
    (2, 37, 8, 2, 64, 32, torch.float32),
    (1, 131, 5, 1, 128, 128, torch.bfloat16),
    (3, 50, 32, 8, 128, 64, torch.float32),
    (1, 19, 16, 16, 256, 256, torch.bfloat16),
    (1, 5000, 6, 2, 128, 128, torch.bfloat16),
    (2, 9, 3, 1, 256, 16, torch.float32),
])
def test_norm_rope_prompt(L, B, N, Hq, Hkv, d, rot, dtype):
    """[B,N,H,d] slices of a fused projection to [B,H,N,d], values laid out with them."""
    g = _gen(N)
    qkv = (torch.randn(B, N, Hq + 2 * Hkv, d, generator=g) * 3).to(dtype)
    w = [(1 + 0.3 * torch.randn(d, generator=g)).to(t) for t in (torch.float32, torch.bfloat16)]
    table = L.rope_table(N, rot, 1e4, device="cpu")
    q, k, v = qkv.cuda().split([Hq, Hkv, Hkv], dim=2)
    got = L.qk_norm_rope(q, k, v, w[0].cuda(), w[1].cuda(), table.cuda(), eps=1e-5)
    for x, gain, y in ((qkv[:, :, :Hq], w[0], got[0]), (qkv[:, :, Hq:Hq + Hkv], w[1], got[1])):
        for b in range(B):
            for h in range(x.shape[2]):
                want, err = R.norm_rope(x[b, :, h], gain, table, torch.arange(N), 1e-5)
                R.near(y[b, h], want, R.BF16 * want.abs() + 1.01 * err + 1e-38, "head %d" % h)
    assert torch.equal(got[2].cpu(), qkv[:, :, Hq + Hkv:].transpose(1, 2).to(torch.bfloat16))


@pytest.mark.parametrize("d", [64, 128, 256])
def test_norm_rope_tokens_in_place_and_parts(L, d):
    """[T,H,d] by given positions, in place; norm alone; rotation alone; a position outside the table."""
    g = _gen(d)
    T, Hq, Hkv = 7, 6, 2
    x = torch.randn(T, Hq + 2 * Hkv, d, generator=g).to(torch.bfloat16)
    w = (1 + 0.3 * torch.randn(d, generator=g)).to(torch.bfloat16)
    table = L.rope_table(70000, d, 1e6, device="cpu")
    pos = torch.tensor([69999, 0, 5, 5, 70000, -1, 12345], dtype=torch.int32)
    buf = x.cuda()
    q, k = buf[:, :Hq], buf[:, Hq:Hq + Hkv]
    got = L.qk_norm_rope(q, k, None, w.cuda(), None, table.cuda(), pos.cuda(), eps=1e-6, out=(q, k, None))
    assert got[2] is None and got[0].data_ptr() == q.data_ptr()
    for h in range(Hq + Hkv):
        want, err = R.norm_rope(x[:, h], w if h < Hq else None, table, pos.long(), 1e-6)
        # (without the norm only the rotation's roundings are left; the same bound covers them)
        R.near(buf[:, h], want, R.BF16 * want.abs() + 1.01 * err + 1e-38, "head %d" % h)
    assert torch.equal(buf[:, Hq + Hkv:].cpu(), x[:, Hq + Hkv:])
    only = L.qk_norm_rope(x.cuda()[:, :Hq], q_weight=w.cuda(), eps=0.0)
    assert only[1] is None and only[2] is None
    for h in range(Hq):
        want, err = R.norm_rope(x[:, h], w, None, None, 0.0)
        R.near(only[0][:, h], want, R.BF16 * want.abs() + 1.01 * err + 1e-38, "norm alone")


def test_norm_rope_of_nothing_and_of_zero_rows(L):
    got = L.qk_norm_rope(torch.empty(0, 4, 64, dtype=torch.bfloat16, device="cuda"))
    assert got[0].shape == (0, 4, 64)
    z = torch.zeros(3, 2, 128, dtype=torch.bfloat16, device="cuda")
    w = torch.ones(128, device="cuda")
    assert torch.equal(L.qk_norm_rope(z, q_weight=w)[0], z)
    z[1, 1, 7] = math.inf   # reaches its own row only
    y = L.qk_norm_rope(z, q_weight=w)[0]
    assert not torch.isfinite(y[1, 1]).all() and torch.equal(y[0], z[0]) and torch.equal(y[1, 0], z[1, 0])


# ---------------------------------------------------------------- appending

def _device_cache(L, parts):
    return L.KVCache(*(t.cuda() for t in parts))


def _same_cache(cache, ref, bounds, what):
    assert torch.equal(cache.k_scale.cpu().double(), ref.ks), what + ": key scales"
    assert torch.equal(cache.v_scale.cpu().double(), ref.vs), what + ": value scales"
    for codes, want, scale, bound in ((cache.k, ref.k, ref.ks, bounds[0]), (cache.v, ref.v, ref.vs, bounds[1])):
        s = scale[:, :, None, None]
        R.near(codes.cpu().float().double() * s, want * s, bound, what)


@pytest.mark.parametrize("lens,H,d,page,dtype,norm,rot", [
    ([(0, 1)], 1, 64, 16, torch.bfloat16, True, 64),
    ([(15, 1), (16, 1), (17, 1), (31, 1), (0, 1)], 2, 128, 16, torch.bfloat16, True, 128),
    ([(63, 2), (64, 64), (10, 200), (0, 65)], 2, 128, 64, torch.bfloat16, True, 64),
    ([(5, 0), (0, 0), (100, 3), (7, 0)], 2, 64, 32, torch.float32, False, 64),
    ([(3, 500), (250, 13)], 1, 256, 256, torch.float32, True, 256),
    ([(120, 40), (1, 127), (0, 128)], 3, 256, 128, torch.bfloat16, False, 0),
    ([(i % 70, 1) for i in range(150)], 1, 64, 64, torch.bfloat16, True, 64),
    ([(i % 33, (7 * i) % 5) for i in range(90)], 1, 64, 16, torch.bfloat16, False, 32),
])
def test_append(L, lens, H, d, page, dtype, norm, rot):
    g = _gen(len(lens) * d + page)
    pages, table, kv, starts = R.layout(lens, page, seed=d)
    parts = R.random_cache(pages, H, page, d, g)
    T = starts[-1] + 2   # two tokens of no sequence
    new = (torch.randn(T, 2, H, d, generator=g) * torch.exp(torch.randn(T, 2, 1, 1, generator=g))).to(dtype)
    w = (1 + 0.2 * torch.randn(d, generator=g)) if norm else None
    rope = L.rope_table(max(kv) + 1, rot, 1e4, device="cpu") if rot else None
    ref, cache = R.Cache(*parts), _device_cache(L, parts)
    bounds = R.append(ref, new[:, 0], new[:, 1], table, kv, starts, page, w, rope)
    nd = new.cuda()
    L.kv_append(nd[:, 0], nd[:, 1], cache, table.cuda(), _i32(kv), _i32(starts), None if w is None else w.cuda(),
                None if rope is None else rope.cuda())
    _same_cache(cache, ref, bounds, "append")


def test_append_grows_the_scale_token_by_token(L):
    """Single tokens of growing size into one page: codes already there are rescaled, exactly while they stay normal."""
    g = _gen(5)
    d, page, H = 64, 32, 2
    parts = R.random_cache(4, H, page, d, g)
    ref, cache = R.Cache(*parts), _device_cache(L, parts)
    table = torch.tensor([[2, 0]], dtype=torch.int32)
    for i in range(40):
        x = (torch.randn(1, 2, H, d, generator=g) * 1.7 ** i).to(torch.bfloat16)
        bounds = R.append(ref, x[:, 0], x[:, 1], table, [i + 1], [0, 1], page)
        xd = x.cuda()
        L.kv_append(xd[:, 0], xd[:, 1], cache, table.cuda(), _i32([i + 1]))
        _same_cache(cache, ref, bounds, "token %d" % i)


def test_append_not_finite_tiny_and_zero(L):
    """NaN and infinities are stored as NaN and leave the scale alone; zeros; the smallest and the largest numbers."""
    d, page = 64, 16
    g = _gen(6)
    x = torch.randn(6, 2, 1, d, generator=g)
    x[0, :, 0, 3], x[1, :, 0, 4], x[1, :, 0, 5] = math.nan, math.inf, -math.inf
    x[2] = 0.0
    x[3] *= 1e-38
    x[4, :, 0, 0] = 3.3e38
    x[5] = math.nan
    parts = R.random_cache(6, 1, page, d, g)
    table = torch.arange(6, dtype=torch.int32).view(6, 1).flip(0).contiguous()
    ref, cache = R.Cache(*parts), _device_cache(L, parts)
    bounds = R.append(ref, x[:, 0], x[:, 1], table, [1] * 6, list(range(7)), page)
    xd = x.cuda()
    L.kv_append(xd[:, 0], xd[:, 1], cache, table.cuda(), _i32([1] * 6))
    _same_cache(cache, ref, bounds, "not finite")


def test_append_drops_tokens_without_a_page(L):
    """Missing entries (-1, too large, beyond the table's width) and negative positions: those tokens alone are dropped.
    A position outside the rope table stores NaN."""
    d, page, H = 128, 16, 1
    g = _gen(7)
    parts = R.random_cache(5, H, page, d, g)
    table = torch.tensor([[1, -1, 2], [5, 0, -7], [3, 4, 4]], dtype=torch.int32)
    kv, starts = [48, 60, 3], [0, 48, 98, 106]
    new = torch.randn(110, 2, H, d, generator=g).to(torch.bfloat16)
    rope = L.rope_table(40, d, 1e4, device="cpu")
    ref, cache = R.Cache(*parts), _device_cache(L, parts)
    bounds = R.append(ref, new[:, 0], new[:, 1], table, kv, starts, page, None, rope)
    nd = new.cuda()
    L.kv_append(nd[:, 0], nd[:, 1], cache, table.cuda(), _i32(kv), _i32(starts), None, rope.cuda())
    _same_cache(cache, ref, bounds, "dropped")
    assert torch.isnan(ref.k).any()


# ---------------------------------------------------------------- attention

def _attn_case(L, lens, Hq, H, d, page, causal=True, window=0, scale=None, seed=1, poison=True, trailing=0, stride=1):
    g = _gen(seed)
    pages, table, kv, starts = R.layout(lens, page, seed=seed)
    parts = R.random_cache(pages, H, page, d, g)
    if poison:   # NaN in every slot that belongs to no sequence
        free = torch.ones(pages, page, dtype=torch.bool)
        for s, n in enumerate(kv):
            for j in range(-(-n // page)):
                free[int(table[s, j]), :max(0, n - j * page)] = False
        kc, vc = parts[0].view(torch.uint8), parts[1].view(torch.uint8)
        kc[free[:, None].expand(pages, H, page)] = NAN_CODES[0]
        vc.transpose(2, 3)[free[:, None].expand(pages, H, page)] = NAN_CODES[1]
        unused = sorted(set(range(pages)) - {int(x) for x in table.flatten()})
        parts[2][unused] = math.nan
        parts[3][unused] = math.inf
    T = starts[-1] + trailing
    q = (torch.randn(T, Hq * stride, d, generator=g) * 1.5).to(torch.bfloat16)
    return q, parts, table, kv, starts


def _run_attn(L, q, parts, table, kv, starts, page, Hq, **kw):
    ref = R.Cache(*parts)
    view = q[:, :Hq]
    o, lse, ob, lb = R.attention(view, ref, table, kv, starts, page, kw.get("causal", True), kw.get("window", 0), kw.get("scale"))
    got = L.attn_cache(q.cuda()[:, :Hq], _device_cache(L, parts), table.cuda(), _i32(kv), _i32(starts), **kw)
    R.near(got[0], o, ob, "o")
    R.near(got[1], lse, lb, "lse")
    return got


ATTN = [
    # (cached, new) lengths, Hq, Hkv, d, page
    ([(0, 1)], 1, 1, 64, 16),
    ([(0, 1)], 8, 1, 256, 256),
    ([(0, 37)], 8, 8, 64, 16),
    ([(62, 1), (63, 1), (64, 1), (65, 1), (0, 1), (255, 1), (256, 1)], 8, 2, 128, 64),
    ([(15, 1), (16, 1), (17, 1), (48, 3)], 3, 1, 256, 16),
    ([(300, 17), (0, 0), (5, 0), (129, 1), (0, 40)], 6, 2, 128, 32),
    ([(1000, 5)], 16, 1, 128, 128),
    ([(511, 130)], 4, 4, 64, 64),
    ([(3000, 1), (10, 1)], 32, 8, 128, 64),
    ([(2000, 2), (1, 300)], 5, 1, 256, 32),
    ([(i * 13 % 400, 1 + i % 3) for i in range(130)], 4, 1, 64, 16),
]


@pytest.mark.parametrize("i", range(len(ATTN)))
def test_attention_causal(L, i):
    lens, Hq, H, d, page = ATTN[i]
    _run_attn(L, *_attn_case(L, lens, Hq, H, d, page), page, Hq)


@pytest.mark.parametrize("i", [2, 3, 5, 8, 9])
def test_attention_not_causal(L, i):
    lens, Hq, H, d, page = ATTN[i]
    _run_attn(L, *_attn_case(L, lens, Hq, H, d, page, seed=2), page, Hq, causal=False, scale=0.05)


@pytest.mark.parametrize("i", [2, 3, 5, 7, 8, 9])
@pytest.mark.parametrize("window", [1, 33, 200])
def test_attention_window(L, i, window):
    lens, Hq, H, d, page = ATTN[i]
    _run_attn(L, *_attn_case(L, lens, Hq, H, d, page, seed=3), page, Hq, window=window)


def test_attention_window_of_the_largest_int(L):
    lens, Hq, H, d, page = ATTN[5]
    _run_attn(L, *_attn_case(L, lens, Hq, H, d, page, seed=3), page, Hq, window=2 ** 31 - 1)


@pytest.mark.parametrize("lens,Hq,H,d", [([(20010, 1)], 32, 8, 128), ([(9000, 300)], 8, 2, 128), ([(12000, 700), (40, 1)], 4, 2, 256),
                                         ([(0, 2500)], 4, 4, 64)])
def test_attention_long(L, lens, Hq, H, d):
    _run_attn(L, *_attn_case(L, lens, Hq, H, d, 64, seed=4), 64, Hq)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("window", [0, 70])
def test_attention_both_forms_every_page(L, d, page, window):
    """Chunks of many rows beside single tokens, lengths around the pages' and the tiles' ends."""
    lens = [(70, 150), (page - 1, 1), (2 * page, 1), (31, 64), (0, 129)]
    _run_attn(L, *_attn_case(L, lens, 4, 2, d, page, seed=d + page), page, 4, window=window)


def test_attention_many_sequences_of_many_rows(L):
    """More sequences than a wave has lanes, more than a workgroup has threads, in both forms."""
    lens = [(i % 50, 17 + i % 9) for i in range(70)] + [(i % 70, 1) for i in range(60)]
    _run_attn(L, *_attn_case(L, lens, 6, 1, 64, 16, seed=20), 16, 6)
    lens = [(i % 5, 1 + i % 2) for i in range(600)]
    _run_attn(L, *_attn_case(L, lens, 2, 1, 64, 16, seed=21), 16, 2)


@pytest.mark.parametrize("lens,window", [([(0, 1100)], 0), ([(0, 1100), (300, 20), (700, 1)], 0), ([(0, 900), (0, 200)], 0), ([(900, 300)], 400)])
def test_attention_row_tiles_of_unlike_lengths(L, lens, window):
    """Between half and all of the workgroups that fill the device: row tiles cut in two, or not, alone and beside tokens."""
    _run_attn(L, *_attn_case(L, lens, 32, 8, 64, 64, seed=33), 64, 32, window=window)


def test_attention_more_sequences_than_the_plan_has_threads(L):
    """Sequences of 0 to 2 new tokens and some of many among 2100, cut in pieces and not, tokens of none behind them."""
    lens = [(i % 37, (i + 1) % 3) for i in range(2100)]
    lens[5], lens[1030], lens[2099] = (700, 3), (900, 70), (0, 90)
    q, parts, table, kv, starts = _attn_case(L, lens, 2, 1, 64, 16, seed=30, trailing=5)
    o, lse = torch.full((starts[-1] + 5, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((starts[-1] + 5, 2), 7.0, device="cuda")
    ref, rl, ob, lb = R.attention(q[:starts[-1]], R.Cache(*parts), table, kv, starts, 16)
    L.attn_cache(q.cuda(), _device_cache(L, parts), table.cuda(), _i32(kv), _i32(starts), out=(o, lse))
    R.near(o[:-5], ref, ob, "o")
    R.near(lse[:-5], rl, lb, "lse")
    assert bool((o[-5:] == 7).all()) and bool((lse[-5:] == 7).all())


@pytest.mark.parametrize("more", [90, 400])
def test_attention_tables_of_many_sequences_that_break_their_rules(L, more):
    """As test_attention_tables_that_break_their_rules, with many sequences behind the first."""
    lens = [(40, 30)] + [(9, 1)] * more
    q, parts, table, kv, starts = _attn_case(L, lens, 4, 2, 64, 16, seed=31)
    o, lse, ob, lb = R.attention(q, R.Cache(*parts), table, kv, starts, 16)
    wild = table.clone()
    wild[1:] = torch.tensor([-(2 ** 31), 2 ** 31 - 1, 12345678, -5, 99, 7], dtype=torch.int32)
    st = _i32(starts)
    for s in (st.flip(0), torch.where(torch.arange(more + 2, device="cuda") % 2 == 0, st, 2 ** 31 - 1), torch.full_like(st, -(2 ** 31))):
        s = s.to(torch.int32)
        s[0], s[1] = 0, 30
        for kv1 in (_i32([70] + [2 ** 31 - 1] * more), _i32([70] + [-5] * more)):
            s[2:] = s[2:].clamp(min=30)   # (rows from 30 on may be several sequences')
            got = L.attn_cache(q.cuda(), _device_cache(L, parts), wild.cuda(), kv1, s)
            R.near(got[0][:30], o[:30], ob[:30], "o")
            R.near(got[1][:30], lse[:30], lb[:30], "lse")


@pytest.mark.parametrize("S", [80, 300])
def test_captured_plan_follows_the_lengths(L, S):
    """Many sequences, short and in pieces, captured once and replayed with other lengths and starts, eager work between."""
    T = 2 * S
    lens = [(900, 2)] * S
    q, parts, table, _, _ = _attn_case(L, lens, 4, 1, 64, 16, seed=32, poison=False)
    c, td, qd = _device_cache(L, parts), table.cuda(), q.cuda()
    steps = []
    for i in range(4):
        n = [(7 * s + i) % 3 for s in range(S)]
        n[i] += 20
        kv = [min(902, (s * 53 * (i + 1)) % 880 + n[s]) for s in range(S)]
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
        torch.randn(1000, 1000, device="cuda").sum().item()


@pytest.mark.parametrize("scale", [-0.1, 0.0, 3.0])
@pytest.mark.parametrize("lens", [[(200, 1), (30, 4)], [(100, 180)]])
def test_attention_scales(L, lens, scale):
    """Logits of either sign, none, and so large that the softmax is one key."""
    for page in (16, 64):
        _run_attn(L, *_attn_case(L, lens, 4, 2, 128, page, seed=22), page, 4, scale=scale)


@pytest.mark.parametrize("d,page", [(128, 64), (64, 16), (256, 64)])
def test_attention_value_scales_far_apart(L, d, page):
    """Pages whose values lie 2^140 apart; a page of scale 0."""
    q, parts, table, kv, starts = _attn_case(L, [(250, 1), (60, 200), (3, 90)], 4, 2, d, page, seed=23)
    for s in range(3):
        for j in range(table.shape[1]):
            if int(table[s, j]) >= 0:
                parts[3][int(table[s, j])] = [2.0 ** 70, 2.0 ** -70, 1.0, 0.0, 2.0 ** -100][(s + j) % 5]
    _run_attn(L, q, parts, table, kv, starts, page, 4)


def test_attention_logits_that_keep_growing(L):
    """Keys whose logits rise and fall by hundreds along the sequence: the running maximum moves in most tiles."""
    for lens, page in (([(600, 1)], 64), ([(100, 500)], 64), ([(100, 500)], 16)):
        q, parts, table, kv, starts = _attn_case(L, lens, 2, 1, 128, page, seed=24)
        for j in range(-(-kv[0] // page)):
            parts[2][int(table[0, j])] = 2.0 ** (-8 + (j * page) // 64)
        _run_attn(L, q, parts, table, kv, starts, page, 2)


def test_attention_shared_pages_and_no_table(L):
    """Two sequences that share the pages of a prefix; tables of no columns; no sequences."""
    q, parts, table, kv, starts = _attn_case(L, [(100, 40), (100, 40)], 4, 2, 128, 32, seed=25)
    table[1, :3] = table[0, :3]
    _run_attn(L, q, parts, table, kv, starts, 32, 4)
    cache, qd = _device_cache(L, parts), q.cuda()
    none = torch.empty(2, 0, dtype=torch.int32, device="cuda")
    o, lse = L.attn_cache(qd, cache, none, _i32([0, 5]), _i32(starts))
    assert not o[:40].any() and bool((lse[:40] == -math.inf).all())        # a length of 0
    assert not o[40:75].any() and torch.isnan(o[75:]).all()               # 5 keys, none in the table: the last 5 rows see them
    for t in L.attn_cache(qd[:0], cache, none[:0], _i32([]), _i32([0])):
        assert t.shape[0] == 0
    before = [t.clone() for t in cache]
    new = torch.randn(80, 2, 128, dtype=torch.bfloat16, device="cuda")
    L.kv_append(new, new, cache, none, _i32([0, 5]), _i32(starts))
    L.kv_append(new[:0], new[:0], cache, none[:0], _i32([]))
    for a, b in zip(before, cache):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_attention_tables_that_break_their_rules(L):
    """Starts that decrease, overlap or pass T, negative lengths, wild table entries of the other sequences: the rows that
    belong to the first sequence alone, and its pages, are right (the kernels bound every index they take from the tables)."""
    Hq, H, d, page = 4, 2, 64, 16
    q, parts, table, kv, starts = _attn_case(L, [(40, 30), (0, 20), (9, 50)], Hq, H, d, page, seed=26)
    ref = R.Cache(*parts)
    o, lse, ob, lb = R.attention(q, ref, table, kv, starts, page)
    wild = table.clone()
    wild[1] = torch.tensor([-(2 ** 31), 2 ** 31 - 1, 12345678, -5, 99][:wild.shape[1]] + [7] * max(0, wild.shape[1] - 5), dtype=torch.int32)
    for s1, kv1 in (([0, 30, 50, 100], [70, -7, 59]), ([0, 30, 20, 100], [70, 20, 59]), ([0, 30, 5000, 100], [70, 20, 59])):
        got = L.attn_cache(q.cuda(), _device_cache(L, parts), wild.cuda(), _i32(kv1), _i32(s1))
        n = min([30] + s1[1:])   # (rows from 20 on are the third sequence's too where it starts there)
        R.near(got[0][:n], o[:n], ob[:n], "o")
        R.near(got[1][:n], lse[:n], lb[:n], "lse")
        cache = _device_cache(L, parts)
        new = torch.randn(100, 2, H, d, generator=_gen(27)).to(torch.bfloat16)
        nd = new.cuda()
        L.kv_append(nd[:, 0], nd[:, 1], cache, wild.cuda(), _i32(kv1), _i32(s1))
        want = R.Cache(*parts)
        R.append(want, new[:, 0], new[:, 1], table[:1], kv[:1], starts[:2], page)
        for j in range(5):
            g = int(table[0, j])
            assert torch.equal(cache.k[g].cpu().float().double().nan_to_num(7e9), want.k[g].nan_to_num(7e9))
            assert torch.equal(cache.v[g].cpu().float().double().nan_to_num(7e9), want.v[g].nan_to_num(7e9))


def test_binding_refuses(L):
    """Wrong types, shapes, strides and devices of every argument, before anything is launched."""
    q = torch.zeros(3, 4, 64, dtype=torch.bfloat16, device="cuda")
    k = torch.zeros(3, 2, 64, dtype=torch.bfloat16, device="cuda")
    w, rope = torch.ones(64, device="cuda"), L.rope_table(8, 64)
    pos = torch.zeros(3, dtype=torch.int32, device="cuda")
    bad = [dict(q=q.cpu()), dict(q=q.half()), dict(q=q[0]), dict(k=k.float()), dict(k=k[:2]), dict(v=k[:, :1]), dict(q=q.transpose(1, 2)),
           dict(q_weight=w.half()), dict(q_weight=w[:32]), dict(k_weight=w.cpu()), dict(rope=rope.double()), dict(rope=rope[0]),
           dict(rope=rope[:, ::2]), dict(positions=pos.long()), dict(positions=pos[:2]), dict(out=(q, None, None)),
           dict(out=(q.float(), k, k)), dict(out=(q[:2], k, k))]
    for kw in bad:
        with pytest.raises(ValueError):
            L.qk_norm_rope(**{**dict(q=q, k=k, v=k, q_weight=w, k_weight=w, rope=rope, positions=pos), **kw})
    wide = torch.zeros(3, 4, 65, dtype=torch.bfloat16, device="cuda")[..., :64]
    for kw in (dict(q=wide), dict(q=q, eps=-1.0), dict(q=q, rope=L.rope_table(8, 24))):
        with pytest.raises(L.LampError):
            L.qk_norm_rope(**kw)
    cache = L.kv_cache(6, 2, 64, 16)
    table, kv = torch.zeros(3, 2, dtype=torch.int32, device="cuda"), _i32([1, 1, 1])
    st = _i32([0, 1, 2, 3])
    parts = [dict(cache=cache._replace(k=cache.k.view(torch.uint8))), dict(cache=cache._replace(v=cache.k)), dict(cache=cache._replace(k_scale=cache.k_scale[:3])),
             dict(cache=cache._replace(v_scale=cache.v_scale.double())), dict(block_table=table.long()), dict(block_table=table[0]),
             dict(block_table=table.t()), dict(kv_lens=kv.long()), dict(kv_lens=kv[:2]), dict(q_start=st[:3]), dict(q_start=st.float()),
             dict(kv_lens=kv.cpu())]
    base = dict(cache=cache, block_table=table, kv_lens=kv, q_start=st)
    for kw in parts + [dict(k=k.half()), dict(v=k.float()), dict(k=k[:, :1], v=k[:, :1]), dict(k=k[0], v=k[0]), dict(k=q, v=q), dict(k_weight=w.half())]:
        with pytest.raises(ValueError):
            L.kv_append(**{**dict(k=k, v=k), **base, **kw})
    for kw in parts + [dict(q=q.float()), dict(q=q[0]), dict(q=q.cpu()), dict(out=(q, w)), dict(out=(q.float(), torch.zeros(3, 4, device="cuda"))),
                       dict(workspace=torch.zeros(9)), dict(q=torch.zeros(3, 4, 128, dtype=torch.bfloat16, device="cuda"))]:
        with pytest.raises(ValueError):
            L.attn_cache(**{**dict(q=q), **base, **kw})
    with pytest.raises(ValueError):
        L.attn_cache(q[:2], cache, table, kv)      # without q_start: one token for each sequence
    for kw in (dict(window=-1), dict(causal=False, window=3), dict(scale=math.nan)):
        with pytest.raises(L.LampError):
            L.attn_cache(q, **base, **kw)
    with pytest.raises(L.LampError):
        L.attn_cache(torch.zeros(3, 3, 64, dtype=torch.bfloat16, device="cuda"), **base)
    long = torch.zeros(3, 40, dtype=torch.int32, device="cuda")
    with pytest.raises(L.LampError):               # a workspace that is too small
        L.attn_cache(q, cache, long, kv, st, workspace=torch.zeros(512, dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()


def test_attention_rows_that_see_nothing_and_rows_of_no_sequence(L):
    """kv_lens below the new tokens (negative positions), length 0, and rows behind the last sequence."""
    Hq, H, d, page = 4, 2, 128, 16
    g = _gen(8)
    parts = R.random_cache(8, H, page, d, g)
    table = torch.tensor([[1, 2], [-1, -1], [3, 4]], dtype=torch.int32)
    kv, starts = [3, 0, 20], [0, 8, 10, 15]
    q = torch.randn(20, Hq, d, generator=g).to(torch.bfloat16)
    ref = R.Cache(*parts)
    o, lse, ob, lb = R.attention(q, ref, table, kv, starts, page)
    out = (torch.full((20, Hq, d), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((20, Hq), 7.0, device="cuda"))
    got = L.attn_cache(q.cuda(), _device_cache(L, parts), table.cuda(), _i32(kv), _i32(starts), out=out)
    assert got[0].data_ptr() == out[0].data_ptr()
    R.near(got[0][:15], o[:15], ob[:15], "o")
    R.near(got[1][:15], lse[:15], lb[:15], "lse")
    assert torch.equal(got[1][:5].cpu(), torch.full((5, Hq), -math.inf)) and not got[0][:5].any()
    assert bool((got[0][15:] == 7.0).all()) and bool((got[1][15:] == 7.0).all())


@pytest.mark.parametrize("n,d", [(1, 128), (9, 64), (200, 128), (150, 256)])
def test_attention_missing_pages(L, n, d):
    """A row that sees a missing page is NaN; rows whose window (or position) leaves it out are not."""
    Hq, H, page = 4, 1, 32
    q, parts, table, kv, starts = _attn_case(L, [(300, n), (40, 1)], Hq, H, d, page, seed=9)
    table[0, 2] = -1
    table[0, 9] = parts[0].shape[0]
    for window in (0, 20, 150):
        _run_attn(L, q, parts, table, kv, starts, page, Hq, window=window)
    # a length beyond the table's reach
    kv2 = [kv[0] + 5000, kv[1]]
    got = L.attn_cache(q.cuda(), _device_cache(L, parts), table.cuda(), _i32(kv2), _i32(starts))
    assert torch.isnan(got[0][:n]).all() and torch.isnan(got[1][:n]).all() and torch.isfinite(got[0][n:]).all()


@pytest.mark.parametrize("n,Hq,d,window", [(1, 4, 128, 0), (6, 4, 64, 0), (6, 2, 256, 9), (120, 4, 128, 0), (120, 4, 128, 50), (90, 2, 256, 0),
                                            (150, 1, 64, 70)])
def test_attention_nan_reaches_only_rows_that_see_it(L, n, Hq, d, window):
    """NaN keys, values and queries: values channel by channel."""
    page, H = 16, 1
    q, parts, table, kv, starts = _attn_case(L, [(50, n)], Hq, H, d, page, seed=10)
    kc, vc = parts[0].view(torch.uint8), parts[1].view(torch.uint8)
    L0 = kv[0]
    for back, chan in ((1, 3), (n // 2 + 1, 40), (n + 20, 41)):
        j = L0 - back
        vc[int(table[0, j // page]), 0, chan, j % page] = NAN_CODES[back % 2]
    if n > 1:
        j = L0 - 2
        kc[int(table[0, j // page]), 0, j % page, 5] = NAN_CODES[0]
    q[0, 0, 0] = math.nan
    _run_attn(L, q, parts, table, kv, starts, page, Hq, window=window)


def test_attention_strides_streams_and_repeats(L):
    """Heads sliced from a wider tensor, a non-default stream, bit-equal repeats, a given workspace of any contents."""
    lens, Hq, H, d, page = ATTN[5]
    q, parts, table, kv, starts = _attn_case(L, lens, Hq, H, d, page, seed=11, stride=2, trailing=3)
    first = _run_attn(L, q, parts, table, kv, starts, page, Hq)
    n = starts[-1]
    cache, qd = _device_cache(L, parts), q.cuda()
    wide = torch.full((table.shape[0], 3 * table.shape[1]), 9999, dtype=torch.int32, device="cuda")
    wide[:, :table.shape[1]] = table.cuda()   # a table whose rows lie farther apart
    need = L.attn_cache_workspace_size(q.shape[0], len(kv), Hq, H, d, page, table.shape[1])
    ws = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device="cuda")
    kvd, st = _i32(kv), _i32(starts)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        second = L.attn_cache(qd[:, :Hq], cache, wide[:, :table.shape[1]], kvd, st, workspace=ws)
    s.synchronize()
    for a, b in zip(first, second):
        assert torch.equal(a[:n].view(torch.int16 if a.dtype == torch.bfloat16 else torch.int32),
                           b[:n].view(torch.int16 if b.dtype == torch.bfloat16 else torch.int32))


def test_offsets_beyond_32_bits(L):
    """A pool of over 4 GB of keys: the last pages appended to and read."""
    H, d, page = 8, 128, 64
    pages = 70000
    cache = L.kv_cache(pages, H, d, page)
    assert cache.k.numel() > 1 << 32
    g = _gen(12)
    T = 100
    new = torch.randn(T, 2, H, d, generator=g).to(torch.bfloat16)
    q = torch.randn(T, 2 * H, d, generator=g).to(torch.bfloat16)
    table = torch.tensor([[pages - 1, pages - 2]], dtype=torch.int32)
    nd = new.cuda()
    L.kv_append(nd[:, 0], nd[:, 1], cache, table.cuda(), _i32([T]), _i32([0, T]))
    got = L.attn_cache(q.cuda(), cache, table.cuda(), _i32([T]), _i32([0, T]))
    small = [t[-2:].cpu() for t in cache]
    zero = [torch.zeros(2, H, page, d), torch.zeros(2, H, d, page), torch.zeros(2, H), torch.zeros(2, H)]
    ref = R.Cache(*zero)
    local = torch.tensor([[1, 0]], dtype=torch.int32)
    bounds = R.append(ref, new[:, 0], new[:, 1], local, [T], [0, T], page)
    _same_cache(L.KVCache(*small), ref, bounds, "last pages")
    o, lse, ob, lb = R.attention(q, R.Cache(*small), local, [T], [0, T], page)
    R.near(got[0], o, ob, "o")
    R.near(got[1], lse, lb, "lse")


# ---------------------------------------------------------------- together

def _serve(L, x, w, rope, cache, table, kv, st, pos, Hq, Hkv):
    """One layer's step: x [T,(Hq+2Hkv),d] from the projection."""
    q, k, v = x.split([Hq, Hkv, Hkv], dim=1)
    q = L.qk_norm_rope(q, q_weight=w[0], rope=rope, positions=pos)[0]
    L.kv_append(k, v, cache, table, kv, st, k_weight=w[1], rope=rope)
    return L.attn_cache(q, cache, table, kv, st)


def test_prompt_then_tokens_as_served(L):
    """Prompts of two sequences, then single tokens, through the three operators: each step against attention in 64
    bits over the cache as it stands, and the cache against the definition."""
    Hq, Hkv, d, page = 8, 2, 128, 32
    g = _gen(13)
    w = [(1 + 0.2 * torch.randn(d, generator=g)) for _ in range(2)]
    rope = L.rope_table(256, d, 1e4, device="cpu")
    wd, rd = [t.cuda() for t in w], rope.cuda()
    pages, table, _, _ = R.layout([(0, 100), (0, 90)], page, seed=13)
    cache = L.kv_cache(pages, Hkv, d, page)
    ref = R.Cache(*cache)
    have = [0, 0]
    for new in ([70, 33], [1, 1], [1, 1], [3, 0], [1, 40], [1, 1]):
        starts = [0, new[0], new[0] + new[1]]
        kv = [have[i] + new[i] for i in range(2)]
        x = torch.randn(starts[-1], Hq + 2 * Hkv, d, generator=g).to(torch.bfloat16)
        pos = torch.cat([torch.arange(have[i], kv[i]) for i in range(2)]).int()
        got = _serve(L, x.cuda(), wd, rd, cache, table.cuda(), _i32(kv), _i32(starts), pos.cuda(), Hq, Hkv)
        bounds = R.append(ref, x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], table, kv, starts, page, w[1], rope)
        _same_cache(cache, ref, bounds, "cache")
        ref = R.Cache(*cache)   # (codes next to a rounding border may differ by one: go on from the device's)
        q = L.qk_norm_rope(x.cuda()[:, :Hq], q_weight=wd[0], rope=rd, positions=pos.cuda())[0].cpu()
        o, lse, ob, lb = R.attention(q, ref, table, kv, starts, page)
        R.near(got[0], o, ob, "o")
        R.near(got[1], lse, lb, "lse")
        have = kv


def test_prompt_into_the_prompt_pass(L):
    """The norms' head-major outputs are what attn_fwd reads: equal to it on the same rows laid out by torch."""
    B, N, Hq, Hkv, d = 1, 200, 4, 2, 128
    g = _gen(14)
    x = torch.randn(B, N, Hq + 2 * Hkv, d, generator=g).to(torch.bfloat16).cuda()
    w = (1 + 0.2 * torch.randn(d, generator=g)).cuda()
    rope = L.rope_table(N, d, 1e6)
    q, k, v = x.split([Hq, Hkv, Hkv], dim=2)
    a = L.qk_norm_rope(q, k, v, w, w, rope)
    pos = torch.arange(N, dtype=torch.int32, device="cuda")
    tq, tk, _ = L.qk_norm_rope(q[0], k[0], None, w, w, rope, pos)
    b = (tq.transpose(0, 1)[None].contiguous(), tk.transpose(0, 1)[None].contiguous(), v.transpose(1, 2).contiguous())
    for s, t in zip(L.attn_fwd(*a), L.attn_fwd(*b)):
        assert torch.equal(s, t)


def test_captured_step_follows_the_lengths(L):
    """A decode step captured once and replayed while the lengths grow in place, eager work between the replays."""
    Hq, Hkv, d, page, S = 8, 2, 128, 16, 3
    g = _gen(15)
    w = [torch.ones(d, device="cuda") for _ in range(2)]
    rope = L.rope_table(4096, d, 1e4)
    pages, table, _, _ = R.layout([(0, 900)] * S, page, seed=15)
    lens = [5, 300, 511]
    parts = R.random_cache(pages, Hkv, page, d, g)
    cache, eager = _device_cache(L, parts), _device_cache(L, parts)
    td, kv = table.cuda(), _i32(lens)
    xs = [torch.randn(S, Hq + 2 * Hkv, d, generator=g).to(torch.bfloat16).cuda() for _ in range(6)]
    x, pos = xs[0].clone(), torch.zeros(S, dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _serve(L, x, w, rope, eager, td, kv, None, pos, Hq, Hkv)   # loads the code
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    cache, eager = _device_cache(L, parts), _device_cache(L, parts)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kv.add_(1)
        torch.sub(kv, 1, out=pos)
        out = _serve(L, x, w, rope, cache, td, kv, None, pos, Hq, Hkv)
    ekv = _i32(lens)
    for i, xi in enumerate(xs):
        x.copy_(xi)
        graph.replay()
        torch.cuda.synchronize()
        ekv += 1
        want = _serve(L, xi, w, rope, eager, td, ekv, None, ekv - 1, Hq, Hkv)
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1]), "replay %d" % i
        for a, b in zip(cache, eager):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), "replay %d" % i
        torch.randn(1000, 1000, device="cuda").sum().item()
