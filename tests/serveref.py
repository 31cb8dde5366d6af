"""The serving operators in plain 64-bit arithmetic on the CPU, one sequence,
page and head after another, and the error bounds their kernels are held to.

A rounding is off by at most half a step: 2^-8 of the value in bf16, 2^-24 in
fp32, 2^-4 in e4m3 (half its smallest step, 2^-10, below 2^-6)."""
import math
import random

import torch

BF16, F32, E4M3 = 2.0 ** -8, 2.0 ** -24, 2.0 ** -4
# norm and rotation in fp32: a sum of d <= 256 squares (16 in sequence in a
# lane, 4 additions over lanes), the mean, eps, root, division, two products,
# two products and an addition of the rotation: below 32 roundings
NORM_ERR = 32 * F32


def norm_rope(x, w, table, pos, eps):
    """(y, bound on the fp32 error) of rows x [n, d] at positions pos; w, table may be None."""
    y = x.double()
    err = torch.zeros_like(y)
    if w is not None:
        y = y / torch.sqrt(y.pow(2).mean(-1, keepdim=True) + eps) * w.double()
        err = y.abs() * NORM_ERR
    if table is None:
        return y, err
    rot = table.shape[1]
    h = rot // 2
    z = torch.full((x.shape[0], rot), math.nan, dtype=torch.float64)
    ok = (pos >= 0) & (pos < table.shape[0])
    z[ok] = table[pos[ok]].double()
    c, s = z[:, :h], z[:, h:]
    a, b = y[:, :h], y[:, h:rot]
    out = torch.cat([a * c - b * s, b * c + a * s, y[:, rot:]], 1)
    mag = a.abs() + b.abs()
    err = torch.cat([mag * NORM_ERR, mag * NORM_ERR, err[:, rot:]], 1)
    return out, err


def e4m3(x):
    """x rounded to nearest even to e4m3 (|x| <= 448), as values."""
    e = (torch.frexp(x.abs())[1] - 1).clamp(min=-6)
    step = torch.ldexp(torch.ones_like(x), e - 3)
    return torch.round(x / step) * step


def need_scale(x):
    """Smallest power of two s >= 2^-100 with max |finite x| <= 448 s."""
    f = x[torch.isfinite(x)].abs()
    m = float(f.max()) if f.numel() else 0.0
    e = -100
    while m > 448.0 * 2.0 ** e:
        e += 1
    return 2.0 ** e


class Cache:
    """Codes (as values) and scales on the CPU: k [pages,H,page,d], v [pages,H,d,page]."""

    def __init__(self, k, v, ks, vs):
        self.k, self.v, self.ks, self.vs = (t.cpu().float().double() for t in (k, v, ks, vs))

    def dense(self, table_row, length, h, page):
        """(k, v) [length, d] of one sequence and head (pages that are missing: NaN)."""
        ks, vs = [], []
        for j in range(-(-length // page)):
            g = int(table_row[j]) if j < len(table_row) else -1
            if 0 <= g < self.k.shape[0]:
                ks.append(self.k[g, h] * self.ks[g, h])
                vs.append((self.v[g, h] * self.vs[g, h]).T)
            else:
                ks.append(torch.full((page, self.k.shape[3]), math.nan, dtype=torch.float64))
                vs.append(torch.full((page, self.k.shape[3]), math.nan, dtype=torch.float64))
        if not ks:
            z = torch.zeros((0, self.k.shape[3]), dtype=torch.float64)
            return z, z
        return torch.cat(ks)[:length], torch.cat(vs)[:length]


def append(ref, k, v, table, kv_lens, q_start, page, w=None, rope=None, eps=1e-6):
    """Appends to the Cache `ref`; returns the bounds (same layouts) of what
    the stored values (code * scale) may be off, 0 for the slots not new."""
    ke, ve = torch.zeros_like(ref.k), torch.zeros_like(ref.v)
    for s in range(len(kv_lens)):
        a, e = q_start[s], q_start[s + 1]
        p0 = kv_lens[s] - (e - a)
        pages = {}
        for i in range(e - a):
            p = p0 + i
            j = p // page
            if p >= 0 and j < table.shape[1] and 0 <= int(table[s, j]) < ref.k.shape[0]:
                pages.setdefault(int(table[s, j]), []).append((p, a + i))
        for g, toks in pages.items():
            pos, rows = torch.tensor([t[0] for t in toks]), [t[1] for t in toks]
            f, n = int(pos[0]) % page, len(toks)
            for h in range(ref.k.shape[1]):
                y, yerr = norm_rope(k[rows, h], w, rope, pos, eps)
                z = v[rows, h].double()
                for x, err, scale, codes, bound in ((y, yerr, ref.ks, ref.k[g, h], ke[g, h]),
                                                    (z, torch.zeros_like(z), ref.vs, ref.v[g, h].T, ve[g, h].T)):
                    x = torch.where(torch.isfinite(x), x, math.nan)
                    now = need_scale(x)
                    if f > 0:
                        old = float(scale[g, h])
                        now = max(now, old)
                        codes[:f] = e4m3(codes[:f] * (old / now))
                    codes[f:f + n] = e4m3(x / now)
                    scale[g, h] = now
                    # half a step of the value, and one more where the fp32 error can move it over a border
                    half = torch.clamp(x.abs() * E4M3, min=now * 2.0 ** -10)
                    bound[f:f + n] = torch.where(err > 0, 2 * half + err, 0.0)
    return ke, ve


def attention(q, ref, table, kv_lens, q_start, page, causal=True, window=0, scale=None):
    """(o, lse, bound of o, bound of lse) for q [T,Hq,d]; rows of no sequence hold NaN bounds."""
    T, Hq, d = q.shape
    H = ref.k.shape[1]
    G = Hq // H
    scale = d ** -0.5 if scale is None else scale
    o = torch.zeros(T, Hq, d, dtype=torch.float64)
    lse = torch.full((T, Hq), -math.inf, dtype=torch.float64)
    ob, lb = torch.full_like(o, math.nan), torch.full_like(lse, math.nan)
    for s in range(len(kv_lens)):
        a, e = q_start[s], q_start[s + 1]
        n, L = e - a, max(0, kv_lens[s])
        if n == 0:
            continue
        pos = kv_lens[s] - n + torch.arange(n)[:, None]
        j = torch.arange(L)[None]
        see = (j <= pos) if causal else (j < L).expand(n, L)
        if window:
            see = see & (j > pos - window)
        for h in range(H):
            k, v = ref.dense(table[s], L, h, page)
            for g in range(h * G, h * G + G):
                x = q[a:e, g].double()
                raw = x @ k.nan_to_num(nan=0.0).T * scale
                # (a NaN key makes the logit NaN, and only there)
                raw = torch.where(torch.isnan(k).any(1)[None], math.nan, raw)
                raw = torch.where(torch.isnan(x).any(1)[:, None], math.nan, raw)
                size = x.abs().nan_to_num() @ k.nan_to_num(nan=0.0).abs().T * abs(scale)
                l = torch.where(see, raw, -math.inf)
                some = see.any(1)
                ls = torch.where(some, torch.logsumexp(l, 1) if L else torch.full((n,), -math.inf, dtype=torch.float64), -math.inf)
                p = torch.where(see, torch.exp(l - ls[:, None]), 0.0) if L else l
                # NaN values reach the rows that see them, channel by channel
                hidden = ~torch.isnan(v)
                out = p @ v.nan_to_num(nan=0.0) if L else torch.zeros(n, d, dtype=torch.float64)
                if L:
                    out = torch.where(see.double() @ (~hidden).double() > 0, math.nan, out)
                out[~some] = 0.0
                # fp32 logits: d products summed, the scale and log2 e, and exp2 of a difference
                # of numbers up to their size (a few roundings of its own); the same again in the sum
                delta = ((d + 8) * F32 * torch.where(see, size, 0.0)).amax(1) if L else torch.zeros(n, dtype=torch.float64)
                delta = delta + 8 * F32 * (1 + l.masked_fill(~see, 0.0).nan_to_num().abs().amax(1) if L else 1.0) * 2
                sums = (L / 16 + 80) * F32   # additions one after another at most, over lanes, waves and pieces
                mag = p.nan_to_num() @ v.nan_to_num(nan=0.0).abs() if L else torch.zeros(n, d, dtype=torch.float64)
                o[a:e, g], lse[a:e, g] = out, ls
                # probabilities rounded to bf16, the result rounded to bf16
                ob[a:e, g] = (BF16 + 2 * delta[:, None] + 2 * sums) * mag * (1 + BF16) + BF16 * out.abs() + 1e-30
                lb[a:e, g] = 2 * delta + sums + 4 * F32 * ls.abs().nan_to_num(posinf=0.0, neginf=0.0) + 1e-30
    return o, lse, ob, lb


def near(got, want, bound, what):
    """got within bound of want, NaN and infinities in the same places."""
    got, want = got.cpu().double(), want.cpu()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    skip = torch.isnan(bound)
    assert torch.equal(torch.isnan(got) & ~skip, torch.isnan(want) & ~skip), what + ": NaN in other places"
    fine = torch.isfinite(want) & ~skip
    rest = ~fine & ~torch.isnan(want) & ~skip
    assert torch.equal(got[rest], want[rest]), what + ": infinities"
    off = (got - want).abs()[fine] - bound[fine]
    assert not off.numel() or float(off.max()) <= 0, "%s: %.3g over its bound" % (what, float(off.max()))


def layout(lens, page, extra=3, seed=0):
    """(pages, table [S][width], kv_lens, q_start) for (cached, new) lengths;
    shuffled pages, unused entries -1."""
    need = [max(0, -(-(a + b) // page)) for a, b in lens]
    pages, width = sum(need) + extra, max(need + [0]) + 1
    order = list(range(pages))
    random.Random(seed).shuffle(order)
    table = torch.full((len(lens), width), -1, dtype=torch.int32)
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
        at += n
    starts = [0]
    for _, b in lens:
        starts.append(starts[-1] + b)
    return pages, table, [a + b for a, b in lens], starts


def random_cache(pages, H, page, d, g, spread=3):
    """Codes of N(0,1)-like values (as uint8, e4m3fn bits) and scales 2^-spread .. 2^spread / 64."""
    def codes(*shape):
        x = torch.randn(shape, generator=g) * 64
        return x.clamp(-448, 448).to(torch.float8_e4m3fn)
    scale = lambda: torch.ldexp(torch.ones(pages, H), torch.randint(-spread, spread + 1, (pages, H), generator=g) - 6)  # noqa: E731
    return codes(pages, H, page, d), codes(pages, H, d, page), scale(), scale()
