"""The serving operators, as they are measured: what a server does around the
attention of its layers, from the projections' outputs to the attention over an
8-bit paged cache.

  norm_rope  lamp.qk_norm_rope: RMS norm of every query and key head and the
             position rotation, for prompts (outputs head-major) and for the
             tokens of a serving step
  append     lamp.kv_append: new keys (normed and rotated on the way) and values
             into the pages of an 8-bit cache (e4m3, a power-of-two scale for
             each page and head; V transposed within its page)
  attn       lamp.attn_cache: attention of a ragged batch of new tokens over
             that cache

A case's ragged lengths come from the case alone (`mix`), its values from the
seed.  `kv_lens` counts the new tokens: token i of n new ones of a sequence is
at position kv_lens - n + i.
"""
import math
import random

import torch

own = False

EPS = 1e-6
FP8 = torch.float8_e4m3fn
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def _norm(name, **kw):
    c = dict(op="norm_rope", form="tokens", B=1, N=1, Hq=32, Hkv=8, d=128, rot=128, dtype="bf16", base=1e6, start=0)
    c.update(kw)
    return dict(c, name=name) if name else c


def _append(name, **kw):
    c = dict(op="append", S=1, new_lo=1, new_hi=1, old_lo=0, old_hi=0, mix=0, page=64, Hkv=8, d=128, rot=128,
             dtype="bf16", norm=True, base=1e6)
    c.update(kw)
    return dict(c, name=name) if name else c


def _attn(name, **kw):
    c = dict(op="attn", S=1, new_lo=1, new_hi=1, old_lo=0, old_hi=0, chunk=0, mix=0, page=64, Hq=32, Hkv=8, d=128,
             causal=True, window=0)
    c.update(kw)
    return dict(c, name=name) if name else c


def listed():
    """The listed cases: each operator from its smallest calls to its largest."""
    return [
        # one user's next token: launch latency
        _norm("norm_rope_1_token", start=20010),
        # one chat prompt of odd length, split off the fused projection, into the prompt pass's layout
        _norm("norm_rope_prompt_1999", form="prompt", N=1999),
        # a batch of 8K prompts
        _norm("norm_rope_prompt_4x8192", form="prompt", B=4, N=8192),
        # a serving step: the next token of 32 sequences, at the ends of odd-length caches
        _append("append_32_tokens", S=32, old_lo=100, old_hi=4000, mix=1),
        # seven short prompts behind cached prefixes, fp32 projections, small heads, small pages
        _append("append_ragged_d64", S=7, new_lo=33, new_hi=1500, old_lo=0, old_hi=900, mix=2, page=16, d=64, rot=64,
                dtype="fp32", base=1e4),
        # a long prompt's whole cache
        _append("append_prompt_32k", new_lo=32768, new_hi=32768),
        # a first question: short, small heads, no grouping
        _attn("attn_37_tokens_d64", new_lo=37, new_hi=37, Hq=8, Hkv=8, d=64, page=16),
        # one user's next token against a long cache of odd length
        _attn("attn_1x20011", old_lo=20010, old_hi=20010),
        # a serving batch: the next token of 32 sequences against 8K caches
        _attn("attn_32x8192", S=32, old_lo=8191, old_hi=8191),
        # continuous batching: one prompt chunk beside the next tokens of 15 other sequences
        _attn("attn_chunk_and_15_tokens", S=16, old_lo=200, old_hi=8000, chunk=512, mix=3),
        # a local layer (d = 256, window 1024): chunks of two long documents
        _attn("attn_window_d256", S=2, new_lo=2048, new_hi=2048, old_lo=9000, old_hi=14000, mix=4, Hq=8, Hkv=4, d=256,
              window=1024, page=128),
        # an 8K prompt
        _attn("attn_prompt_8192", new_lo=8192, new_hi=8192),
    ]


def _log_int(rng, lo, hi):
    return lo if hi <= lo else min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo + 1), math.log(hi + 2)))) - 1)))


def _lens(c):
    """(cached, new) tokens of each sequence."""
    rng = random.Random(c["mix"])
    got = [(_log_int(rng, c["old_lo"], c["old_hi"]), _log_int(rng, c["new_lo"], c["new_hi"])) for _ in range(c["S"])]
    if c.get("chunk"):
        got[0] = (got[0][0], c["chunk"])
    return got


# a drawn case stays below the largest listed one, and its plain form in memory
_MOST_FLOPS = 4 * 32 * 128 * (8192 * 8193 // 2)
_MOST_SCORES = 1 << 30
_MOST_CACHE = 1 << 29


def draw(rng):
    """One more case of the ranges that the listed ones stand for."""
    while True:
        d = rng.choice([64, 128, 128, 256])
        hkv = rng.choice([1, 2, 4, 8])
        hq = hkv * rng.choice([1, 2, 3, 4, 8])
        page = rng.choice([16, 32, 64, 64, 128, 256])
        dtype = rng.choice(["bf16", "bf16", "fp32"])
        rot = rng.choice([d, d, d // 2])
        base = rng.choice([1e4, 1e6])
        mix = rng.randrange(1 << 20)
        op = rng.choice(["norm_rope", "append", "attn", "attn"])
        if op == "norm_rope":
            form = rng.choice(["tokens", "prompt"])
            n = _log_int(rng, 1, 512 if form == "tokens" else 16384)
            c = _norm("", form=form, B=1 if form == "tokens" else rng.choice([1, 1, 2, 4]), N=n, Hq=hq, Hkv=hkv, d=d,
                      rot=rot, dtype=dtype, base=base, start=rng.randrange(30000) if form == "tokens" else 0)
            if c["B"] * n * (hq + 2 * hkv) * d > 4 * 8192 * 48 * 128:
                continue
            return c
        one = rng.random() < 0.5
        S = _log_int(rng, 1, 64) if one else _log_int(rng, 1, 8)
        new_hi = 1 if one else _log_int(rng, 2, 8192)
        new_lo = 1 if one else max(1, new_hi // rng.choice([1, 4, 16]))
        old_hi = _log_int(rng, 0, 32000)
        old_lo = old_hi // rng.choice([1, 2, 10])
        if op == "append":
            c = _append("", S=S, new_lo=new_lo, new_hi=new_hi, old_lo=old_lo, old_hi=old_hi, mix=mix, page=page, Hkv=hkv,
                        d=d, rot=rot, dtype=dtype, norm=rng.random() < 0.7, base=base)
            if sum(a + b + page for a, b in _lens(c)) * hkv * d <= _MOST_CACHE // 8:
                return c
            continue
        window = rng.choice([0, 0, 0, 512, 1024])
        c = _attn("", S=S, new_lo=new_lo, new_hi=new_hi, old_lo=old_lo, old_hi=old_hi, mix=mix, page=page, Hq=hq, Hkv=hkv,
                  d=d, window=window, causal=window > 0 or rng.random() < 0.85,
                  chunk=_log_int(rng, 16, 1024) if one and rng.random() < 0.3 else 0)
        ln = _lens(c)
        longest = max(a + b for a, b in ln) + page
        if S * hq * max(b for _, b in ln) * longest > _MOST_SCORES or S * longest * hkv * d > _MOST_CACHE:
            continue
        if work(c)["flops"] <= _MOST_FLOPS:
            return c


# ---------------------------------------------------------------- inputs

def _rope_table(n, rot, base):
    inv = base ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot)
    ang = torch.arange(n, device="cuda", dtype=torch.float64)[:, None] * inv
    return torch.cat([ang.cos(), ang.sin()], -1).float()


def _gen(seed):
    g = torch.Generator("cuda")
    g.manual_seed(1000003 * (seed + 1) + 29)
    return lambda *shape: torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def _quantised(x):
    """(codes, scale) of x [pages, Hkv, a, b]: e4m3 and the power of two for each page and head."""
    m, e = torch.frexp(x.abs().amax((-1, -2)))
    s = torch.ldexp(torch.ones_like(m), e - 9 + (m > 0.875).int())
    return (x / s[..., None, None]).to(FP8), s


def _cache(case, randn, seed):
    """A filled cache: pages in shuffled order (unused entries of the table hold -1), keys with heavy-tailed channels."""
    page, hkv, d = case["page"], case["Hkv"], case["d"]
    ln = _lens(case)
    need = [-(-(a + b) // page) for a, b in ln]
    pages, width = sum(need) + 3, max(need) + 1
    order = list(range(pages))
    random.Random(seed).shuffle(order)
    table = [[-1] * width for _ in ln]
    at = 0
    for s, n in enumerate(need):
        table[s][:n] = order[at:at + n]
        at += n
    gain = (0.5 * randn(1, hkv, 1, d)).exp()
    k, ks = _quantised(randn(pages, hkv, page, d) * gain)
    v, vs = _quantised(randn(pages, hkv, d, page))
    starts = [0]
    for _, b in ln:
        starts.append(starts[-1] + b)
    dev = dict(device="cuda", dtype=torch.int32)
    return dict(k=k, v=v, k_scale=ks, v_scale=vs, table=torch.tensor(table, **dev), kv_lens=torch.tensor([a + b for a, b in ln], **dev),
                q_start=torch.tensor(starts, **dev)), starts[-1], max(b for _, b in ln), gain


def prepare(case, seed):
    """What a server has in hand before the call, on the GPU."""
    randn = _gen(seed)
    d = case["d"]
    if case["op"] == "norm_rope":
        B, N, hq, hkv, t = case["B"], case["N"], case["Hq"], case["Hkv"], TYPES[case["dtype"]]
        qkv = (randn(B, N, hq + 2 * hkv, d) * (0.5 * randn(1, 1, hq + 2 * hkv, d)).exp()).to(t)
        qkv = qkv if case["form"] == "prompt" else qkv[0]
        q, k, v = qkv.split([hq, hkv, hkv], dim=-2)
        st = dict(q=q, k=k, v=v if case["form"] == "prompt" else None, rope=_rope_table(case["start"] + N, case["rot"], case["base"]),
                  q_weight=(1 + 0.2 * randn(d)).to(t), k_weight=(1 + 0.2 * randn(d)).to(t))
        st["positions"] = None if case["form"] == "prompt" else (case["start"] + torch.arange(N, device="cuda")).int()
    elif case["op"] == "append":
        st, total, _, gain = _cache(case, randn, seed)
        t, hkv = TYPES[case["dtype"]], case["Hkv"]
        kv = randn(total, 2, hkv, d)
        kv[:, 0] *= gain[:, :, 0]
        kv = kv.to(t)
        st.update(k_new=kv[:, 0], v_new=kv[:, 1], rope=_rope_table(int(max(a + b for a, b in _lens(case))), case["rot"], case["base"]),
                  k_weight=(1 + 0.2 * randn(d)).to(t) if case["norm"] else None)
    else:
        st, total, st_max, gain = _cache(case, randn, seed)
        q = randn(total, case["Hq"], d) / gain.repeat_interleave(case["Hq"] // case["Hkv"], 1)[:, :, 0] * 1.5
        st.update(q=q.to(torch.bfloat16), max_new=st_max)
    st["case"] = case
    return st


# ---------------------------------------------------------------- the operators

def _normed(x, w, rows, rot):
    """x [..., H, d] normed over d by the gain w (None: not normed) and its first rot channels rotated; rows [..., 1, rot]."""
    y = x.float()
    if w is not None:
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS) * w.float()
    h = rot // 2
    cos, sin = rows[..., :h], rows[..., h:]
    a, b = y[..., :h], y[..., h:rot]
    return torch.cat([a * cos - b * sin, b * cos + a * sin, y[..., rot:]], -1)


def _plain_norm_rope(st):
    c = st["case"]
    if c["form"] == "prompt":
        rows = st["rope"][:c["N"], None]
        q, k = _normed(st["q"], st["q_weight"], rows, c["rot"]), _normed(st["k"], st["k_weight"], rows, c["rot"])
        return tuple(x.to(torch.bfloat16).transpose(1, 2).contiguous() for x in (q, k, st["v"]))
    rows = st["rope"][st["positions"].long(), None]
    q, k = _normed(st["q"], st["q_weight"], rows, c["rot"]), _normed(st["k"], st["k_weight"], rows, c["rot"])
    return q.to(torch.bfloat16), k.to(torch.bfloat16), None


def _plain_write(codes, scale, new, page_of, slot, first, touched, transposed):
    """New values [T, Hkv, d] into the codes and scales of one of the caches."""
    need = torch.zeros_like(scale).scatter_reduce_(0, page_of[:, None].expand(-1, scale.shape[1]), new.abs().amax(-1), "amax")
    m, e = torch.frexp(need)
    need = torch.ldexp(torch.ones_like(m), (e - 9 + (m > 0.875).int()).clamp(min=-100))
    old = torch.where(first[:, None] > 0, scale, 0.0)
    s = torch.where(touched[:, None], torch.maximum(old, need), scale)
    # the slots before the first new one keep their values under the new scale, those behind the new ones stay as they are
    slots = torch.arange(codes.shape[3 if transposed else 2], device="cuda")
    ratio = torch.where((touched[:, None] & (slots < first[:, None]))[:, None], (scale / s)[..., None], 1.0)
    codes.copy_((codes.float() * (ratio[:, :, None] if transposed else ratio[..., None])).to(FP8))
    scale.copy_(s)
    got = (new / s[page_of][..., None]).to(FP8).view(torch.uint8)
    raw = codes.view(torch.uint8)
    if transposed:
        raw[page_of, :, :, slot] = got
    else:
        raw[page_of, :, slot] = got


def _places(st, total):
    """(sequence, position) of each new token."""
    t = torch.arange(total, device="cuda")
    start = st["q_start"].long()
    seq = torch.searchsorted(start[1:], t, right=True)
    return seq, st["kv_lens"].long()[seq] - start[seq + 1] + t


def _plain_append(st):
    c = st["case"]
    page, total, pages = c["page"], st["k_new"].shape[0], st["k"].shape[0]
    seq, pos = _places(st, total)
    page_of, slot = st["table"].long()[seq, pos // page], pos % page
    first = torch.full((pages,), page, device="cuda").scatter_reduce_(0, page_of, slot, "amin")
    touched = first < page
    _plain_write(st["k"], st["k_scale"], _normed(st["k_new"], st["k_weight"], st["rope"][pos, None], c["rot"]), page_of, slot, first,
                 touched, False)
    _plain_write(st["v"], st["v_scale"], st["v_new"].float(), page_of, slot, first, touched, True)
    return st["k"], st["v"], st["k_scale"], st["v_scale"]


def _plain_attn(st):
    c = st["case"]
    S, hq, hkv, d, page, n = c["S"], c["Hq"], c["Hkv"], c["d"], c["page"], st["max_new"]
    G = hq // hkv
    table = st["table"].long().clamp(min=0)
    k = (st["k"][table].float() * st["k_scale"][table][..., None, None]).permute(0, 2, 1, 3, 4).reshape(S, hkv, -1, d)
    v = (st["v"][table].float() * st["v_scale"][table][..., None, None]).permute(0, 2, 1, 4, 3).reshape(S, hkv, -1, d)
    L = k.shape[2]
    start, lens = st["q_start"].long(), st["kv_lens"].long()
    i = torch.arange(n, device="cuda")
    new = start[1:] - start[:-1]
    live = i[None] < new[:, None]
    at = (start[:-1, None] + i[None]).clamp(max=st["q"].shape[0] - 1)
    q = st["q"][at].float().view(S, n, hkv, G, d).permute(0, 2, 3, 1, 4).reshape(S, hkv, G * n, d)
    x = torch.matmul(q, k.transpose(-1, -2)).mul_(d ** -0.5).view(S, hkv, G, n, L)
    j, p = torch.arange(L, device="cuda")[None, None], (lens[:, None] - new[:, None] + i[None])[..., None]
    see = (j < lens[:, None, None]) & ((j <= p) if c["causal"] else (p == p))
    if c["window"]:
        see = see & (j > p - c["window"])
    x.masked_fill_(~see[:, None, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    x.sub_(m).exp_()
    l = x.sum(-1, keepdim=True)
    o = torch.matmul(x.view(S, hkv, G * n, L), v).view(S, hkv, G, n, d) / torch.where(l > 0, l, 1.0)
    lse = (m + l.log())[..., 0]
    o = o.permute(0, 3, 1, 2, 4).reshape(S, n, hq, d)[live]
    return o.to(torch.bfloat16), lse.permute(0, 3, 1, 2).reshape(S, n, hq)[live]


def _own_run(st):
    from paper_2609_39361_amd import lamp
    c = st["case"]
    if c["op"] == "norm_rope":
        return lamp.qk_norm_rope(st["q"], st["k"], st["v"], q_weight=st["q_weight"], k_weight=st["k_weight"], rope=st["rope"],
                                 positions=st["positions"], eps=EPS)
    cache = lamp.KVCache(st["k"], st["v"], st["k_scale"], st["v_scale"])
    if c["op"] == "append":
        lamp.kv_append(st["k_new"], st["v_new"], cache, st["table"], st["kv_lens"], q_start=st["q_start"], k_weight=st["k_weight"],
                       rope=st["rope"], eps=EPS)
        return tuple(cache)
    return lamp.attn_cache(st["q"], cache, st["table"], st["kv_lens"], q_start=st["q_start"], causal=c["causal"], window=c["window"])


def run(state):
    """One call: (q, k, v), the cache's codes and scales, or (o, lse)."""
    if own:
        return _own_run(state)
    return {"norm_rope": _plain_norm_rope, "append": _plain_append, "attn": _plain_attn}[state["case"]["op"]](state)


# ---------------------------------------------------------------- what a pass cannot do without

def _seen(old, new, causal, window):
    """Visible pairs, and keys that some row sees, of one sequence."""
    L = old + new
    if not causal:
        return new * L, L
    if not window:
        return sum(range(old + 1, L + 1)), L
    return sum(min(p + 1, window) for p in range(old, L)), min(L, new + window - 1)


def work(case):
    d, e = case["d"], 4 if case.get("dtype") == "fp32" else 2
    if case["op"] == "norm_rope":
        rows = case["B"] * case["N"]
        heads = case["Hq"] + case["Hkv"] * (2 if case["form"] == "prompt" else 1)
        return {"bytes": rows * heads * d * (e + 2) + case["N"] * case["rot"] * 4 + 2 * d * e,
                "flops": rows * (case["Hq"] + case["Hkv"]) * d * 7}
    ln = _lens(case)
    if case["op"] == "append":
        total = sum(b for _, b in ln)
        return {"bytes": 2 * total * case["Hkv"] * d * (e + 1) + total * case["rot"] * 4, "flops": total * case["Hkv"] * d * 11}
    seen = [_seen(a, b, case["causal"], case["window"]) for a, b in ln]
    total = sum(b for _, b in ln)
    return {"bytes": 2 * sum(x[1] for x in seen) * case["Hkv"] * d + total * case["Hq"] * (4 * d + 4),
            "flops": 4 * case["Hq"] * d * sum(x[0] for x in seen)}


# ---------------------------------------------------------------- 64 bits, from the definitions

def _e4m3(x):
    e = (torch.frexp(x.abs())[1] - 1).clamp(min=-6)
    step = torch.ldexp(torch.ones_like(x), e - 3)
    return torch.round(x / step) * step


def _rotated64(x, w, pos, rot, table):
    """One head's rows x [n, d] (fp64) at positions pos."""
    if w is not None:
        x = x / (x.pow(2).mean(-1, keepdim=True) + EPS).sqrt() * w.double()
    z = torch.complex(x[:, :rot // 2], x[:, rot // 2:rot]) * torch.complex(table[pos, :rot // 2], table[pos, rot // 2:])
    return torch.cat([z.real, z.imag, x[:, rot:]], -1)


def _exact_norm_rope(st):
    c, table = st["case"], st["rope"].double()
    pos = torch.arange(c["N"], device="cuda") if st["positions"] is None else st["positions"].long()
    heads = lambda x, w: torch.stack([_rotated64(x[:, h].double(), w, pos, c["rot"], table) for h in range(x.shape[1])], 1)  # noqa: E731
    if c["form"] != "prompt":
        return heads(st["q"], st["q_weight"]), heads(st["k"], st["k_weight"]), None
    q, k = (torch.stack([heads(x[b], w).transpose(0, 1) for b in range(c["B"])]) for x, w in ((st["q"], st["q_weight"]), (st["k"], st["k_weight"])))
    return q, k, st["v"].double().permute(0, 2, 1, 3)


def _exact_append(st):
    c, table = st["case"], st["rope"].double()
    page, out, at = c["page"], [], 0
    ks, vs = st["k_scale"].double().clone(), st["v_scale"].double().clone()
    kc, vc = st["k"].double(), st["v"].double()
    for s, (old, new) in enumerate(_lens(c)):
        pos = torch.arange(old, old + new, device="cuda")
        y = torch.stack([_rotated64(st["k_new"][at:at + new, h].double(), st["k_weight"], pos, c["rot"], table) for h in range(c["Hkv"])], 0)
        z = st["v_new"][at:at + new].double().transpose(0, 1)
        at += new
        pages = st["table"][s].tolist()
        p = old
        while p < old + new:
            end = min(old + new, (p // page + 1) * page)
            g, f, m = pages[p // page], p % page, end - p
            for codes, scale, x, vt in ((kc, ks, y, False), (vc, vs, z, True)):
                x = x[:, p - old:end - old]
                need = torch.exp2(torch.ceil(torch.log2(x.abs().amax((1, 2)) / 448)).clamp(min=-100))
                now = torch.maximum(need, scale[g]) if f else need
                view = codes[g].transpose(1, 2) if vt else codes[g]
                view[:, :f] = _e4m3(view[:, :f] * (scale[g] / now)[:, None, None])
                view[:, f:f + m] = _e4m3(x / now[:, None, None])
                scale[g] = now
            p = end
    return kc, vc, ks, vs


def _exact_attn(st):
    c = st["case"]
    G, page, d = c["Hq"] // c["Hkv"], c["page"], c["d"]
    o = torch.empty(st["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(st["q"].shape[:2], dtype=torch.float64, device="cuda")
    at = 0
    for s, (old, new) in enumerate(_lens(c)):
        L = old + new
        pages = st["table"][s, :-(-L // page)].long()
        p, j = torch.arange(old, L, device="cuda")[:, None], torch.arange(L, device="cuda")[None]
        hide = torch.zeros(new, L, dtype=torch.bool, device="cuda")
        if c["causal"]:
            hide |= j > p
        if c["window"]:
            hide |= j <= p - c["window"]
        for h in range(c["Hkv"]):
            k = (st["k"][pages, h].double() * st["k_scale"][pages, h].double()[:, None, None]).reshape(-1, d)[:L]
            v = (st["v"][pages, h].double() * st["v_scale"][pages, h].double()[:, None, None]).transpose(1, 2).reshape(-1, d)[:L]
            for g in range(h * G, h * G + G):
                x = (st["q"][at:at + new, g].double() @ k.T / math.sqrt(d)).masked_fill_(hide, -math.inf)
                lse[at:at + new, g] = torch.logsumexp(x, -1)
                o[at:at + new, g] = torch.softmax(x, -1) @ v
        at += new
    return o, lse


def exact(case, seed):
    """What run() returns, from the operators' definitions in 64 bits."""
    return {"norm_rope": _exact_norm_rope, "append": _exact_append, "attn": _exact_attn}[case["op"]](prepare(case, seed))
