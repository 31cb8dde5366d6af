"""The operators of long contexts and changing batches in plain arithmetic on the
CPU: integers, which the kernels' have to equal, and serveref's attention in 64
bits with its error bounds."""
import math

import torch

import serveref as R


def advance(lens, add, prefix, table, page, T, ring, state):
    """(kv_lens, q_start, positions, state, table, ring) of one step; lists, table and ring int32 tensors (copied)."""
    S, width, pages = len(lens), table.shape[1], len(ring)
    table, ring, old = table.clone(), ring.clone(), table
    held = [-(-n // page) for n in lens]
    new = [max(0, a) for a in add]
    need = [0 if add[s] < 0 else -(-(lens[s] + new[s]) // page) - held[s] for s in range(S)]
    kept = [min(held[s], prefix[s] // page if prefix else 0) for s in range(S)]
    back = [held[s] - kept[s] if add[s] < 0 else 0 for s in range(S)]
    why = (sum(need) > state[1]) + 2 * any(add[s] >= 0 and lens[s] + new[s] > width * page for s in range(S)) + 4 * (sum(new) > T)
    put, take, count = state[0] + state[1], state[0], state[1]
    no = why
    if sum(back) > pages - count:
        no |= 8
        back = [0] * S
    for s in range(S):
        for j in range(kept[s], kept[s] + back[s]):
            ring[put % pages] = old[s, j]
            put += 1
    kv, starts, positions = [], [0], []
    for s in range(S):
        n = 0 if why else new[s]
        for j in range(held[s], held[s] + (0 if why else need[s])):
            table[s, j] = ring[take % pages]
            take += 1
        kv.append(0 if add[s] < 0 else lens[s] + n)
        starts.append(starts[-1] + n)
        positions += range(lens[s], lens[s] + n)
    positions += [0] * (T - len(positions))
    return kv, starts, positions, [take % pages, put - take, sum(need), no], table, ring


def bounds(ref, got, table, kv_lens, q_start, page):
    """int8 [pages,H,2,d] that kv_bounds leaves where `got` was; ref: a serveref Cache."""
    got = got.clone()
    for s in range(len(kv_lens)):
        n = q_start[s + 1] - q_start[s]
        if n <= 0 or kv_lens[s] <= 0:
            continue
        for j in range(max(0, kv_lens[s] - n) // page, -(-kv_lens[s] // page)):
            g = int(table[s, j]) if j < table.shape[1] else -1
            if not 0 <= g < ref.k.shape[0]:
                continue
            x = ref.k[g, :, :min(page, kv_lens[s] - j * page)]
            none = torch.isnan(x).all(1)
            hi = torch.where(torch.isnan(x), -math.inf, x).amax(1)
            lo = torch.where(torch.isnan(x), math.inf, x).amin(1)
            got[g, :, 0] = torch.where(none, 0.0, torch.ceil(hi / 4)).to(torch.int8)
            got[g, :, 1] = torch.where(none, 0.0, torch.floor(lo / 4)).to(torch.int8)
    return got


def rounded(q):
    """Integers of bf16 q [G, d] (int64), and e."""
    f = torch.where(torch.isfinite(q.double()), q.double(), 0.0)
    m, e = float(f.abs().max()), -100
    while m > 127.0 * 2.0 ** e:
        e += 1
    return torch.round(f / 2.0 ** e).long(), e


def scores(q, rng, scale):
    """Scores (fp64, exact) of q [G, d] for ranges int8 [n, 2, d] with scales [n]."""
    x = rounded(q)[0][:, None]
    hi, lo = rng[:, 0].long(), rng[:, 1].long()
    return torch.maximum(x * hi, x * lo).sum(-1).amax(0).double() * scale.double()


def select(q, rng, ks, table, kv_lens, q_start, page, budget, first, last):
    """places int32 [T,H,budget]; rows of no sequence hold -2."""
    T, Hq, _ = q.shape
    H = ks.shape[1]
    out = torch.full((T, H, budget), -2, dtype=torch.int32)
    for s in range(len(kv_lens)):
        a, e = q_start[s], q_start[s + 1]
        for t in range(a, e):
            pos = kv_lens[s] - e + t
            n = min(pos // page + 1, table.shape[1]) if pos >= 0 else 0
            pg = table[s, :n].long()
            there = (pg >= 0) & (pg < ks.shape[0])
            at = torch.where(there, pg, 0)
            for h in range(H):
                x = scores(q[t, h * (Hq // H):(h + 1) * (Hq // H)], rng[at, h], ks[at, h]) if n else torch.zeros(0, dtype=torch.float64)
                x = torch.where(there, x, -math.inf)
                x[:first] = math.inf
                x[max(0, n - last):] = math.inf
                take = torch.sort(x, descending=True, stable=True)[1][:budget].sort()[0]
                out[t, h] = -1
                out[t, h, :len(take)] = take.int()
    return out


def attention_of_places(q, ref, table, kv_lens, q_start, page, places, scale=None):
    """As serveref.attention, of attn_pages."""
    T, Hq, d = q.shape
    H = ref.k.shape[1]
    G = Hq // H
    o = torch.zeros(T, Hq, d, dtype=torch.float64)
    lse = torch.full((T, Hq), -math.inf, dtype=torch.float64)
    ob, lb = torch.full_like(o, math.nan), torch.full_like(lse, math.nan)
    for h in range(H):
        one = R.Cache(ref.k[:, h:h + 1], ref.v[:, h:h + 1], ref.ks[:, h:h + 1], ref.vs[:, h:h + 1])
        for s in range(len(kv_lens)):
            for t in range(q_start[s], q_start[s + 1]):
                pos = kv_lens[s] - q_start[s + 1] + t
                mine = sorted(j for j in places[t, h].tolist() if 0 <= j < table.shape[1] and j * page <= pos)
                row = table[s, mine].unsqueeze(0) if mine else torch.zeros(1, 0, dtype=torch.int32)
                keys = sum(min(page, pos + 1 - j * page) for j in mine)
                got = R.attention(q[t:t + 1, h * G:(h + 1) * G], one, row, [keys], [0, 1], page, True, 0, scale)
                for x, y in zip((o, lse, ob, lb), got):
                    x[t, h * G:(h + 1) * G] = y[0]
    return o, lse, ob, lb


def shared_layout(groups, page, seed=0):
    """serveref.layout for groups [(prefix, [(own cached, new), ...]), ...]: (pages, table, kv_lens, q_start, prefix_lens,
    group_start), the rows of a group beginning with the same pages."""
    lens, prefix, starts = [], [], [0]
    for p, own in groups:
        lens += [(p + a, b) for a, b in own]
        prefix += [p] * len(own)
        starts.append(len(lens))
    pages, table, kv, q_start = R.layout(lens, page, seed=seed)
    for g, (p, own) in enumerate(groups):
        n = p // page
        if n and own:
            width = max(table.shape[1], n)
            if width > table.shape[1]:
                table = torch.nn.functional.pad(table, (0, width - table.shape[1]), value=-1)
            table[starts[g] + 1:starts[g + 1], :n] = table[starts[g], :n]
    return pages, table, kv, q_start, prefix, starts
