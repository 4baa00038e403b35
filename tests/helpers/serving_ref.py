"""A cache with given contents and the serving operators on it in 64 bits, one sequence and head at a time.

Bytes that no operator may use (rows behind the last distant token, pages no table lists, ring slots not
written yet) hold NaN."""
import math

import torch

D, PAGE = 64, 64
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def filled_cache(dar, seed, dtype, Hkv, dd, w, lens, group=None, pages=None, spare=1, values=1.0, device="cuda"):
    """A DarCache holding lens[b] tokens; members of group i list the same first pages[i] pages, which only the
    first member's table names (the others hold -1 there) when they are all distant for it."""
    B = len(lens)
    g = torch.Generator().manual_seed(seed)
    need = [-(-max(0, n - w) // PAGE) for n in lens]
    common = [pages[group[b]] if group and group[b] >= 0 and max(0, lens[b] - w) >= PAGE * pages[group[b]] else 0
              for b in range(B)]
    total = sum(n - c for n, c in zip(need, common)) + sum(pages or ()) + spare
    ids = torch.randperm(total, generator=g).tolist()
    maxp = max(1, max(need, default=0), max(pages or [0]))
    table = torch.full((B, maxp), -1, dtype=torch.int32)
    first = {}
    full = [[] for _ in range(B)]  # the pages that each sequence really reads
    for b in range(B):
        mine = []
        if common[b]:
            leader = group[b] in first
            if not leader:
                first[group[b]] = [ids.pop() for _ in range(common[b])]
            mine = list(first[group[b]])
            if not leader:
                table[b, :common[b]] = torch.tensor(mine, dtype=torch.int32)
        rest = [ids.pop() for _ in range(need[b] - common[b])]
        if rest:
            table[b, common[b]:need[b]] = torch.tensor(rest, dtype=torch.int32)
        full[b] = mine + rest
    c = dar.DarCache(B, Hkv, dd, w, maxp, total, dtype=DT[dtype], block_table=table, device=device)
    nan = float("nan")
    kd, vd = (torch.full((total, Hkv, PAGE, dd), nan) for _ in range(2))
    for b in range(B):
        n = max(0, lens[b] - w)
        for i, pg in enumerate(full[b]):
            rows = min(PAGE, n - i * PAGE)
            if torch.isnan(kd[pg, :, :rows]).any():
                for t in (kd, vd):
                    t[pg, :, :rows] = torch.randn((Hkv, rows, dd), generator=g) * values
    wk, wv = (torch.full((B, Hkv, w, D), nan) for _ in range(2))
    for b in range(B):
        m = min(lens[b], w)
        for t in (wk, wv):
            t[b, :, :m] = torch.randn((Hkv, m, D), generator=g) * values
    for t, x in ((c.pool_kd, kd), (c.pool_vd, vd), (c.win_k, wk), (c.win_v, wv)):
        t.copy_(x)
    c.seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))
    return c, full


def operands(seed, dtype, B, Hq, Hkv, dd, q_std=1.0, device="cuda"):
    g = torch.Generator().manual_seed(seed + 1)
    q = (torch.randn((B, Hq, D), generator=g) * q_std).to(DT[dtype]).to(device)
    Uk, Uv = ((torch.randn((Hkv, dd, D), generator=g) * dd ** -0.5).to(device) for _ in range(2))
    return q, Uk, Uv


def contents(c, full, b):
    """Distant keys and values [Hkv][n][dd] and ring keys and values by position [Hkv][nwin][64], in 64 bits."""
    L = int(c.seq_lens[b])
    near = min(L, c.w)
    n = L - near
    pg = torch.tensor(full[b], dtype=torch.long)
    out = []
    for t in (c.pool_kd, c.pool_vd):
        x = t.cpu().double()[pg].permute(1, 0, 2, 3).reshape(c.Hkv, -1, c.d_down)
        out.append(x[:, :n])
    slots = torch.arange(n, L) % c.w
    for t in (c.win_k, c.win_v):
        out.append(t[b].cpu().double()[:, slots])
    return out


def attend(q, kd, vd, k, v, Uk, Uv, scale=D ** -0.5):
    """One sequence: q [Hq][64] in 64 bits -> output [Hq][64], weights [Hq][L], and for tolerances sum p |v| lifted
    by |Uv| [Hq][64] and the largest sum of absolute products that a score is made of."""
    Hkv, G = kd.shape[0], q.shape[0] // kd.shape[0]
    out, wts, mag, top = [], [], [], 0.0
    for h in range(q.shape[0]):
        g = h // G
        keys = torch.cat((kd[g] @ Uk[g], k[g]))
        vals = torch.cat((vd[g] @ Uv[g], v[g]))
        s = keys @ q[h] * scale
        p = torch.exp(s - s.max())
        p = p / p.sum()
        n = kd.shape[1]
        out.append(p @ vals)
        wts.append(p)
        mag.append((p[:n] @ vd[g].abs()) @ Uv[g].abs() + p[n:] @ v[g].abs())
        absolute = torch.cat((kd[g].abs() @ (Uk[g].abs() @ q[h].abs()), k[g].abs() @ q[h].abs()))
        top = max(top, float(absolute.max()) * scale)
    return torch.stack(out), torch.stack(wts), torch.stack(mag), top


def tolerances(dtype, out, mag, top):
    """How far an output may be off, element by element.

    Scores: chains of at most 64 + 64 fp32 multiply-adds, the split of q~ into bf16 terms (2^-16 with two) and a few
    more roundings: each relative 2^-24 (or 2^-16) of the absolute products' sum `top`.  An error d of a score
    changes its weight by the factor e^d, numerator and sum alike: 2 d.  Weights as bf16 operands: 2^-8 of sum p |v|.
    exp2 and the sums: 2^-18 of it.  The output's own rounding: half a step."""
    bf = dtype == "bf16"
    d = top * (140 * 2.0 ** -24 + (2.0 ** -16 if bf else 0.0))
    return mag * (math.expm1(2 * d) + 2.0 ** -18 + (2.0 ** -8 if bf else 0.0)) \
        + out.abs() * torch.finfo(DT[dtype]).eps / 2 + 1e-30


def weight_tolerance(p, old, top):
    """As above without operands of 8 bits (q~ in three bf16 terms: 2^-24), and two roundings of the total."""
    return p * (math.expm1(2 * top * 150 * 2.0 ** -24) + 2.0 ** -18) + (p + old.abs()) * 2.0 ** -23 + 1e-30


def evict(kd, vd, k, v, w8, keep, protect, w):
    """One head: distant rows [n][dd], ring rows by position, totals [slots] -> the same after eviction."""
    n = kd.shape[0]
    if n <= keep:
        return kd, vd, k, v, w8
    order = sorted(range(protect, n), key=lambda j: (-(w8[j] if w8[j] == w8[j] else -math.inf), w8[j] != w8[j], j))
    stays = set(range(protect)) | set(order[:keep - protect])
    holes = [j for j in range(keep) if j not in stays]
    movers = [j for j in range(keep, n) if j in stays]
    assert len(holes) == len(movers)
    kd, vd, w8 = kd.clone(), vd.clone(), list(w8)
    for to, at in zip(holes, movers):
        kd[to], vd[to], w8[to] = kd[at], vd[at], w8[at]
    window = w8[n:n + w]
    w8[keep:n + w] = window + [0.0] * (n - keep)
    return kd, vd, k, v, w8
