"""Serving operators over the mixed-dimension cache, as measurable cases.

Three operators work on one cache (the last ``w`` tokens of a sequence at full
width in a ring, older ones as ``d_down`` vectors in 64-token pages):

``shared``  a decode step for a batch whose sequences, in groups, share the
            first pages of their contexts: samples of one prompt, or requests
            behind one system prompt or document
``scored``  a decode step that also adds every token's attention weight, summed
            over the query heads of its KV head, to a running total
``evict``   eviction by those totals: per KV head the tokens with the largest
            ones stay, and the context gets shorter

``run`` computes them with elementary torch operations, or with the library's
entry points where ``own`` is set.  ``exact`` is the definition in 64 bits:
keys and values lifted one by one, no absorption.

A pass can be repeated on its state.  Totals that a pass adds to are set back
first, and so are the lengths, the totals and, where it turns, the ring of a
cache that a pass evicts from (the pages need no setting back: rows that move
stay where they were as well).
"""
from __future__ import annotations

import math
from types import SimpleNamespace

import torch

own = False

D = 64
PAGE = 64
DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}


# ----------------------------------------------------------------------- cases


def listed():
    return [
        # two samples of one short prompt on the smallest shape, in full precision: the least that is shared
        dict(name="shared_f32_pair", kind="shared", dtype="f32", B=2, Hq=4, Hkv=4, w=32, dd=16, groups=1, alone=0,
             Pmin=3, Pmax=3, extra=40, shuffled=False),
        # 32 samples of one prompt on the 160M shape
        dict(name="shared_160m_samples", kind="shared", dtype="bf16", B=32, Hq=12, Hkv=12, w=128, dd=16, groups=1,
             alone=0, Pmin=62, Pmax=62, extra=250, shuffled=False),
        # grouped-query serving of the 1B shape: four system prompts, some requests with none, recycled pages
        dict(name="shared_1b_prompts", kind="shared", dtype="bf16", B=64, Hq=32, Hkv=8, w=256, dd=16, groups=4,
             alone=5, Pmin=37, Pmax=256, extra=1500, shuffled=True),
        # 64 questions about one long document on the 1B shape
        dict(name="shared_1b_document", kind="shared", dtype="bf16", B=64, Hq=32, Hkv=8, w=256, dd=16, groups=1,
             alone=0, Pmin=508, Pmax=508, extra=600, shuffled=True),
        # one short chat turn on the 70M shape, still inside the window
        dict(name="scored_70m_b1", kind="scored", dtype="bf16", B=1, Hq=8, Hkv=8, w=128, dd=16, Lmin=101, Lmax=101,
             decay=1.0, shuffled=False),
        # full precision, two query heads a KV head, odd lengths
        dict(name="scored_f32", kind="scored", dtype="f32", B=3, Hq=8, Hkv=4, w=37, dd=16, Lmin=20, Lmax=1501,
             decay=0.9, shuffled=True),
        # batched serving of the 160M shape, the last step's weights alone
        dict(name="scored_160m", kind="scored", dtype="bf16", B=32, Hq=12, Hkv=12, w=128, dd=16, Lmin=4096,
             Lmax=4096, decay=0.0, shuffled=False),
        # grouped-query serving of the 1B shape with ragged contexts and recycled pages
        dict(name="scored_1b_gqa", kind="scored", dtype="bf16", B=64, Hq=32, Hkv=8, w=256, dd=16, Lmin=1024,
             Lmax=32768, decay=1.0, shuffled=True),
        # one conversation of the 70M shape goes back to its budget
        dict(name="evict_70m_b1", kind="evict", dtype="bf16", B=1, Hkv=8, w=128, dd=16, keep=896, protect=4, emin=128,
             emax=128, step=128, shuffled=False),
        # full precision, evicted counts that turn the ring
        dict(name="evict_f32_odd", kind="evict", dtype="f32", B=5, Hkv=4, w=100, dd=8, keep=777, protect=64, emin=0,
             emax=2600, step=1, shuffled=True),
        # the 160M shape: every sequence gives up half its context, and the ring turns
        dict(name="evict_160m_half", kind="evict", dtype="bf16", B=32, Hkv=12, w=128, dd=16, keep=2000, protect=4,
             emin=1968, emax=1968, step=1, shuffled=False),
        # the 1B shape: long contexts behind a protected prompt go back to a budget of 8192, whole windows at a time
        dict(name="evict_1b_gqa", kind="evict", dtype="bf16", B=64, Hkv=8, w=256, dd=16, keep=8192, protect=1024,
             emin=256, emax=16384, step=256, shuffled=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng):
    while True:
        Hkv, G = rng.choice((1, 2, 4, 8, 12, 16)), rng.choice((1, 1, 2, 3, 4, 8))
        if Hkv * G <= 32:
            return Hkv * G, Hkv


def draw(rng):
    kind = rng.choice(("shared", "scored", "evict"))
    f32 = rng.random() < 0.2
    dt = "f32" if f32 else "bf16"
    dd = rng.choice((8, 16, 16, 16, 32, 64))
    Hq, Hkv = _heads(rng)
    w = _log(rng, 16, 1024)
    B = _log(rng, 1, 16 if f32 else 64)
    shuffled = rng.random() < 0.5
    # no more than a quarter (fp32: an eighth) of 64 sequences of 32768 tokens, 8 KV heads, d_down 16
    most = 64 * 32768 * 8 * 16 / (8 if f32 else 4)
    if kind == "shared":
        B = max(2, B)
        P, extra = _log(rng, 1, 64 if f32 else 508), _log(rng, 1, 2000)
        while B > 2 and B * Hkv * ((64 * P + extra) * dd + w * D) > most:
            B = B // 2
        groups = rng.randint(1, max(1, min(6, B // 2)))
        return dict(kind=kind, dtype=dt, B=B, Hq=Hq, Hkv=Hkv, w=w, dd=dd, groups=groups,
                    alone=rng.randint(0, max(0, B - 2 * groups)) if rng.random() < 0.5 else 0,
                    Pmin=max(1, int(P * rng.uniform(0.1, 1.0))), Pmax=P, extra=extra, shuffled=shuffled)
    if kind == "scored":
        Lmax = _log(rng, 1, 4096 if f32 else 32768)
        while B > 1 and B * Hkv * (Lmax * dd + w * D) > most:
            B = B // 2
        return dict(kind=kind, dtype=dt, B=B, Hq=Hq, Hkv=Hkv, w=w, dd=dd, Lmin=max(1, int(Lmax * rng.uniform(0.1, 1))),
                    Lmax=Lmax, decay=rng.choice((1.0, 1.0, 0.0, 0.95)), shuffled=shuffled)
    keep, gone = _log(rng, 1, 8192), _log(rng, 1, 16384)
    while B > 1 and B * Hkv * ((keep + gone) * dd + w * D) > most:
        B = B // 2
    step = w if gone >= w and rng.random() < 0.5 else 1
    return dict(kind=kind, dtype=dt, B=B, Hkv=Hkv, w=w, dd=dd, keep=keep, protect=rng.choice((0, 4, keep // 8, keep)),
                emin=0 if rng.random() < 0.3 else gone // 2 // step * step, emax=gone // step * step, step=step,
                shuffled=shuffled)


def _spread(lo, hi, n):
    """n whole numbers spread over [lo, hi] in no particular order (multiples of the golden ratio)."""
    if lo == hi:
        return [lo] * n
    return [lo + int(math.modf((i + 1) * 0.6180339887498949)[0] * (hi - lo + 1)) for i in range(n)]


def _layout(case):
    """Tokens of each sequence; for "shared" also each sequence's group (-1: none) and each group's pages."""
    B, w = case["B"], case["w"]
    if case["kind"] == "scored":
        return _spread(case["Lmin"], case["Lmax"], B), None, None
    if case["kind"] == "evict":
        lo, hi = case["emin"] // case["step"], case["emax"] // case["step"]
        return [w + case["keep"] + case["step"] * e for e in _spread(lo, hi, B)], None, None
    pages = _spread(case["Pmin"], case["Pmax"], case["groups"])
    together = B - case["alone"]
    group = [(b * case["groups"]) // together if b < together else -1 for b in range(B)]
    group = [group[(b * 5 + 2) % B] for b in range(B)] if B % 5 else group  # requests come in any order
    own_pages = _spread(case["Pmin"], case["Pmax"], B)
    lens = [w + PAGE * (pages[g] if g >= 0 else own_pages[b]) + e
            for b, (g, e) in enumerate(zip(group, _spread(0, case["extra"], B)))]
    return lens, group, pages


# ---------------------------------------------------------------------- inputs


def _normal(g, shape, std=1.0, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=g)


def _block_table(case, lens, group, pages, seed):
    """Pages of the distant tokens: a group's first pages are the same in the rows of all its members."""
    need = [-(-max(0, n - case["w"]) // PAGE) for n in lens]
    common = [pages[g] if g >= 0 else 0 for g in group] if group else [0] * len(need)
    total = max(1, sum(n - c for n, c in zip(need, common)) + (sum(pages) if pages else 0))
    ids = torch.randperm(total, generator=torch.Generator().manual_seed(seed)) if case["shuffled"] \
        else torch.arange(total)
    table = torch.full((len(need), max(1, max(need))), -1, dtype=torch.int32)
    first, at = [], 0
    for n in pages or ():
        first.append(at)
        at += n
    for b, (n, c) in enumerate(zip(need, common)):
        if c:
            table[b, :c] = ids[first[group[b]]:first[group[b]] + c]
        table[b, c:n] = ids[at:at + n - c]
        at += n - c
    return table, total


def _totals(g, shape):
    """Weights summed over many steps: a few tokens hold most, many hold equal counts, some hold nothing."""
    t = torch.exp(2.0 * _normal(g, shape, dtype=torch.float32)) * 0.05
    u = torch.rand(shape, device="cuda", generator=g)
    return torch.where(u < 0.1, 0.0, torch.where(u < 0.3, torch.round(t * 16) / 16, t))


def prepare(case, seed):
    torch.cuda.set_device(0)
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt, B, Hkv, w, dd = DTYPE[case["dtype"]], case["B"], case["Hkv"], case["w"], case["dd"]
    lens, group, pages = _layout(case)
    table, total = _block_table(case, lens, group, pages, seed)
    i32 = dict(dtype=torch.int32, device="cuda")
    s = SimpleNamespace(case=case, lens=torch.tensor(lens, **i32), lens_host=lens, group_host=group)
    if own:
        from paper_2606_18587_gb300 import dar
        c = s.cache = dar.DarCache(B, Hkv, dd, w, table.shape[1], total, dtype=dt, block_table=table)
    else:
        c = s.cache = SimpleNamespace(
            win_k=torch.empty((B, Hkv, w, D), dtype=dt, device="cuda"),
            pool_kd=torch.empty((total, Hkv, PAGE, dd), dtype=dt, device="cuda"),
            block_table=table.cuda(), seq_lens=torch.empty(B, **i32))
        c.win_v, c.pool_vd = torch.empty_like(c.win_k), torch.empty_like(c.pool_kd)
    for t in (c.win_k, c.win_v, c.pool_kd, c.pool_vd):
        t.normal_(generator=g)
    c.seq_lens.copy_(s.lens)
    slots = table.shape[1] * PAGE + w
    if case["kind"] != "shared":
        s.totals = _totals(g, (B, Hkv, slots))
        s.totals.masked_fill_((torch.arange(slots, device="cuda") >= s.lens[:, None])[:, None], 0.0)
        s.weights = s.totals.clone()
    if case["kind"] == "evict":
        s.keep = torch.full((B,), case["keep"], **i32)
        s.protect = torch.full((B,), min(case["protect"], case["keep"]), **i32)
        s.turns = any((n - w - case["keep"]) % w for n in lens)
        if s.turns:
            s.ring = (c.win_k.clone(), c.win_v.clone())
        if own:
            s.workspace = dar.evict_workspace(c)
        return s
    s.q = _normal(g, (B, case["Hq"], D), 2.0, dt)  # scores of standard deviation 2
    s.Uk, s.Uv = (_normal(g, (Hkv, dd, D), dd ** -0.5, torch.float32) for _ in range(2))
    s.out = torch.empty_like(s.q)
    if group:
        s.group, s.pages = torch.tensor(group, **i32), torch.tensor(pages, **i32)
    if own:
        s.workspace = (dar.shared_decode_workspace if group else dar.scored_decode_workspace)(c, case["Hq"])
    return s


# ------------------------------------------------------------------ plain forms


def _attend(s):
    """Output and weights of one decode step, all sequences at once, in 32 bits.  Weights are
    [B][Hkv][G][slots of the ring, then the table's tokens], zero where a sequence holds nothing."""
    case, c = s.case, s.cache
    B, Hkv, w, dd = case["B"], case["Hkv"], case["w"], case["dd"]
    G, P = case["Hq"] // Hkv, c.block_table.shape[1]
    L = c.seq_lens.long()
    in_ring = (torch.arange(w, device="cuda") < L[:, None])[:, None, None]
    in_pages = (torch.arange(P * PAGE, device="cuda") < (L - w)[:, None])[:, None, None]
    pages = c.block_table.long().clamp(min=0)

    def paged(pool):
        x = pool[pages].permute(0, 2, 1, 3, 4).reshape(B, Hkv, P * PAGE, dd).float()
        return x.masked_fill_(~in_pages[:, 0, 0, None, :, None], 0.0)

    q = s.q.float().view(B, Hkv, G, D)
    qt = q @ s.Uk.mT
    near = (q @ c.win_k.float().mT).masked_fill_(~in_ring, -math.inf)
    far = (qt @ paged(c.pool_kd).mT).masked_fill_(~in_pages, -math.inf)
    scores = torch.cat((near, far), -1) * D ** -0.5
    p = torch.exp(scores - scores.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    v = c.win_v.float().masked_fill(~in_ring[:, 0, 0, None, :, None], 0.0)
    out = p[..., :w] @ v + (p[..., w:] @ paged(c.pool_vd)) @ s.Uv
    return out.reshape(B, case["Hq"], D).to(s.q.dtype), p


def _plain_scored(s):
    case, c, w = s.case, s.cache, s.case["w"]
    s.weights.copy_(s.totals)
    out, p = _attend(s)
    p = p.sum(2)
    L = c.seq_lens.long()[:, None]
    slot = torch.arange(w, device="cuda")[None]
    at = (L - 1) - ((L - 1 - slot) % w)  # the position that a ring slot holds
    step = torch.zeros_like(s.weights)
    step[..., :p.shape[-1] - w] = p[..., w:]
    step.scatter_add_(2, at.clamp(min=0)[:, None].expand(-1, case["Hkv"], -1),
                      torch.where(at >= 0, 1.0, 0.0)[:, None] * p[..., :w])
    held = (torch.arange(step.shape[-1], device="cuda") < L)[:, None]
    old = case["decay"] * s.weights if case["decay"] else 0.0
    s.weights.copy_(torch.where(held, old + step, s.weights))
    return dict(out=out, weights=s.weights)


def _set_back(s):
    c = s.cache
    c.seq_lens.copy_(s.lens)
    s.weights.copy_(s.totals)
    if s.turns:
        c.win_k.copy_(s.ring[0])
        c.win_v.copy_(s.ring[1])


def _held(s):
    c = s.cache
    return dict(pool_kd=c.pool_kd, pool_vd=c.pool_vd, win_k=c.win_k, win_v=c.win_v, seq_lens=c.seq_lens,
                weights=s.weights)


def _plain_evict(s):
    c, w = s.cache, s.case["w"]
    _set_back(s)
    L = c.seq_lens.long()
    n = (L - w).clamp(min=0)
    gone = (n - s.keep).clamp(min=0)
    keep = torch.where(gone > 0, s.keep, n)
    pos = torch.arange(s.weights.shape[-1], device="cuda")
    rank_of = s.weights.masked_fill((pos < s.protect[:, None])[:, None], math.inf)
    rank_of = rank_of.masked_fill_((pos >= n[:, None])[:, None], -math.inf)
    order = torch.sort(rank_of, dim=-1, descending=True, stable=True).indices
    rank = torch.empty_like(order).scatter_(2, order, pos.expand_as(order).contiguous())
    stays = rank < keep[:, None, None]
    hole = ~stays & (pos < keep[:, None])[:, None]
    mover = stays & (pos >= keep[:, None])[:, None]
    b, h, to = hole.nonzero(as_tuple=True)  # both ascending within each head, and equally many
    at = mover.nonzero(as_tuple=True)[2]
    page_to, page_at = (c.block_table.long()[b, x // PAGE] for x in (to, at))
    for pool in (c.pool_kd, c.pool_vd):
        pool[page_to, h, to % PAGE] = pool[page_at, h, at % PAGE]
    moved = s.weights.clone()
    moved[b, h, to] = s.weights[b, h, at]
    # the window's totals come down to the new end, and nothing is left behind it
    after = moved.gather(2, (pos + gone[:, None] * (pos >= keep[:, None])).clamp(max=len(pos) - 1)[:, None]
                         .expand_as(moved))
    after.masked_fill_(((pos >= (L - gone)[:, None]) & (pos < L[:, None]))[:, None], 0.0)
    s.weights.copy_(torch.where((pos < L[:, None])[:, None], after, moved))
    slot = (torch.arange(w, device="cuda") + gone[:, None]) % w
    slot = slot[:, None, :, None].expand_as(c.win_k)
    c.win_k.copy_(c.win_k.gather(2, slot))
    c.win_v.copy_(c.win_v.gather(2, slot))
    c.seq_lens.copy_(L - gone)
    return _held(s)


def run(s):
    kind = s.case["kind"]
    if not own:
        return _attend(s)[0] if kind == "shared" else _plain_scored(s) if kind == "scored" else _plain_evict(s)
    from paper_2606_18587_gb300 import dar
    if kind == "shared":
        return dar.dar_attn_decode_shared(s.cache, s.q, s.Uk, s.Uv, s.group, s.pages, s.workspace, out=s.out)
    if kind == "scored":
        if s.case["decay"]:
            s.weights.copy_(s.totals)
        dar.dar_attn_decode_scored(s.cache, s.q, s.Uk, s.Uv, s.weights, s.workspace, decay=s.case["decay"],
                                   out=s.out)
        return dict(out=s.out, weights=s.weights)
    _set_back(s)
    dar.dar_cache_evict(s.cache, s.weights, s.keep, s.workspace, protect=s.protect)
    return _held(s)


# ------------------------------------------------------------- necessary work


def work(case):
    lens, group, pages = _layout(case)
    Hkv, w, dd = case["Hkv"], case["w"], case["dd"]
    e = 4 if case["dtype"] == "f32" else 2
    row, small = 2 * D * e, 2 * dd * e  # keys and values of a token at either width
    nbytes = flops = 0
    if case["kind"] == "evict":
        keep, first = case["keep"], min(case["protect"], case["keep"])
        for L in lens:
            n = L - w
            if n <= keep:
                continue
            # totals have no order, so this many of the tokens that stay lie behind the budget
            moves = (keep - first) * (n - keep) / (n - first)
            nbytes += Hkv * (4 * (n - first) + moves * 2 * (small + 4) + 4 * (w + n - keep + w))
            if (n - keep) % w:
                nbytes += Hkv * w * 2 * row
        return dict(bytes=int(nbytes), flops=0)
    Hq = case["Hq"]
    for b, L in enumerate(lens):
        near = min(L, w)
        far = L - near
        own_far = far - (PAGE * pages[group[b]] if group and group[b] >= 0 else 0)
        nbytes += Hkv * (near * row + own_far * small) + 2 * Hq * D * e
        flops += Hq * (4 * near * D + 4 * far * dd + 4 * D * dd)
        if case["kind"] == "scored":
            nbytes += Hkv * L * (8 if case["decay"] else 4)
    if group:
        nbytes += sum(Hkv * PAGE * pages[g] * small for g in set(group) if g >= 0)
    nbytes += 2 * Hkv * D * dd * 4
    return dict(bytes=int(nbytes), flops=int(flops))


# ------------------------------------------------------------ the same in 64 bits


def _exact_step(s):
    """One sequence at a time: every key and value by position at full width, then softmax attention over them."""
    case, c = s.case, s.cache
    Hq, Hkv, w = case["Hq"], case["Hkv"], case["w"]
    Uk, Uv = s.Uk.double(), s.Uv.double()
    out = torch.empty(s.q.shape, dtype=torch.float64, device="cuda")
    weights = s.totals.double() if case["kind"] == "scored" else None
    for b, L in enumerate(s.lens_host):
        at = torch.arange(L, device="cuda")
        old, new = at[:max(0, L - w)], at[max(0, L - w):]
        page = c.block_table[b].long()[old // PAGE]
        k, v = (torch.cat((pool[page, :, old % PAGE].double().transpose(0, 1) @ U, ring[b][:, new % w].double()), 1)
                for pool, U, ring in ((c.pool_kd, Uk, c.win_k), (c.pool_vd, Uv, c.win_v)))
        q = s.q[b].double().view(Hkv, Hq // Hkv, D)
        p = torch.softmax(torch.einsum("ghd,gjd->ghj", q, k) / math.sqrt(D), -1)
        out[b] = torch.einsum("ghj,gjd->ghd", p, v).reshape(Hq, D)
        if weights is not None:
            weights[b, :, :L] = case["decay"] * weights[b, :, :L] + p.sum(1)
    return out if weights is None else dict(out=out, weights=weights)


def _exact_evict(s):
    """One head at a time: the totals above the last one that stays, then the first equal ones."""
    case, c, w = s.case, s.cache, s.case["w"]
    held = {n: (t.double() if t.is_floating_point() else t.clone()) for n, t in _held(s).items()}
    table = c.block_table.long()
    for b, L in enumerate(s.lens_host):
        n, keep, first = L - w, case["keep"], min(case["protect"], case["keep"])
        gone = n - keep
        if gone <= 0:
            continue
        for h in range(case["Hkv"]):
            t = s.totals[b, h, first:n]
            stays = torch.zeros(n, dtype=torch.bool, device="cuda")
            stays[:first] = True
            if keep > first:
                last = t.kthvalue(len(t) - (keep - first) + 1).values
                above = t > last
                equal = (t == last).nonzero()[:keep - first - int(above.sum()), 0]
                stays[first:] = above
                stays[first + equal] = True
            to, at = (~stays[:keep]).nonzero()[:, 0], keep + stays[keep:].nonzero()[:, 0]
            for name in ("pool_kd", "pool_vd"):
                pool = held[name]
                pool[table[b, to // PAGE], h, to % PAGE] = pool[table[b, at // PAGE], h, at % PAGE]
            weights = held["weights"][b, h]
            weights[to] = s.totals[b, h, at].double()
            weights[keep:keep + w] = s.totals[b, h, n:n + w].double()
            weights[keep + w:L] = 0.0
        for name in ("win_k", "win_v"):
            held[name][b] = held[name][b].roll(-(gone % w), 1)
        held["seq_lens"][b] = L - gone
    return held


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_evict(s) if case["kind"] == "evict" else _exact_step(s)
