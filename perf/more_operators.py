"""Operators over a cache whose distant tokens are held in 4 bits, as measurable cases.

The last ``w`` tokens of a sequence stay at full width in a ring; the ``d_down``
vectors of older ones lie in 64-token pages, in groups of 16 entries (a whole
vector of 8) that share a scale:

    a = max |x|,  s = a / 7 rounded to 5 significant bits (at most 1.125 * 2^125),
    code = x / s rounded to the nearest whole number (ties to even), within +-7

so a stored value ``code * s`` has at most 8 significant bits and is a bf16 number.
A group with an infinite or NaN entry is NaN as a whole.

``append``   tokens join the sequences; the vectors of those that leave the window
             are formed, rounded to the storage type, quantised and written, and
             what was written is read back into pages of the storage type
``convert``  pages of an ordinary cache are quantised, and read back: contexts are
             parked between two turns, or a chunk that has just been processed is
``decode``   attention of one token of each sequence over ring and pages
``step``     a serving step, an append of one token and the attention behind it

``run`` computes them with elementary torch operations, or with the library's
entry points where ``own`` is set.  ``exact`` is the definition in 64 bits: sums in
one go, keys and values lifted one by one, no absorption.

A pass can be repeated on its state: an appending one sets the lengths back first,
and its ring already holds the tokens that join, so that the tokens that leave are
the same in every pass.
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
        # full precision, ragged numbers of tokens, some still within the window, the narrowest vectors
        dict(name="append_f32_odd", kind="append", dtype="f32", B=5, Hkv=4, w=37, dd=8, Lmin=0, Lmax=301, nmin=0,
             nmax=67, shuffled=True),
        # a token joins each sequence of the 160M shape
        dict(name="append_160m", kind="append", dtype="bf16", B=32, Hkv=12, w=128, dd=16, Lmin=4096, Lmax=4096,
             nmin=1, nmax=1, shuffled=False),
        # a batch of prompts of different lengths enters an empty 160M cache
        dict(name="append_prompts_160m", kind="append", dtype="bf16", B=32, Hkv=12, w=128, dd=16, Lmin=0, Lmax=0,
             nmin=1000, nmax=4096, shuffled=False),
        # the last tokens of a few contexts, in full precision and wider vectors
        dict(name="convert_f32_odd", kind="convert", dtype="f32", B=3, Hkv=4, w=37, dd=32, Lmin=20, Lmax=1501, new=333,
             shuffled=True),
        # all contexts of the 1B shape are parked and taken up again
        dict(name="convert_1b_gqa", kind="convert", dtype="bf16", B=64, Hkv=8, w=256, dd=16, Lmin=1024, Lmax=32768,
             new=0, shuffled=True),
        # one chat of the 70M shape
        dict(name="decode_70m_b1", kind="decode", dtype="bf16", B=1, Hq=8, Hkv=8, w=128, dd=16, Lmin=901, Lmax=901,
             shuffled=False),
        # full precision, three query heads a KV head, odd lengths, one of them empty
        dict(name="decode_f32_odd", kind="decode", dtype="f32", B=4, Hq=12, Hkv=4, w=37, dd=16, Lmin=0, Lmax=1501,
             shuffled=True),
        # batched serving of the 160M shape
        dict(name="decode_160m", kind="decode", dtype="bf16", B=32, Hq=12, Hkv=12, w=128, dd=16, Lmin=4096, Lmax=4096,
             shuffled=False),
        # grouped-query serving of the 1B shape with ragged contexts and recycled pages
        dict(name="decode_1b_gqa", kind="decode", dtype="bf16", B=64, Hq=32, Hkv=8, w=256, dd=16, Lmin=1024,
             Lmax=32768, shuffled=True),
        # a long-context point of the window x d_down sweep: narrow window, the widest vectors
        dict(name="decode_sweep_w64_dd64", kind="decode", dtype="bf16", B=16, Hq=16, Hkv=16, w=64, dd=64, Lmin=16384,
             Lmax=16384, shuffled=False),
        # a short chat turn of the 70M shape: one token joins and attends
        dict(name="step_70m_b1", kind="step", dtype="bf16", B=1, Hq=8, Hkv=8, w=128, dd=16, Lmin=300, Lmax=300,
             shuffled=False),
        # the serving step of the 160M shape
        dict(name="step_160m", kind="step", dtype="bf16", B=32, Hq=12, Hkv=12, w=128, dd=16, Lmin=4096, Lmax=4096,
             shuffled=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng):
    while True:
        Hkv, G = rng.choice((1, 2, 4, 8, 12, 16)), rng.choice((1, 1, 2, 3, 4, 5, 8))
        if Hkv * G <= 32:
            return Hkv * G, Hkv


def draw(rng):
    kind = rng.choice(("append", "convert", "decode", "decode", "step"))
    f32 = rng.random() < 0.2
    Hq, Hkv = _heads(rng)
    case = dict(kind=kind, dtype="f32" if f32 else "bf16", Hkv=Hkv, w=_log(rng, 16, 1024),
                dd=rng.choice((8, 16, 16, 16, 32, 64)), shuffled=rng.random() < 0.5)
    B = _log(rng, 1, 16 if f32 else 64)
    Lmax = _log(rng, 1, 4096 if f32 else 32768)
    nmin = nmax = 0
    if kind == "convert":  # contexts that have left the window
        Lmax += case["w"]
    if kind in ("append", "step"):
        nmax = 1 if kind == "step" or rng.random() < 0.4 else _log(rng, 2, 256 if f32 else 4096)
        nmin = nmax if nmax == 1 else int(nmax * rng.uniform(0.0, 1.0))
        if nmax > 64:
            Lmax = rng.choice((0, Lmax // 4))
    # no more than a quarter (fp32: a sixteenth) of 64 sequences of 32768 tokens, 8 KV heads, d_down 16, and of what
    # joins no more than half of 32 prompts of 4096 tokens, 12 heads
    most = 64 * 32768 * 8 * 16 / (16 if f32 else 4)
    while B > 1 and (B * Hkv * (Lmax * case["dd"] + case["w"] * D) > most or B * Hkv * nmax * case["dd"] > 3 << 22):
        B = B // 2
    case.update(B=B, Lmin=int(Lmax * rng.uniform(0.0, 1.0)), Lmax=Lmax)
    if kind == "append":
        case.update(nmin=nmin, nmax=nmax)
    elif kind == "convert":
        case.update(new=rng.choice((0, 0, _log(rng, 1, 2048))))
    else:
        case.update(Hq=Hq)
    return case


def _spread(lo, hi, n):
    """n whole numbers spread over [lo, hi] in no particular order (multiples of the golden ratio), both ends among
    them where there is room."""
    if lo == hi:
        return [lo] * n
    v = [lo + int(math.modf((i + 1) * 0.6180339887498949)[0] * (hi - lo + 1)) for i in range(n)]
    v[-1] = lo
    v[0] = hi
    return v


def _layout(case):
    """Tokens of each sequence before the pass, and how many join."""
    B = case["B"]
    n = [1] * B if case["kind"] == "step" else [0] * B
    if case["kind"] == "append":
        n = _spread(case["nmin"], case["nmax"], B)[::-1]
    return _spread(case["Lmin"], case["Lmax"], B), n


# ---------------------------------------------------------------------- inputs


def _normal(g, shape, std=1.0, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=g)


def _tables(first, last, shuffled, seed, columns):
    """A block table [B][columns] with a page for every one that holds tokens [first[b], last[b]), and their number."""
    pages = [(b, p) for b in range(len(last)) for p in range(first[b] // PAGE, -(-last[b] // PAGE))
             if last[b] > first[b]]
    ids = torch.randperm(len(pages), generator=torch.Generator().manual_seed(seed)) if shuffled \
        else torch.arange(len(pages))
    table = torch.full((len(last), max(1, columns)), -1, dtype=torch.int32)
    if pages:
        b, p = torch.tensor(pages).unbind(1)
        table[b, p] = ids.int()
    return table, max(1, len(pages))


def _joined(ring, new, L, n):
    """The ring once the first n[b] tokens of `new` have joined sequence b."""
    w = ring.shape[2]
    slot = torch.arange(w, device="cuda")
    at = (L + n)[:, None] - 1 - ((L + n)[:, None] - 1 - slot) % w  # the position that a slot holds then
    i = at - L[:, None]
    row = i.clamp(0, new.shape[2] - 1)[:, None, :, None].expand(-1, ring.shape[1], -1, D)
    return torch.where((i >= 0)[:, None, :, None], new.gather(2, row), ring)


def prepare(case, seed):
    return _state(case, seed, own)


def _state(case, seed, own):
    torch.cuda.set_device(0)
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt, B, Hkv, w, dd = DTYPE[case["dtype"]], case["B"], case["Hkv"], case["w"], case["dd"]
    lens, n = _layout(case)
    before = [max(0, L - w) for L in lens]  # distant tokens
    after = [max(0, L + m - w) for L, m in zip(lens, n)]
    columns = -(-max(after) // PAGE)
    table, total = _tables([0] * B, after, case["shuffled"], seed, columns)
    i32 = dict(dtype=torch.int32, device="cuda")
    s = SimpleNamespace(case=case, lens=torch.tensor(lens, **i32), lens_host=lens, n_host=n)
    s.n = torch.tensor(n, **i32)
    if own:
        from paper_2606_18587_gb300 import dar
    kd, vd = (_normal(g, (total, Hkv, PAGE, dd), 1.0, dt) for _ in range(2))
    ring = [_normal(g, (B, Hkv, w, D), 1.0, dt) for _ in range(2)]
    if max(n):
        s.k_new, s.v_new = (_normal(g, (B, Hkv, max(n), D), 1.0, dt) for _ in range(2))
        s.Dk, s.Dv = (_normal(g, (Hkv, D, dd), D ** -0.5, torch.float32) for _ in range(2))
        ring = [_joined(r, x, s.lens.long(), s.n.long()) for r, x in zip(ring, (s.k_new, s.v_new))]
    if own:
        pages = dar.DarCache(B, Hkv, dd, w, table.shape[1], total, dtype=dt, block_table=table)
        c = dar.DarCacheQ4.beside(pages)
    else:
        pages = SimpleNamespace(win_k=ring[0], win_v=ring[1], block_table=table.cuda(), seq_lens=s.lens.clone())
        c = SimpleNamespace(**vars(pages))
    s.cache = c
    if own:
        pages.pool_kd.copy_(kd)
        pages.pool_vd.copy_(vd)
        pages.win_k.copy_(ring[0])
        pages.win_v.copy_(ring[1])
        pages.seq_lens.copy_(s.lens)
    else:
        pages.pool_kd, pages.pool_vd = kd, vd
    if case["kind"] == "convert":
        first = [max(0, m - case["new"]) if case["new"] else 0 for m in before]
        s.pages = pages
        s.first = torch.tensor(first, **i32)
        s.back_table, s.back_first, back_total = table, first, total
    elif case["kind"] == "append":
        s.first = torch.tensor(before, **i32)
        s.back_table, back_total = _tables(before, after, False, seed, columns)
    else:
        s.q = _normal(g, (B, case["Hq"], D), 2.0, dt)  # scores of standard deviation 2
        s.Uk, s.Uv = (_normal(g, (Hkv, dd, D), dd ** -0.5, torch.float32) for _ in range(2))
        s.out = torch.empty_like(s.q)
    if case["kind"] in ("convert", "append"):  # pages of the storage type that are read back to
        if own:
            s.back = dar.DarCache(B, Hkv, dd, w, table.shape[1], back_total, dtype=dt, block_table=s.back_table)
        else:
            s.back = SimpleNamespace(pool_kd=torch.zeros((back_total, Hkv, PAGE, dd), dtype=dt, device="cuda"),
                                     block_table=s.back_table.cuda())
            s.back.pool_vd = torch.zeros_like(s.back.pool_kd)
    if own:
        if case["kind"] != "convert":
            dar.dar_cache_pack_q4(pages, c)
        if case["kind"] in ("decode", "step"):
            s.workspace = dar.decode_q4_workspace(c, case["Hq"])
    else:
        c.kd, c.vd = ((torch.zeros_like(kd, dtype=torch.int8), torch.zeros((*kd.shape[:3], _groups(dd)), device="cuda"))
                      for _ in range(2))
        if case["kind"] != "convert":
            c.kd, c.vd = _quantised(kd), _quantised(vd)
    return s


# ------------------------------------------------------------------ plain forms


def _groups(dd):
    return max(1, dd // 16)


def _quantised(x):
    """Codes [..., dd] (int8) and scales [..., groups] (fp32) of vectors x."""
    y = x.float().unflatten(-1, (_groups(x.shape[-1]), -1))
    a = y.abs().amax(-1, keepdim=True)
    bits = (a / 7).view(torch.int32)
    half = 0x3ffff + ((bits >> 19) & 1)  # nearest, ties to even, above 19 bits that go
    s = ((bits + half) & ~0x7ffff).view(torch.float32).clamp(max=1.125 * 2.0 ** 125)
    code = torch.round(y / s).clamp(-7, 7)
    code = torch.where(a > 0, code, 0.0).nan_to_num(nan=0.0)
    s = torch.where(torch.isfinite(a), s, math.nan)
    return code.flatten(-2).to(torch.int8), s[..., 0]


def _values(held):
    code, s = held
    return (code.unflatten(-1, (s.shape[-1], -1)).float() * s[..., None]).flatten(-2)


def _down(x, W):
    """Eq. 1 per KV head, one fused multiply-add in 32 bits after the other (the bits of a cached vector are defined by
    this order): a product of two 32-bit numbers is exact in 64, and the sum is rounded back to 32."""
    acc = torch.zeros((*x.shape[:-1], W.shape[-1]), dtype=torch.float64, device=x.device)
    for t in range(D):
        acc = acc.addcmul(x[..., t, None].double(), W[:, t, None].double()).float().double()
    return acc.to(x.dtype)


def _at(table, b, p):
    return table.long()[b, p // PAGE]


def _append(s):
    """Vectors of the tokens that leave the window into their pages; the ring and the lengths.  Returns where: the
    sequence and the position of each."""
    c, w = s.cache, s.case["w"]
    c.seq_lens.copy_(s.lens)
    L, n = s.lens.long(), s.n.long()
    first, last = (L - w).clamp(min=0), (L + n - w).clamp(min=0)
    b, i = (torch.arange(int(max(s.n_host)), device="cuda") < (last - first)[:, None]).nonzero(as_tuple=True)
    p = first[b] + i
    from_ring = (p < L[b])[:, None, None]
    for held, ring, new, W in ((c.kd, c.win_k, s.k_new, s.Dk), (c.vd, c.win_v, s.v_new, s.Dv)):
        x = torch.where(from_ring, ring[b, :, p % w], new[b, :, (p - L[b]).clamp(min=0)])
        code, scale = _quantised(_down(x[:, :, None], W)[:, :, 0])
        held[0][_at(c.block_table, b, p), :, p % PAGE] = code
        held[1][_at(c.block_table, b, p), :, p % PAGE] = scale
    c.win_k.copy_(_joined(c.win_k, s.k_new, L, n))
    c.win_v.copy_(_joined(c.win_v, s.v_new, L, n))
    c.seq_lens.add_(s.n)
    return b, p


def _read_back(s, b, p):
    for pool, held in ((s.back.pool_kd, s.cache.kd), (s.back.pool_vd, s.cache.vd)):
        x = _values([t[_at(s.cache.block_table, b, p), :, p % PAGE] for t in held])
        pool[_at(s.back.block_table, b, p), :, p % PAGE] = x.to(pool.dtype)


def _convert(s):
    c = s.cache
    last = (c.seq_lens.long() - s.case["w"]).clamp(min=0)
    pos = torch.arange(c.block_table.shape[1] * PAGE, device="cuda")
    b, p = ((pos >= s.first[:, None]) & (pos < last[:, None])).nonzero(as_tuple=True)
    page, row = _at(c.block_table, b, p), p % PAGE
    for held, pool in ((c.kd, s.pages.pool_kd), (c.vd, s.pages.pool_vd)):
        code, scale = _quantised(pool[page, :, row])
        held[0][page, :, row] = code
        held[1][page, :, row] = scale
    _read_back(s, b, p)


def _attend(s):
    """One decode step, all sequences at once, in 32 bits."""
    case, c = s.case, s.cache
    B, Hkv, w, dd = case["B"], case["Hkv"], case["w"], case["dd"]
    G, P = case["Hq"] // Hkv, c.block_table.shape[1]
    L = c.seq_lens.long()
    in_ring = (torch.arange(w, device="cuda") < L[:, None])[:, None, None]
    in_pages = (torch.arange(P * PAGE, device="cuda") < (L - w)[:, None])[:, None, None]
    pages = c.block_table.long().clamp(min=0)

    def paged(held):
        x = _values([t[pages] for t in held]).permute(0, 2, 1, 3, 4).reshape(B, Hkv, P * PAGE, dd)
        return x.masked_fill_(~in_pages[:, 0, 0, None, :, None], 0.0)

    q = s.q.float().view(B, Hkv, G, D)
    qt = q @ s.Uk.mT
    near = (q @ c.win_k.float().mT).masked_fill_(~in_ring, -math.inf)
    far = (qt @ paged(c.kd).mT).masked_fill_(~in_pages, -math.inf)
    scores = torch.cat((near, far), -1) * D ** -0.5
    m = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - torch.where(m > -math.inf, m, 0.0))
    p = p / p.sum(-1, keepdim=True).clamp(min=1e-30)  # an empty sequence gives zeros
    v = c.win_v.float().masked_fill(~in_ring[:, 0, 0, None, :, None], 0.0)
    out = p[..., :w] @ v + (p[..., w:] @ paged(c.vd)) @ s.Uv
    return out.reshape(B, case["Hq"], D).to(s.q.dtype)


def run(s):
    c, kind = s.cache, s.case["kind"]
    if own:
        from paper_2606_18587_gb300 import dar
        if kind in ("append", "step"):
            c.seq_lens.copy_(s.lens)
        if kind == "append":
            dar.dar_cache_append_q4(c, s.k_new, s.v_new, s.Dk, s.Dv, n_per_seq=s.n)
            dar.dar_cache_unpack_q4(c, s.back, first=s.first)
        elif kind == "convert":
            dar.dar_cache_pack_q4(s.pages, c, first=s.first)
            dar.dar_cache_unpack_q4(c, s.back, first=s.first)
        elif kind == "decode":
            return dar.dar_attn_decode_q4(c, s.q, s.Uk, s.Uv, s.workspace, out=s.out)
        else:
            dar.dar_decode_step_q4(c, s.k_new, s.v_new, s.Dk, s.Dv, s.q, s.Uk, s.Uv, s.workspace, out=s.out)
    elif kind == "append":
        _read_back(s, *_append(s))
    elif kind == "convert":
        _convert(s)
    elif kind == "decode":
        return _attend(s)
    else:
        _append(s)
        s.out = _attend(s)
    if kind == "step":
        return dict(out=s.out, win_k=c.win_k, win_v=c.win_v, seq_lens=c.seq_lens)
    read = dict(pool_kd=s.back.pool_kd, pool_vd=s.back.pool_vd)
    return read if kind == "convert" else dict(read, win_k=c.win_k, win_v=c.win_v, seq_lens=c.seq_lens)


# ------------------------------------------------------------- necessary work


def work(case):
    lens, joins = _layout(case)
    Hkv, w, dd, kind = case["Hkv"], case["w"], case["dd"], case["kind"]
    e = 4 if case["dtype"] == "f32" else 2
    row, vec = 2 * D * e, 2 * dd * e  # keys and values of a token at either width
    held = 2 * (dd // 2 + 2 * _groups(dd))  # the same in 4 bits, with scales of 16
    nbytes = flops = 0
    for L, n in zip(lens, joins):
        far = max(0, L - w)
        if kind == "convert":
            m = min(far, case["new"]) if case["new"] else far
            nbytes += Hkv * m * 2 * (vec + held)
            continue
        out = max(0, L + n - w) - far  # tokens that leave the window
        nbytes += Hkv * (out * (row + held) + min(n, w) * 2 * row)
        flops += Hkv * out * 4 * D * dd
        if kind == "append":
            nbytes += Hkv * out * (held + vec)
        else:
            near, far = min(L + n, w), far + out
            Hq = case["Hq"]
            nbytes += Hkv * (near * row + far * held) + 2 * Hq * D * e
            flops += Hq * (4 * near * D + 4 * far * dd + 4 * D * dd)
    if kind in ("append", "step"):
        nbytes += 2 * Hkv * D * dd * 4
    if kind in ("decode", "step"):
        nbytes += 2 * Hkv * D * dd * 4
    return dict(bytes=int(nbytes), flops=int(flops))


# ------------------------------------------------------------ the same in 64 bits


def _held_exactly(x):
    """What 4 bits make of vectors x (any type), as 64-bit numbers."""
    y = x.double().unflatten(-1, (_groups(x.shape[-1]), -1))
    top = y.abs().max(-1, keepdim=True).values
    mantissa, exponent = torch.frexp(top / 7)
    s = torch.ldexp(torch.round(mantissa * 32), exponent - 5).clamp(max=1.125 * 2.0 ** 125)
    code = torch.where(top > 0, torch.round(y / torch.where(top > 0, s, 1.0)), 0.0).clamp(-7, 7)
    return (code * s).flatten(-2)


def _exact_append(s):
    """One sequence after the other.  Returns the distant vectors of each as 64-bit numbers by position."""
    case, c, w = s.case, s.cache, s.case["w"]
    rings, far = [c.win_k.double(), c.win_v.double()], []
    for b, (L, n) in enumerate(zip(s.lens_host, s.n_host)):
        first, last = max(0, L - w), max(0, L + n - w)
        old = torch.arange(first, device="cuda")
        page = c.block_table[b].long()[old // PAGE]
        pair = []
        for ring, held, new, W in zip(rings, (c.kd, c.vd), (s.k_new, s.v_new), (s.Dk, s.Dv)):
            tail = torch.arange(first, L, device="cuda") % w
            x = torch.cat((ring[b][:, tail], new[b, :, :n].double()), 1)  # positions [first, L + n)
            vec = torch.einsum("gjt,gtc->gjc", x[:, :last - first], W.double()).to(new.dtype)
            was = _values([t[page, :, old % PAGE] for t in held]).double().transpose(0, 1)
            pair.append(torch.cat((was, _held_exactly(vec)), 1))
            stay = torch.arange(max(first, L + n - w), L + n, device="cuda")
            ring[b][:, stay % w] = x[:, stay - first]
        far.append(pair)
    return rings, far


def _exact_attend(s, rings, far, lens):
    """One sequence after the other: every key and value by position at full width, then softmax attention."""
    case = s.case
    Hq, Hkv, w = case["Hq"], case["Hkv"], case["w"]
    out = torch.zeros(s.q.shape, dtype=torch.float64, device="cuda")
    for b, L in enumerate(lens):
        if L == 0:
            continue
        near = torch.arange(max(0, L - w), L, device="cuda") % w
        k, v = (torch.cat((x @ U.double(), ring[b][:, near].double()), 1)
                for x, U, ring in zip(far[b], (s.Uk, s.Uv), rings))
        q = s.q[b].double().view(Hkv, Hq // Hkv, D)
        p = torch.softmax(torch.einsum("ghd,gjd->ghj", q, k) / math.sqrt(D), -1)
        out[b] = torch.einsum("ghj,gjd->ghd", p, v).reshape(Hq, D)
    return out


def exact(case, seed):
    s = _state(case, seed, False)  # codes and scales are looked at one by one
    c, kind = s.cache, case["kind"]
    if kind == "convert":
        back = [torch.zeros(s.back.pool_kd.shape, dtype=torch.float64, device="cuda") for _ in range(2)]
        for b, L in enumerate(s.lens_host):
            for x, pool in zip(back, (s.pages.pool_kd, s.pages.pool_vd)):
                at = torch.arange(s.back_first[b], max(s.back_first[b], L - case["w"]), device="cuda")
                page = c.block_table[b].long()[at // PAGE]
                x[page, :, at % PAGE] = _held_exactly(pool[page, :, at % PAGE])
        return dict(pool_kd=back[0], pool_vd=back[1])
    if kind == "decode":
        far = []
        for b, L in enumerate(s.lens_host):
            at = torch.arange(max(0, L - case["w"]), device="cuda")
            page = c.block_table[b].long()[at // PAGE]
            far.append([_values([t[page, :, at % PAGE] for t in held]).double().transpose(0, 1)
                        for held in (c.kd, c.vd)])
        return _exact_attend(s, (c.win_k, c.win_v), far, s.lens_host)
    rings, far = _exact_append(s)
    lens = [L + n for L, n in zip(s.lens_host, s.n_host)]
    rest = dict(win_k=rings[0], win_v=rings[1], seq_lens=torch.tensor(lens, dtype=torch.int32, device="cuda"))
    if kind == "step":
        return dict(out=_exact_attend(s, rings, far, lens), **rest)
    back = [torch.zeros(s.back.pool_kd.shape, dtype=torch.float64, device="cuda") for _ in range(2)]
    for b, L in enumerate(lens):
        at = torch.arange(max(0, s.lens_host[b] - case["w"]), max(0, L - case["w"]), device="cuda")
        page = s.back.block_table[b].long()[at // PAGE]
        for x, vec in zip(back, far[b]):
            x[page, :, at % PAGE] = vec[:, at].transpose(0, 1)
    return dict(pool_kd=back[0], pool_vd=back[1], **rest)
