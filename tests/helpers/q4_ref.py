"""What a page in 4 bits holds, from its definition, and caches of such pages."""
import math

import torch

from tests.helpers import serving_ref as R


def held(x):
    """The values that 4 bits make of vectors x [..., dd] (fp32 or bf16), in 64 bits: groups of 16 entries (8 of 8),
    s = max |x| / 7 at 5 significant bits, x / s to the nearest whole number."""
    dd = x.shape[-1]
    y = x.double().unflatten(-1, (max(1, dd // 16), -1))
    a = y.abs().amax(-1, keepdim=True)
    # the quotient is rounded to 32 bits first: below 2^-126 that decides
    mantissa, exponent = torch.frexp((a.float() / 7).double())
    # 5 significant bits, or whole multiples of 2^-130 below the normal range
    unit = torch.maximum(torch.ldexp(torch.ones_like(a), exponent - 5), torch.tensor(2.0 ** -130, dtype=torch.float64))
    s = torch.where(torch.isfinite(a), (torch.round(mantissa * torch.ldexp(torch.ones_like(a), exponent) / unit) * unit)
                    .clamp(max=1.125 * 2.0 ** 125), math.nan)
    code = torch.where(s > 0, torch.round(y / torch.where(s > 0, s, 1.0)), 0.0).clamp(-7, 7)
    return (code * s).flatten(-2)


def beside(dar, c, seed=0):
    """A cache in 4 bits beside c whose pages hold arbitrary bytes."""
    c4 = dar.DarCacheQ4.beside(c)
    g = torch.Generator().manual_seed(seed)
    c4.pool.copy_(torch.randint(0, 256, c4.pool.shape, dtype=torch.uint8, generator=g))
    return c4


def read_back(dar, c4, device="cuda"):
    """A DarCache with c4's ring, lengths and table whose pages hold what c4's distant tokens stand for (NaN elsewhere)."""
    c = dar.DarCache(c4.B, c4.Hkv, c4.d_down, c4.w, c4.max_pages_per_seq, c4.num_pages, dtype=c4.dtype,
                     block_table=c4.block_table.cpu(), device=device)
    c.pool_kd.fill_(math.nan)
    c.pool_vd.fill_(math.nan)
    c.win_k.copy_(c4.win_k)
    c.win_v.copy_(c4.win_v)
    c.seq_lens.copy_(c4.seq_lens)
    dar.dar_cache_unpack_q4(c4, c)
    return c


def tolerances(dtype, out, mag, top):
    """How far an output may be off, element by element (see serving_ref.tolerances for mag and top).

    Scores: chains of at most 64 + 64 fp32 multiply-adds, q~ split into terms of 16 bits at least, and a few more
    roundings, each relative 2^-24 (2^-16) of the absolute products' sum `top`.  An error d of a score changes its
    weight by the factor e^d, numerator and sum alike: 2 d.  Weights as operands of 16 bits with an 11-bit
    significand: half a step, 2^-11, of sum p |v|.  exp2 and the sums: 2^-18 of it.  The output's own rounding: half a
    step."""
    bf = dtype == "bf16"
    d = top * (140 * 2.0 ** -24 + (2.0 ** -16 if bf else 0.0))
    return mag * (math.expm1(2 * d) + 2.0 ** -18 + (2.0 ** -11 if bf else 0.0)) \
        + out.abs() * torch.finfo(R.DT[dtype]).eps / 2 + 1e-40


def check_outputs(dtype, cache, full, q, Uk, Uv, got, scale=R.D ** -0.5):
    """got [B][Hq][64] against softmax attention over the keys and values that `cache` (a DarCache) holds."""
    worst = 0.0
    for b in range(cache.B):
        kd, vd, k, v = R.contents(cache, full, b)
        if kd.shape[1] + k.shape[1] == 0:
            assert not got[b].any()
            continue
        out, _, mag, top = R.attend(q[b].cpu().double(), kd, vd, k, v, Uk.cpu().double(), Uv.cpu().double(), scale)
        err, tol = (got[b].cpu().double() - out).abs(), tolerances(dtype, out, mag, top)
        assert not torch.isnan(err).any(), b
        worst = max(worst, float((err / tol).max()))
        assert (err <= tol).all(), (b, worst)
    return worst
