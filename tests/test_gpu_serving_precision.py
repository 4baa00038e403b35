"""The shared and the scored decode step lose nothing that dar_attn_decode keeps: where that holds the weights of
distant tokens and the absorbed query in 32 bits (an odd number of query heads per KV head at d_down 16, any at d_down
8), and in every scored step, a bf16 output is the exact value rounded once, but for what 32-bit arithmetic leaves."""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)

from paper_2606_18587_gb300 import dar  # noqa: E402
from tests.helpers import serving_ref as R  # noqa: E402


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def rounded_once(x, err):
    """How far a bf16 number may be off x if it is x, off by err, rounded to the nearest: err and half the spacing of
    bf16 (2^-7 of the binade) where |x| + err lies."""
    return err + 2.0 ** (torch.floor(torch.log2(x.abs() + err + 1e-30)) - 8)


def check(c, full, q, Uk, Uv, got):
    """Each element: weights as two bf16 terms, 2^-15 and 2^-22 of sum p |v|; q~ as three and chains of fp32
    multiply-adds, 150 * 2^-24 of the absolute products; exp2 and the sums, 2^-18.

    Their mean square: values are independent and of mean zero here, so errors e_j of the weights leave e of the output's
    mean square, sum p_j^2 v_j^2 e_j^2 against sum p_j^2 v_j^2.  The output's own rounding is 2^-9.2 of it (uniform over a
    step).  A weight's terms leave 2^-15 / sqrt(12); its score, sqrt(150) roundings of 2^-25 of at most 128 (the largest
    `top` here), twice: 2^-13.4 in all, (2^-4.2)^2 = 0.003 of the rounding's square, and 1.03 covers its root.  Weights
    of 8 bits leave 2^-9.8: 1.1 to 1.4, the less the more weight one token has."""
    near = far = 0.0
    for b in range(c.B):
        out, _, mag, top = R.attend(q[b].cpu().double(), *R.contents(c, full, b), Uk.cpu().double(), Uv.cpu().double())
        err = mag * (math.expm1(2 * top * 150 * 2.0 ** -24) + 2.0 ** -18 + 2.0 ** -15 + 2.0 ** -22)
        off = (got[b].cpu().double() - out).abs()
        assert (off <= rounded_once(out, err)).all(), (b, float((off / rounded_once(out, err)).max()))
        assert top <= 128.0
        near += float((out.to(got.dtype).double() - out).pow(2).sum())
        far += float(off.pow(2).sum())
    assert far <= 1.03 ** 2 * near, (far / near) ** 0.5


@pytest.mark.parametrize("Hq,Hkv,dd,w", [
    (4, 4, 16, 40),    # multi-head
    (6, 2, 16, 40),    # three query heads a KV head
    (9, 1, 16, 17),    # more rows than eight
    (42, 2, 16, 300),
    (4, 4, 8, 40),
    (8, 2, 8, 300),
    (16, 1, 8, 17),
])
def test_shared(Hq, Hkv, dd, w):
    lens, group, pages = [1000 + w + 77 * i for i in range(6)], [0, 0, 0, 0, 0, -1], [15]
    c, full = R.filled_cache(dar, dd + w, "bf16", Hkv, dd, w, lens, group, pages)
    q, Uk, Uv = R.operands(dd + Hq, "bf16", 6, Hq, Hkv, dd, q_std=2.0)
    got = dar.dar_attn_decode_shared(c, q, Uk, Uv, ints(group), ints(pages), dar.shared_decode_workspace(c, Hq))
    torch.cuda.synchronize()
    check(c, full, q, Uk, Uv, got)


@pytest.mark.parametrize("Hq,Hkv,dd,w", [(4, 4, 16, 40), (8, 2, 16, 300), (32, 2, 16, 40), (8, 2, 8, 40), (16, 1, 8, 40),
                                         (6, 2, 32, 300), (12, 1, 32, 40), (4, 4, 64, 40), (24, 2, 64, 300)])
def test_scored(Hq, Hkv, dd, w):
    lens = [1000 + 77 * i for i in range(4)]
    c, full = R.filled_cache(dar, dd + w, "bf16", Hkv, dd, w, lens)
    q, Uk, Uv = R.operands(dd + Hq, "bf16", 4, Hq, Hkv, dd, q_std=2.0)
    got = dar.dar_attn_decode_scored(c, q, Uk, Uv, dar.attention_weights(c), dar.scored_decode_workspace(c, Hq))
    torch.cuda.synchronize()
    check(c, full, q, Uk, Uv, got)


@pytest.mark.parametrize("Hq,Hkv,dd", [(4, 4, 16), (9, 1, 16), (8, 2, 8), (16, 1, 8), (8, 2, 32), (24, 2, 64)])
def test_infinite_values_keep_their_sign(Hq, Hkv, dd):
    """One infinite entry of a ring value makes its column infinite and no other; one of a distant value makes every
    column infinite with the sign of its lift.  (The weights there are positive: scores are small.)"""
    lens, group, pages = [700, 720, 740], [0, 0, 0], [9]
    c, full = R.filled_cache(dar, 5, "bf16", Hkv, dd, 40, lens, group, pages)
    q, Uk, Uv = R.operands(6, "bf16", 3, Hq, Hkv, dd, q_std=0.25)
    c.win_v[0, :, 3, 5] = float("inf")
    c.win_v[0, :, 7, 9] = -float("inf")
    c.pool_vd[full[1][9], :, 2, 1] = float("inf")  # a page of its own
    weights = dar.attention_weights(c)
    for got in (dar.dar_attn_decode_shared(c, q, Uk, Uv, ints(group), ints(pages), dar.shared_decode_workspace(c, Hq)),
                None):
        if got is None:  # the scored step reads each sequence's own table
            for b in (1, 2):
                c.block_table[b, :9] = c.block_table[0, :9]
            got = dar.dar_attn_decode_scored(c, q, Uk, Uv, weights, dar.scored_decode_workspace(c, Hq))
        got = got.float().cpu()
        want = torch.zeros(64)
        want[5], want[9] = math.inf, -math.inf
        finite = torch.ones(64, dtype=torch.bool)
        finite[[5, 9]] = False
        assert torch.isfinite(got[0][:, finite]).all() and (got[0][:, ~finite] == want[~finite]).all()
        lift = torch.sign(Uv[:, 1].cpu()).repeat_interleave(Hq // Hkv, 0)
        assert (got[1] == lift * math.inf).all()
        assert torch.isfinite(got[2]).all()
