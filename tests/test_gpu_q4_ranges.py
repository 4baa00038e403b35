"""Decode over 4-bit pages where sizes lie far apart: groups of a vector, queries and keys."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)

from paper_2606_18587_gb300 import dar  # noqa: E402
from tests.helpers import q4_ref as Q  # noqa: E402
from tests.helpers import serving_ref as R  # noqa: E402


def decode(c4, q, Uk, Uv, **kw):
    return dar.dar_attn_decode_q4(c4, q, Uk, Uv, dar.decode_q4_workspace(c4, q.shape[1]), **kw)


@pytest.mark.parametrize("Hq", [2, 4, 16])
@pytest.mark.parametrize("dtype,dd", [("bf16", 32), ("bf16", 64), ("f32", 64)])
@pytest.mark.parametrize("step", [8, 16, 24])
def test_groups_far_apart(dtype, dd, Hq, step):
    """Values of each group of 16 entries 2^-step of the group's before, lifted by as much more to outputs of their own.

    bf16: a weight times a group's scale is off by 2^-11 of it (as in q4_ref.tolerances), or by half a step of the
    smallest fp16 numbers, 2^-25 where the row's largest such product is 2^8 at least: 2^-33 of that one.  Such an error
    of each of n tokens times a code of 7 at most goes into a sum that Uv lifts."""
    lens, w = [300, 41, 700], 40
    c, full = R.filled_cache(dar, 3, dtype, 2, dd, w, lens)
    groups = dd // 16
    size = 2.0 ** (-step * torch.arange(groups, device="cuda").float()).repeat_interleave(16)
    c.pool_vd.mul_(size)
    c4 = Q.beside(dar, c)
    dar.dar_cache_pack_q4(c, c4)
    q, Uk, Uv = R.operands(4, dtype, 3, Hq, 2, dd)
    own = torch.arange(dd, device="cuda")[:, None] // 16 == torch.arange(64, device="cuda") * groups // 64
    Uv = (Uv * own / size[:, None]).contiguous()
    got = decode(c4, q, Uk, Uv)
    back = Q.read_back(dar, c4)
    for b in range(3):
        kd, vd, k, v = R.contents(back, full, b)
        out, p, mag, top = R.attend(q[b].cpu().double(), kd, vd, k, v, Uk.cpu().double(), Uv.cpu().double())
        n = kd.shape[1]
        tol = Q.tolerances(dtype, out, mag, top)
        if dtype == "bf16":
            for h in range(Hq):
                g = h // (Hq // 2)
                scales = vd[g].unflatten(-1, (groups, 16)).abs().amax(-1) / 7  # the largest entry's code is 7
                largest = (p[h, :n, None] * scales).max()
                tol[h] += n * 7 * 2.0 ** -33 * largest * Uv[g].cpu().double().abs().sum(0)
        err = (got[b].cpu().double() - out).abs()
        assert (err <= tol).all(), (b, float((err / tol).max()))


@pytest.mark.parametrize("Hq", [2, 4, 16])
@pytest.mark.parametrize("dtype,dd", [("bf16", 8), ("bf16", 16), ("bf16", 64), ("f32", 16)])
@pytest.mark.parametrize("size,scale,best", [
    (1e30, 0.125, None), (1e36, 0.125, None), (1e30, 1e7, None), (1e3, 1e34, None),
    (1e5, 0.125, 5), (1e-5, 1e9, 5), (3e4, 0.4, 5),
])
def test_large_queries(dtype, dd, Hq, size, scale, best):
    """Queries times scale up to 2^125: keys of zero have equal weights.  Scores of up to 2^25: the one token whose score
    is positive, the others' being its negative, has all of the weight."""
    w, lens = 20, [300, 33, 84]
    c, full = R.filled_cache(dar, 3, dtype, 2, dd, w, lens)
    q, Uk, Uv = R.operands(4, dtype, 3, Hq, 2, dd)
    q = q.abs().clamp(0.25, 2.0).mul(size).contiguous()
    Uk = Uk.abs() + 0.1
    key = 0.0 if best is None else -1.0
    c.pool_kd.copy_(torch.where(c.pool_kd.isnan(), c.pool_kd, key))
    c.win_k.copy_(torch.where(c.win_k.isnan(), c.win_k, key))
    if best is not None:
        for b in range(3):
            c.pool_kd[full[b][0], :, best] = 1.0
    c4 = Q.beside(dar, c)
    dar.dar_cache_pack_q4(c, c4)
    back = Q.read_back(dar, c4)
    got = decode(c4, q, Uk, Uv, scale=scale)
    for b in range(3):
        out, _, mag, top = R.attend(q[b].cpu().double(), *R.contents(back, full, b), Uk.cpu().double(),
                                    Uv.cpu().double(), scale)
        assert top < 2.0 ** 25
        # equal scores are exactly equal, and the others are so far apart that errors of theirs change no weight
        tol = Q.tolerances(dtype, out, mag, 0.0)
        err = (got[b].cpu().double() - out).abs()
        assert (err <= tol).all(), (b, float((err / tol).max()))
