"""Decode over 4-bit pages whose values are zero, in pages of every number of tokens: the weights' reference, which
follows weights times the scales of values, has nothing to go by there."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)

from paper_2606_18587_gb300 import dar  # noqa: E402
from tests.helpers import q4_ref as Q  # noqa: E402
from tests.helpers import serving_ref as R  # noqa: E402

W = 20
SHORT = [W + n for n in range(18)] + [W + 63, W + 64]


def decode(c4, q, Uk, Uv, **kw):
    return dar.dar_attn_decode_q4(c4, q, Uk, Uv, dar.decode_q4_workspace(c4, q.shape[1]), **kw)


def check(dtype, c, full, Hq, seed=4):
    c4 = Q.beside(dar, c)
    dar.dar_cache_pack_q4(c, c4)
    q, Uk, Uv = R.operands(seed, dtype, c.B, Hq, c.Hkv, c.d_down)
    got = decode(c4, q, Uk, Uv)
    assert c4.device_status() == 0
    Q.check_outputs(dtype, Q.read_back(dar, c4), full, q, Uk, Uv, got)


@pytest.mark.parametrize("dtype,dd", [("bf16", 8), ("bf16", 16), ("bf16", 32), ("bf16", 64), ("f32", 16)])
@pytest.mark.parametrize("G", [1, 2, 3, 8, 11])
@pytest.mark.parametrize("zero", ["all", "head", "group", "tiny"])
def test_first_page(dtype, dd, G, zero):
    """0 to 17 distant tokens, and about a page of them: zero values in all heads, in one, in the first group of 16
    entries, and values whose scales are no normal bf16 numbers."""
    c, full = R.filled_cache(dar, dd + G, dtype, 2, dd, W, SHORT)
    v = c.pool_vd
    if zero == "all":
        v.mul_(0.0)
    elif zero == "head":
        v[:, 1].mul_(0.0)
    elif zero == "group":
        v[..., :16].mul_(0.0)
    else:
        v.mul_(2.0 ** -130)
    v[torch.isnan(c.pool_kd)] = float("nan")  # rows behind the last token
    check(dtype, c, full, 2 * G)


@pytest.mark.parametrize("G", [1, 2, 4, 8])
@pytest.mark.parametrize("dd", [8, 16, 64])
def test_last_page(dd, G):
    """Contexts whose last page alone has zero values: with so many shares of work some begin at that page."""
    lens = [W + 64 * pages + n for pages in (1, 2, 3, 4, 5, 6) for n in (1, 2, 4, 7, 12, 13)]
    c, full = R.filled_cache(dar, dd + G, "bf16", 2, dd, W, lens)
    for b, L in enumerate(lens):
        page = full[b][-1]
        c.pool_vd[page, :, :(L - W) % 64] = 0.0
    check("bf16", c, full, 2 * G)


@pytest.mark.parametrize("G", [1, 2, 4, 8])
def test_zero_first_and_values_later(G):
    """A reference set by zero values is raised by the first that are not."""
    lens = [W + n for n in (64 + 5, 128 + 60, 700, 1500)]
    c, full = R.filled_cache(dar, G, "bf16", 2, 16, W, lens)
    for b in range(len(lens)):
        c.pool_vd[full[b][0]] = 0.0
    check("bf16", c, full, 2 * G)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq", [2, 8, 16])
def test_steps_on_zeros(dtype, Hq):
    """Steps before there are data: everything is zero, and so is what comes out; rings that are not keep their average."""
    B, Hkv, dd = 3, 2, 16
    c = dar.DarCacheQ4(B, Hkv, dd, W, 4, dtype=R.DT[dtype])
    zero = torch.zeros((B, Hkv, 1, 64), dtype=R.DT[dtype], device="cuda")
    q, Uk, Uv = R.operands(1, dtype, B, Hq, Hkv, dd)
    Dk, Dv = (torch.ones((Hkv, 64, dd), device="cuda") for _ in range(2))
    ws = dar.decode_q4_workspace(c, Hq)
    for i in range(W + 20):
        out = dar.dar_decode_step_q4(c, zero, zero, Dk, Dv, q if i % 2 else q * 0, Uk, Uv, ws)
        assert torch.equal(out, torch.zeros_like(out)), i
    one = torch.ones_like(zero)
    for i in range(5):
        out = dar.dar_decode_step_q4(c, zero, one, Dk, Dv, q * 0, Uk, Uv, ws)
        want = (i + 1) / (W + 21 + i)
        assert (out.double() - want).abs().max() <= want * (2.0 ** -18 + torch.finfo(R.DT[dtype]).eps / 2), i
    assert c.device_status() == 0
