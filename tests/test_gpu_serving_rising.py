"""Scores that rise along a shared prefix by more than a weight may grow, with values near the top of what bf16 holds:
the attention is finite, and so are the sums it is made of."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)

from paper_2606_18587_gb300 import dar  # noqa: E402
from tests.helpers import serving_ref as R  # noqa: E402

B, HQ, HKV, W, PAGES = 16, 8, 2, 40, 24  # 64 rows a KV head: every warp takes all keys of a stage


def rising(dd, rise, value, device="cuda", cache_of=dar):
    """A cache whose prefix has, for every row, scores of 0 (log2) in the first step of each stage and of `rise` in the
    others, and positive distant values of the size of `value`."""
    lens = [64 * PAGES + W + 3 + 5 * i for i in range(B)]
    c, full = R.filled_cache(cache_of, 3, "bf16", HKV, dd, W, lens, [0] * B, [PAGES], values=0.01, device=device)
    _, Uk, Uv = R.operands(4, "bf16", B, HQ, HKV, dd, device=device)
    g = torch.Generator().manual_seed(7)
    q = torch.randn((1, HKV, 1, 64), generator=g).expand(B, HKV, HQ // HKV, 64)  # the same for all rows of a KV head
    q = q.reshape(B, HQ, 64).bfloat16().to(device)
    qt = torch.einsum("hd,hed->he", q[0, ::HQ // HKV].double().cpu(), Uk.double().cpu())
    unit = qt / qt.pow(2).sum(-1, keepdim=True)  # a key with qt . key = 1
    stage, step = 4096 // dd, {8: 64, 16: 64, 32: 32, 64: 16}[dd]  # tokens
    for i, pg in enumerate(full[0][:PAGES]):
        at = (64 * i + torch.arange(64)) % stage
        high = torch.where(at < step, 0.0, rise * 0.6931471805599453 * 8.0)  # / (log2(e) / sqrt(64))
        key = high[None, :, None] * unit[:, None, :]
        c.pool_kd[pg] = (c.pool_kd[pg].cpu().double() * 0.01 + key).bfloat16().to(device)
    c.pool_vd.abs_().mul_(100.0 * value)  # filled_cache's are 0.01 in size; one sign, so that sums are as large as they get
    return c, full, q, Uk, Uv.abs()


@pytest.mark.parametrize("dd", [8, 16, 32, 64])
@pytest.mark.parametrize("rise", [12.0, 40.0, 58.0, 200.0])
@pytest.mark.parametrize("value", [1.0, 2.0 ** 100])
def test_values_of_any_size(dd, rise, value):
    c, full, q, Uk, Uv = rising(dd, rise, value)
    group, pages = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0] * B, [PAGES]))
    got = dar.dar_attn_decode_shared(c, q, Uk, Uv, group, pages, dar.shared_decode_workspace(c, HQ))
    torch.cuda.synchronize()
    assert c.device_status() == 0 and torch.isfinite(got).all()
    for b in (0, 7, 15):
        out, _, mag, top = R.attend(q[b].cpu().double(), *R.contents(c, full, b), Uk.cpu().double(), Uv.cpu().double())
        assert ((got[b].cpu().double() - out).abs() <= R.tolerances("bf16", out, mag, top)).all(), b
