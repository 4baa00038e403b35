"""The steady state of the shared and the scored step in bf16: calls in which a thread block takes its four slots round
several times, a cut reads more than 32 entries of a block table, and what a row has summed is carried from stage to
stage.  Each test asserts that its call is of that kind."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)

from paper_2606_18587_gb300 import dar  # noqa: E402
from tests.helpers import segments_line  # noqa: E402
from tests.helpers import serving_ref as R  # noqa: E402


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


SHARED = [
    # Hq, Hkv, dd, w, pages of the two groups, pages of the others
    (32, 8, 8, 40, (1400, 900), 800),
    (32, 8, 16, 40, (700, 500), 400),
    (32, 8, 32, 40, (700, 500), 300),
    (32, 8, 64, 40, (700, 500), 300),
    (12, 12, 16, 128, (1500, 900), 400),   # one query head a KV head
    (24, 2, 16, 300, (1600, 900), 900),    # more rows than eight a private unit
]


def shared_case(Hq, Hkv, dd, w, pages, alone):
    """64 sequences of 2048 rows in all (32 query heads), in two groups and eight on their own, in no order."""
    group = [-1 if b % 8 == 3 else int(b % 3 == 0) for b in range(64)]
    lens = [w + 64 * (pages[g] if g >= 0 else alone) + (b * 37) % 190 for b, g in enumerate(group)]
    return lens, group


def check(c, full, q, Uk, Uv, got, sample):
    for b in sample:
        out, p, mag, top = R.attend(q[b].cpu().double(), *R.contents(c, full, b), Uk.cpu().double(), Uv.cpu().double())
        err, tol = (got[b].cpu().double() - out).abs(), R.tolerances("bf16", out, mag, top)
        assert (err <= tol).all(), (b, float((err / tol).max()))
        yield b, p, top


@pytest.mark.parametrize("growth", [0.0, 0.02])
@pytest.mark.parametrize("Hq,Hkv,dd,w,pages,alone", SHARED)
def test_shared(Hq, Hkv, dd, w, pages, alone, growth):
    """growth: keys of the prefix grow by page, so that a row's reference is raised in many stages of a cut."""
    lens, group = shared_case(Hq, Hkv, dd, w, pages, alone)
    cuts = segments_line.cuts(Hq, Hkv, dd, w, lens, group, pages)
    for kind in ("prefix", "private"):
        assert max(p for k, _, _, p, _ in cuts if k == kind) >= 10, kind
        assert max(s for k, _, _, _, s in cuts if k == kind) > 33, kind
    c, full = R.filled_cache(dar, dd, "bf16", Hkv, dd, w, lens, group, list(pages))
    q, Uk, Uv = R.operands(dd, "bf16", 64, Hq, Hkv, dd)
    leaders = [group.index(0), group.index(1)]
    if growth:
        for g in (0, 1):
            scale = 1.0 + growth * torch.arange(pages[g], device="cuda", dtype=torch.float32)
            ids = torch.tensor(full[leaders[g]][:pages[g]], device="cuda")
            c.pool_kd[ids] = (c.pool_kd[ids].float() * scale[:, None, None, None]).bfloat16()
    got = dar.dar_attn_decode_shared(c, q, Uk, Uv, ints(group), ints(pages), dar.shared_decode_workspace(c, Hq))
    torch.cuda.synchronize()
    assert c.device_status() == 0
    list(check(c, full, q, Uk, Uv, got, [leaders[0], leaders[1], 3, 38, 63]))


SCORED = [
    # Hq, Hkv, dd, w, tokens of 16 sequences
    (32, 8, 8, 40, 22000),
    (32, 8, 16, 40, 12000),
    (32, 8, 32, 40, 12000),
    (32, 8, 64, 40, 12000),
    (12, 12, 16, 128, 9000),
    (24, 2, 16, 300, 45000),
    (32, 2, 8, 300, 80000),
]


@pytest.mark.parametrize("Hq,Hkv,dd,w,tokens", SCORED)
def test_scored(Hq, Hkv, dd, w, tokens):
    lens = [tokens + 301 * i - 2000 for i in range(16)]
    lens[5] = 1
    cuts = segments_line.cuts(Hq, Hkv, dd, w, lens)
    assert max(p for _, _, _, p, _ in cuts) >= 10 and max(s for *_, s in cuts) > 33
    assert sorted(p + r for _, _, r, p, _ in cuts)[len(cuts) // 2] > 4  # most blocks reuse slots
    c, full = R.filled_cache(dar, dd, "bf16", Hkv, dd, w, lens)
    q, Uk, Uv = R.operands(dd, "bf16", 16, Hq, Hkv, dd, q_std=2.0)
    weights = dar.attention_weights(c)
    got = dar.dar_attn_decode_scored(c, q, Uk, Uv, weights, dar.scored_decode_workspace(c, Hq))
    torch.cuda.synchronize()
    assert c.device_status() == 0
    for b, p, top in check(c, full, q, Uk, Uv, got, [0, 5, 8, 15]):
        p = p.view(Hkv, Hq // Hkv, -1).sum(1)
        new = weights[b].cpu().double()
        err, tol = (new[:, :lens[b]] - p).abs(), R.weight_tolerance(p, torch.zeros_like(p), top)
        assert (err <= tol).all(), (b, float((err / tol).max()))
        assert not new[:, lens[b]:].any()
