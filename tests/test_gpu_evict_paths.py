"""dar_cache_evict on each of its ways: clusters of 1, 2, 4 and 8 with many heads, bits in shared memory and in the
workspace, rings that turn through shared memory and by reflections.  The launch rule is restated here, and every case
asserts the way that it takes."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)

from paper_2606_18587_gb300 import dar  # noqa: E402
from tests.helpers import serving_ref as R  # noqa: E402


def ways(dtype, B, Hkv, w, maxp, lens, keep, protect):
    """(blocks of a cluster, {where the bits of a sequence that evicts are}, {how its ring turns})."""
    C = 8
    while C > 1 and (B * Hkv * C > 4 * 152 or maxp * 64 < 1024 * C):
        C //= 2
    bits, rings = set(), set()
    for L, k, p in zip(lens, keep, protect):
        n = max(0, L - w)
        if n <= k:
            continue
        if k > p:
            bits.add("workspace" if -(-(n - p) // C) > 256 * 128 else "shared")
        if (n - k) % w:
            pieces = -(-w // C) * 2 * 64 * (2 if dtype == "bf16" else 4) // 16
            rings.add("staged" if pieces <= 2048 else "reflected")
    return C, bits, rings


def totals(kind, shape, seed):
    g = torch.Generator().manual_seed(seed)
    if kind == "spread":
        return torch.exp(2 * torch.randn(shape, generator=g))
    if kind == "few":
        return torch.randint(0, 4, shape, generator=g).float()
    if kind == "equal":
        return torch.full(shape, 0.25)
    u = torch.rand(shape, generator=g)  # "odd": NaN, infinities, negatives
    t = torch.where(u < 0.2, float("nan"), torch.where(u < 0.3, float("inf"), torch.randn(shape, generator=g)))
    return torch.where(u > 0.9, -float("inf"), t)


def places(t, n, keep, protect):
    """Positions (to, at) of the moves: the definition, with a sort by weight, NaN last, and then position."""
    v = t[protect:n].astype(np.float64)
    nan = np.isnan(v)
    order = np.lexsort((np.arange(len(v)), nan, -np.where(nan, -np.inf, v)))
    stays = np.zeros(n, dtype=bool)
    stays[:protect] = True
    stays[protect + order[:keep - protect]] = True
    return np.flatnonzero(~stays[:keep]), keep + np.flatnonzero(stays[keep:])


FAR = [0] * 38
CASES = [
    # dtype, Hkv, dd, w, lens, keep of all, protect of all, totals, (C, bits, rings)
    ("bf16", 1, 8, 16, [270011], 130000, 1000, "spread", (8, "workspace", "staged")),
    ("bf16", 1, 8, 16, [270012], 130000, 1000, "equal", (8, "workspace", "staged")),
    ("bf16", 1, 8, 16, [270013], 200000, 3, "odd", (8, "workspace", "staged")),
    ("bf16", 8, 8, 16, FAR + [40000], 17000, 13, "spread", (1, "workspace", "staged")),
    ("bf16", 8, 8, 16, FAR + [40000], 39000, 0, "few", (1, "workspace", "staged")),
    ("bf16", 2, 8, 16, [32769 + 16 + 512] + [5] * 155, 512, 512, "spread", (1, None, "staged")),  # all that stays is protected
    ("bf16", 16, 16, 20, [4200 + 131 * i for i in range(6)], 2100, 64, "spread", (4, "shared", "staged")),
    ("bf16", 16, 16, 20, [4200 + 131 * i for i in range(6)], 300, 64, "few", (4, "shared", "staged")),
    ("bf16", 16, 16, 20, [2200 + 11 * i for i in range(16)], 1000, 3, "spread", (2, "shared", "staged")),
    ("bf16", 16, 16, 20, [2200 + 11 * i for i in range(16)], 2000, 3, "odd", (2, "shared", "staged")),
    ("bf16", 16, 16, 20, [8300 + 111 * i for i in range(4)], 5000, 7, "spread", (8, "shared", "staged")),
    ("f32", 16, 8, 20, [8300 + 111 * i for i in range(4)], 700, 7, "equal", (8, "shared", "staged")),
    ("bf16", 2, 16, 256, [3000, 2700], 999, 10, "spread", (2, "shared", "staged")),
    ("f32", 2, 8, 128, [3000, 2700], 999, 10, "spread", (2, "shared", "staged")),
    ("bf16", 2, 16, 600, [6000, 5500], 999, 10, "spread", (4, "shared", "reflected")),
    ("bf16", 2, 16, 1100, [9900, 9500], 999, 10, "spread", (8, "shared", "reflected")),
    ("f32", 1, 8, 601, [9900, 9500], 8001, 10, "few", (8, "shared", "reflected")),
    ("bf16", 8, 8, 129, [400] * 40, 100, 10, "spread", (1, "shared", "reflected")),
]


@pytest.mark.parametrize("dtype,Hkv,dd,w,lens,keep,protect,kind,way", CASES)
def test_evict(dtype, Hkv, dd, w, lens, keep, protect, kind, way):
    B = len(lens)
    c, full = R.filled_cache(dar, 7 * B + dd, dtype, Hkv, dd, w, lens)
    C, bits, rings = ways(dtype, B, Hkv, w, c.max_pages_per_seq, lens, [keep] * B, [protect] * B)
    assert (C, bits, rings) == (way[0], {way[1]} - {None}, {way[2]})
    t = totals(kind, (B, Hkv, c.max_pages_per_seq * 64 + w), 5)
    weights = t.cuda()
    want = [x.cpu().clone() for x in (c.pool_kd, c.pool_vd, c.win_k, c.win_v, c.seq_lens)]
    want_w = t.clone()
    k, p = (torch.full((B,), x, dtype=torch.int32, device="cuda") for x in (keep, protect))
    dar.dar_cache_evict(c, weights, k, dar.evict_workspace(c), protect=p)
    torch.cuda.synchronize()
    assert c.device_status() == 0
    for b, L in enumerate(lens):
        n = max(0, L - w)
        if n <= keep:
            continue
        want[4][b] = keep + w
        ids = np.array(full[b])
        for g in range(Hkv):
            to, at = places(t[b, g].numpy(), n, keep, protect)
            assert len(to) == len(at)
            for pool in want[:2]:
                pool[ids[to // 64], g, to % 64] = pool[ids[at // 64], g, at % 64]
            want_w[b, g, to] = t[b, g, at]
            want_w[b, g, keep:keep + w] = t[b, g, n:n + w]
            want_w[b, g, keep + w:L] = 0.0
        for ring in want[2:4]:
            ring[b] = ring[b].roll(-((n - keep) % w), 1)
    for name, got, x in zip(("pool_kd", "pool_vd", "win_k", "win_v", "seq_lens"),
                            (c.pool_kd, c.pool_vd, c.win_k, c.win_v, c.seq_lens), want):
        got = got.cpu()
        assert torch.equal(got.nan_to_num(-77.0), x.nan_to_num(-77.0)) if got.is_floating_point() \
            else torch.equal(got, x), name
    assert torch.equal(weights.cpu().nan_to_num(-77.0), want_w.nan_to_num(-77.0))
