"""dar_cache_evict against its definition, head by head: which tokens stay, where they move, bit for bit."""
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


def totals(kind, c, lens, seed):
    g = torch.Generator().manual_seed(seed)
    t = torch.exp(2 * torch.randn((c.B, c.Hkv, c.max_pages_per_seq * 64 + c.w), generator=g))
    if kind == "few":      # few distinct values, zeros of both signs among them
        t = torch.randint(-1, 3, t.shape, generator=g).float()
        t[t == 0] *= torch.where(torch.rand(t.shape, generator=g)[t == 0] < 0.5, -1.0, 1.0)
    elif kind == "equal":
        t = torch.full_like(t, 0.25)
    elif kind == "odd":    # NaN, infinities, negatives and the smallest numbers
        u = torch.rand(t.shape, generator=g)
        t = torch.where(u < 0.2, float("nan"), torch.where(u < 0.3, math.inf, torch.where(u < 0.4, -math.inf, t)))
        t = torch.where((u > 0.4) & (u < 0.6), -t, torch.where(u > 0.9, 1e-42, t))
    return t


def state(c):
    return [t.cpu().clone() for t in (c.pool_kd, c.pool_vd, c.win_k, c.win_v, c.seq_lens)]


def same(a, b):
    return torch.equal(a.nan_to_num(-77.0), b.nan_to_num(-77.0)) if a.is_floating_point() else torch.equal(a, b)


CASES = [
    # dtype, Hkv, dd, w, lens, keep, protect, totals
    ("bf16", 2, 16, 8, [200, 72, 8, 0, 73], [100, 64, 0, 0, 64], None, "spread"),
    ("bf16", 2, 16, 8, [200, 201, 202], [0, 1, 2], None, "spread"),                   # almost nothing stays
    ("bf16", 3, 16, 33, [1000, 1001, 500], [966, 967, 466], [4, 0, 466], "spread"),   # one or two go
    ("bf16", 1, 16, 128, [5000], [2500], [100], "spread"),
    ("bf16", 2, 16, 128, [3000, 4000], [128, 4096], None, "few"),
    ("bf16", 2, 16, 100, [3000, 2000], [999, 1000], [10, 1000], "equal"),
    ("bf16", 2, 16, 100, [3000, 2000], [999, 1000], [10, 3], "odd"),
    ("bf16", 2, 8, 5, [700, 800, 705, 710], [600, 700, 695, 695], [64, 0, 1, 2], "spread"),
    ("bf16", 2, 32, 1, [700, 800], [600, 1], [0, 1], "few"),
    ("bf16", 2, 64, 64, [700, 800], [64, 128], [0, 64], "spread"),
    ("f32", 2, 8, 50, [700, 800], [300, 700], [0, 64], "spread"),
    ("f32", 2, 16, 50, [700, 800], [300, 700], [0, 64], "few"),
    ("f32", 2, 64, 50, [700, 800], [300, 700], None, "odd"),
    ("bf16", 16, 16, 20, [600 + 31 * i for i in range(6)], [300] * 6, [64] * 6, "spread"),     # clusters of 4
    ("bf16", 16, 16, 20, [400 + 11 * i for i in range(16)], [100] * 16, [3] * 16, "few"),      # of 2
    ("bf16", 16, 8, 7, [300 + i for i in range(45)], [250] * 45, None, "spread"),              # of 1
    ("bf16", 1, 16, 16, [40000], [17000], [1000], "few"),
    ("bf16", 1, 16, 16, [70000], [17001], [13], "equal"),      # slices longer than their bits in shared memory
    ("bf16", 2, 16, 300, [2000, 2300], [999, 1000], [10, 1000], "spread"),  # rings that turn in shared memory
    ("f32", 2, 8, 700, [2000, 2300], [999, 1000], [10, 1000], "spread"),    # and by reflections
]


@pytest.mark.parametrize("dtype,Hkv,dd,w,lens,keep,protect,kind", CASES)
def test_evict(dtype, Hkv, dd, w, lens, keep, protect, kind):
    c, full = R.filled_cache(dar, 17 * len(lens) + dd, dtype, Hkv, dd, w, lens)
    t = totals(kind, c, lens, 5)
    weights = t.cuda()
    before = state(c)
    held = [R.contents(c, full, b) for b in range(c.B)]
    dar.dar_cache_evict(c, weights, ints(keep), dar.evict_workspace(c), protect=None if protect is None else ints(protect))
    torch.cuda.synchronize()
    assert c.device_status() == 0
    want = [x.clone() for x in before]
    want_w = t.clone()
    for b, L in enumerate(lens):
        n = max(0, L - w)
        if n <= keep[b]:
            continue
        want[4][b] = keep[b] + w
        kd, vd, k, v = held[b]
        for g in range(Hkv):
            first = protect[b] if protect else 0
            nkd, nvd, _, _, nw = R.evict(kd[g], vd[g], k[g], v[g], t[b, g, :L].tolist(), keep[b], first, w)
            for j in range(n):
                pg = full[b][j // 64]
                want[0][pg, g, j % 64], want[1][pg, g, j % 64] = nkd[j].to(R.DT[dtype]), nvd[j].to(R.DT[dtype])
            want_w[b, g, :L] = torch.tensor(nw)
            slots = torch.arange(keep[b], keep[b] + w) % w
            want[2][b, g, slots], want[3][b, g, slots] = k[g].to(R.DT[dtype]), v[g].to(R.DT[dtype])
    names = ("pool_kd", "pool_vd", "win_k", "win_v", "seq_lens")
    for name, a, b in zip(names, state(c), want):
        assert same(a, b), name
    assert same(weights.cpu(), want_w)


def test_bad_sequences_are_left_as_they_are():
    lens = [500, 520, 540, 560]
    for what, code in (("keep", dar.DAR_ERR_INVALID_ARG), ("protect", dar.DAR_ERR_INVALID_ARG),
                       ("order", dar.DAR_ERR_INVALID_ARG), ("page", dar.DAR_ERR_CAPACITY),
                       ("length", dar.DAR_ERR_CAPACITY), ("minus", dar.DAR_ERR_CAPACITY)):
        c, full = R.filled_cache(dar, 8, "bf16", 2, 16, 40, lens)
        keep, protect = ints([200] * 4), ints([10] * 4)
        if what == "keep":
            keep[1] = -1
        elif what == "protect":
            protect[1] = -3
        elif what == "order":
            protect[1] = 201
        elif what == "page":
            c.block_table[1, 4] = c.num_pages
        elif what == "length":
            c.seq_lens[1] = c.max_pages_per_seq * 64 + c.w + 1
        else:
            c.seq_lens[1] = -1
        weights = totals("spread", c, lens, 1).cuda()
        before, w0 = state(c), weights.clone()
        dar.dar_cache_evict(c, weights, keep, dar.evict_workspace(c), protect=protect)
        torch.cuda.synchronize()
        assert c.device_status() == code, what
        after = state(c)
        mine = full[1]
        assert same(after[0][mine], before[0][mine]) and same(after[1][mine], before[1][mine])
        assert all(same(after[i][1], before[i][1]) for i in (2, 3, 4)) and torch.equal(weights[1], w0[1])
        assert after[4].tolist()[0] == 240 and after[4].tolist()[2:] == [240, 240]


def test_protected_pages_can_be_shared_and_need_not_be_listed():
    """Pages in the protected part are not looked at: not their ids, not their bytes."""
    c, full = R.filled_cache(dar, 8, "bf16", 2, 16, 40, [700, 720])
    weights = totals("spread", c, None, 1).cuda()
    shared = c.block_table[0, :3].clone()
    c.block_table[1, :3] = -1
    before = state(c)
    dar.dar_cache_evict(c, weights, ints([300, 300]), dar.evict_workspace(c), protect=ints([192, 192]))
    torch.cuda.synchronize()
    assert c.device_status() == 0 and c.seq_lens.tolist() == [340, 340]
    for i in (0, 1):
        assert same(state(c)[i][shared.long().cpu()], before[i][shared.long().cpu()])


def test_captured_and_repeated():
    """A captured call gives the bits of an eager one; a second call in the same state changes nothing."""
    lens = [900, 450, 1000]
    c, _ = R.filled_cache(dar, 8, "bf16", 4, 16, 40, lens)
    weights = totals("few", c, lens, 1).cuda()
    keep, protect, ws = ints([300, 500, 317]), ints([5, 0, 317]), dar.evict_workspace(c)
    tensors = (c.pool_kd, c.pool_vd, c.win_k, c.win_v, c.seq_lens, weights)
    first = [t.clone() for t in tensors]
    dar.dar_cache_evict(c, weights, keep, ws, protect=protect)
    want = [t.clone() for t in tensors]
    dar.dar_cache_evict(c, weights, keep, ws, protect=protect)
    assert all(same(a.cpu(), b.cpu()) for a, b in zip(tensors, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dar.dar_cache_evict(c, weights, keep, ws, protect=protect)
    for _ in range(3):
        for t, x in zip(tensors, first):
            t.copy_(x)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert all(same(a.cpu(), b.cpu()) for a, b in zip(tensors, want))


def test_operands_are_checked():
    c, _ = R.filled_cache(dar, 8, "bf16", 2, 16, 40, [300, 300])
    weights, ws, keep = dar.attention_weights(c), dar.evict_workspace(c), ints([10, 10])
    for call in (lambda: dar.dar_cache_evict(c, weights[:1], keep, ws),
                 lambda: dar.dar_cache_evict(c, weights, keep[:1], ws),
                 lambda: dar.dar_cache_evict(c, weights, keep.long(), ws),
                 lambda: dar.dar_cache_evict(c, weights, keep, ws, protect=keep[:1]),
                 lambda: dar.dar_cache_evict(c, weights, keep.cpu(), ws),
                 lambda: dar.dar_cache_evict(c, weights.half(), keep, ws)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(dar.DarError):
        dar.dar_cache_evict(c, weights, keep, ws[:256])
    assert c.device_status() == 0
