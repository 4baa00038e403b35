"""Pages that several sequences list (a shared prefix, of which each has another number of distant tokens), written by all
of them in one call: the bytes are those of one sequence after the other."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)

from paper_2606_18587_gb300 import dar  # noqa: E402
from tests.helpers import q4_ref as Q  # noqa: E402
from tests.helpers import serving_ref as R  # noqa: E402

W, PAGES = 21, 3


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def shared(dtype, B, Hkv, dd, seed):
    """A cache of B sequences that all list the same pages, which are full."""
    table = torch.tensor([[2, 0, 1]], dtype=torch.int32).repeat(B, 1)
    c = dar.DarCache(B, Hkv, dd, W, PAGES, PAGES, dtype=R.DT[dtype], block_table=table)
    g = torch.Generator(device="cuda").manual_seed(seed)
    for t in (c.pool_kd, c.pool_vd):
        t.normal_(generator=g)
    return c


@pytest.mark.parametrize("dtype,B,Hkv,dd", [
    ("bf16", 64, 2, 16), ("bf16", 64, 2, 8), ("bf16", 64, 1, 64), ("f32", 64, 2, 32), ("f32", 64, 3, 8),
    ("bf16", 260, 8, 16), ("bf16", 260, 8, 8), ("bf16", 260, 7, 32), ("f32", 260, 8, 16),  # a warp takes a whole page
])
@pytest.mark.parametrize("start", ["none", "close", "far"])
def test_pack(dtype, B, Hkv, dd, start):
    """Distant parts that end in all rows of a page, and begin there too."""
    c = shared(dtype, B, Hkv, dd, 5)
    ends = [(64 + 61 * b) % (64 * PAGES + 1) for b in range(B)]
    begin = {"none": [0] * B, "close": [max(0, e - 1 - b % 9) for b, e in enumerate(ends)],
             "far": [(37 * b) % (e + 1) for b, e in enumerate(ends)]}[start]
    first = None if start == "none" else ints(begin)
    before = Q.beside(dar, c, seed=9).pool
    want = dar.DarCacheQ4.beside(c)
    want.pool.copy_(before)
    for b in range(B):
        c.seq_lens.fill_(W)
        c.seq_lens[b] = W + ends[b]
        dar.dar_cache_pack_q4(c, want, first=first)
    assert not torch.equal(want.pool, before)
    got = dar.DarCacheQ4.beside(c)
    c.seq_lens.copy_(ints([W + e for e in ends]))
    for i in range(20):
        got.pool.copy_(before)
        dar.dar_cache_pack_q4(c, got, first=first)
        assert torch.equal(got.pool, want.pool), i
    assert got.device_status() == 0


def appended(dtype, B, Hkv, dd, n, lens, per):
    """Appends of the tokens of one text to sequences at different places of it: one after the other, and together."""
    assert max(L + m for L, m in zip(lens, per)) <= W + 64 * PAGES
    g = torch.Generator(device="cuda").manual_seed(6)
    text = [torch.randn((Hkv, W + 64 * PAGES + n, 64), device="cuda", generator=g).to(R.DT[dtype]) for _ in range(2)]
    Dk, Dv = (torch.randn((Hkv, 64, dd), device="cuda", generator=g) / 8 for _ in range(2))
    new = [torch.stack([t[:, L:L + n] for L in lens]) for t in text]
    c = shared(dtype, B, Hkv, dd, 5)
    before = Q.beside(dar, c, seed=9).pool

    def cache():
        c4 = dar.DarCacheQ4(B, Hkv, dd, W, PAGES, PAGES, dtype=R.DT[dtype], block_table=c.block_table.cpu())
        c4.pool.copy_(before)
        for b, L in enumerate(lens):
            at = torch.arange(max(0, L - W), L, device="cuda")
            c4.win_k[b][:, at % W] = text[0][:, at]
            c4.win_v[b][:, at % W] = text[1][:, at]
        c4.seq_lens.copy_(ints(lens))
        return c4
    want = cache()
    for b in range(B):
        dar.dar_cache_append_q4(want, *new, Dk, Dv, n_per_seq=ints([per[b] if i == b else 0 for i in range(B)]))
    assert not torch.equal(want.pool, before)
    start = cache()
    got = cache()
    for i in range(10):
        for t, s in ((got.pool, before), (got.win_k, start.win_k), (got.win_v, start.win_v), (got.seq_lens, start.seq_lens)):
            t.copy_(s)
        dar.dar_cache_append_q4(got, *new, Dk, Dv, n_per_seq=ints(per))
        assert torch.equal(got.pool, want.pool), i
        for x, y in ((got.win_k, want.win_k), (got.win_v, want.win_v), (got.seq_lens, want.seq_lens)):
            assert torch.equal(x, y)
    assert got.device_status() == 0 and want.device_status() == 0


@pytest.mark.parametrize("dtype,Hkv,dd", [("bf16", 2, 16), ("bf16", 2, 8), ("bf16", 1, 64), ("f32", 2, 32)])
def test_append_of_many_tokens(dtype, Hkv, dd):
    B, n = 48, 70
    lens = [(29 * b) % (W + 64 * PAGES - n + 1) for b in range(B)]
    appended(dtype, B, Hkv, dd, n, lens, [n - (5 * b) % 23 for b in range(B)])


@pytest.mark.parametrize("dtype,B,Hkv,dd,n", [
    ("bf16", 64, 2, 16, 3), ("bf16", 400, 2, 16, 8), ("bf16", 260, 6, 8, 8), ("bf16", 64, 1, 64, 2), ("bf16", 90, 5, 32, 5),
    ("f32", 200, 4, 16, 8), ("f32", 64, 1, 8, 2),
])
def test_append_of_few_tokens(dtype, B, Hkv, dd, n):
    """Sequences one or a few tokens apart, which write neighbouring rows of the same words."""
    lens = [W + 30 + b % 7 + 64 * (b // 7 % 2) for b in range(B)]
    appended(dtype, B, Hkv, dd, n, lens, [n - b % 3 % n for b in range(B)])


@pytest.mark.parametrize("dd,Hq", [(16, 2), (16, 16), (8, 8), (64, 8)])
def test_steps_of_sequences_that_share(dd, Hq):
    """Steps of sequences a token or two apart on one text: each attends as one that has the pages to itself."""
    B, Hkv, n = 12, 2, 1
    lens = [W + 37 + b % 4 for b in range(B)]
    g = torch.Generator(device="cuda").manual_seed(8)
    text = [torch.randn((Hkv, W + 64 * PAGES, 64), device="cuda", generator=g).bfloat16() for _ in range(2)]
    Dk, Dv = (torch.randn((Hkv, 64, dd), device="cuda", generator=g) / 8 for _ in range(2))
    both = []
    for table in (torch.tensor([[2, 0, 1]], dtype=torch.int32).repeat(B, 1), None):
        c4 = dar.DarCacheQ4(B, Hkv, dd, W, PAGES, B * PAGES, block_table=table)
        dar.dar_cache_append_q4(c4, *[t[None, :, :max(lens)].repeat(B, 1, 1, 1) for t in text], Dk, Dv,
                                n_per_seq=ints(lens))
        both.append((c4, dar.decode_q4_workspace(c4, Hq)))
    q, Uk, Uv = R.operands(3, "bf16", B, Hq, Hkv, dd)
    for i in range(40):
        new = [torch.stack([t[:, L + i:L + i + 1] for L in lens]) for t in text]
        a, b = (dar.dar_decode_step_q4(c4, *new, Dk, Dv, q, Uk, Uv, ws) for c4, ws in both)
        assert torch.equal(a, b), i
    assert all(c4.device_status() == 0 for c4, _ in both)
