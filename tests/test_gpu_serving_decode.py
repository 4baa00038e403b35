"""dar_attn_decode_shared and dar_attn_decode_scored against softmax attention over the lifted keys in 64 bits."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)

from paper_2606_18587_gb300 import dar  # noqa: E402
from tests.helpers import serving_ref as R  # noqa: E402


def check_outputs(dtype, cache, full, q, Uk, Uv, got, scale=R.D ** -0.5, rows=None):
    """Compares got [B][Hq][64]; returns each sequence's weights [Hq][L] and top (see attend)."""
    wts = []
    for b in range(cache.B):
        kd, vd, k, v = R.contents(cache, full, b)
        if kd.shape[1] + k.shape[1] == 0:
            assert not got[b].any()
            wts.append(None)
            continue
        out, p, mag, top = R.attend(q[b].cpu().double(), kd, vd, k, v, Uk.cpu().double(), Uv.cpu().double(), scale)
        err, tol = (got[b].cpu().double() - out).abs(), R.tolerances(dtype, out, mag, top)
        assert not torch.isnan(err).any(), b
        assert (err <= tol).all(), (b, float((err / tol).max()))
        wts.append((p, top))
    return wts


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


SHARED = [
    # dtype, Hq, Hkv, dd, w, lens, group, pages
    ("bf16", 4, 4, 16, 8, [200, 200], [0, 0], [3]),                            # one page boundary exactly at the end
    ("bf16", 4, 4, 16, 8, [201, 263, 264, 265], [0, 0, 0, 0], [3]),            # rests of 1, 63, 64 and 65 tokens
    ("bf16", 12, 12, 16, 128, [1300 + 7 * i for i in range(9)], [0] * 9, [18]),
    ("bf16", 8, 2, 16, 33, [700, 0, 400, 1, 33, 650, 640, 34], [0, 0, 1, 1, 1, 0, 0, -1], [9, 5]),  # empty, short
    ("bf16", 8, 1, 16, 64, [900] * 3 + [500] * 2, [1, 0, 1, 0, 1], [4, 2]),    # interleaved groups, G = 8
    ("bf16", 20, 1, 16, 17, [300, 310, 320], [0, 0, 0], [2]),                  # more rows than a tile per sequence
    ("bf16", 4, 4, 16, 8, [500, 600], [0, 1], [3, 4]),                         # groups of one
    ("bf16", 4, 4, 16, 8, [500, 600, 700], [-1, -1, -1], [3]),                 # nobody shares
    ("bf16", 4, 4, 16, 8, [500, 600, 700], [0, 0, 0], [0]),                    # nothing is shared
    ("bf16", 2, 2, 16, 1, [130, 129, 400], [0, 0, 0], [2]),                    # window of one token
    ("bf16", 4, 2, 8, 40, [1111, 1200, 1100], [0, 0, 0], [16]),
    ("bf16", 6, 2, 32, 40, [1111, 1200, 1100], [0, 0, 0], [16]),
    ("bf16", 4, 4, 64, 40, [1111, 1200, 1100], [0, 0, 0], [16]),
    ("bf16", 32, 8, 16, 256, [4500 + 13 * i for i in range(5)], [0, 0, 0, 0, 0], [66]),
    ("bf16", 8, 2, 16, 20, [420 + (i * 37) % 300 for i in range(70)], [i % 3 - (i % 11 == 0) * (i % 3 + 1) for i in
                                                                        range(70)], [6, 3, 1]),  # many rows, many tiles
    ("bf16", 80, 1, 16, 17, [300, 310, 320, 50], [0, 0, 0, -1], [2]),          # two row tiles a sequence
    ("bf16", 16, 1, 64, 30, [300, 310, 320, 50], [0, 0, 0, -1], [2]),          # sixteen rows a private unit
    ("bf16", 9, 1, 8, 30, [300, 310, 320, 50], [0, 0, 0, -1], [2]),
    ("bf16", 2, 2, 16, 500, [100, 400, 500, 501, 564, 565], [0] * 6, [1]),     # windows that hold almost all
    ("bf16", 1, 1, 16, 16, [40000, 40010], [0, 0], [600]),                     # one head over all CTAs
    ("f32", 4, 4, 16, 32, [230, 270], [0, 0], [3]),
    ("f32", 8, 2, 8, 21, [500, 510, 90, 600], [0, 0, 0, 0], [7]),
    ("f32", 6, 2, 32, 21, [500, 510, 90, 600], [0, 0, -1, 0], [7]),
    ("f32", 4, 4, 64, 50, [500, 510, 90, 0, 600], [0, 0, -1, 0, 0], [7]),
    ("f32", 20, 1, 16, 17, [300, 310, 320], [0, 0, 0], [4]),
]


@pytest.mark.parametrize("dtype,Hq,Hkv,dd,w,lens,group,pages", SHARED)
def test_shared(dtype, Hq, Hkv, dd, w, lens, group, pages):
    c, full = R.filled_cache(dar, 11 * len(lens) + dd, dtype, Hkv, dd, w, lens, group, pages)
    q, Uk, Uv = R.operands(dd + w, dtype, len(lens), Hq, Hkv, dd)
    got = dar.dar_attn_decode_shared(c, q, Uk, Uv, ints(group), ints(pages), dar.shared_decode_workspace(c, Hq))
    torch.cuda.synchronize()
    assert c.device_status() == 0
    check_outputs(dtype, c, full, q, Uk, Uv, got)


def test_shared_without_groups():
    c, full = R.filled_cache(dar, 5, "bf16", 2, 16, 20, [300, 0, 5])
    q, Uk, Uv = R.operands(6, "bf16", 3, 4, 2, 16)
    got = dar.dar_attn_decode_shared(c, q, Uk, Uv, ints([-1] * 3), ints([]), dar.shared_decode_workspace(c, 4), scale=0.3)
    check_outputs("bf16", c, full, q, Uk, Uv, got, scale=0.3)
    assert c.device_status() == 0


def test_shared_peaked_scores():
    """Scores of a standard deviation of 12: a few tokens hold all the weight."""
    lens, group, pages = [900, 950, 1000], [0, 0, 0], [12]
    c, full = R.filled_cache(dar, 3, "bf16", 2, 16, 40, lens, group, pages)
    q, Uk, Uv = R.operands(4, "bf16", 3, 8, 2, 16, q_std=12.0)
    got = dar.dar_attn_decode_shared(c, q, Uk, Uv, ints(group), ints(pages), dar.shared_decode_workspace(c, 8))
    check_outputs("bf16", c, full, q, Uk, Uv, got)


@pytest.mark.parametrize("dd,growth", [(16, 3.0), (16, 40.0), (8, 10.0), (64, 10.0), (32, -1.0)])
def test_shared_scores_that_rise_along_the_prefix(dd, growth):
    """Weights are taken relative to a maximum that is raised only when sums get far: keys that grow by page raise
    it again and again; growth -1: the first pages score the lowest numbers there are, the last ordinary ones."""
    lens, group, pages = [900, 950, 1000, 980, 990], [0] * 5, [13]
    c, full = R.filled_cache(dar, 3, "bf16", 2, dd, 40, lens, group, pages)
    q, Uk, Uv = R.operands(4, "bf16", 5, 8, 2, dd)
    for i, pg in enumerate(full[0][:13]):
        if growth > 0:
            c.pool_kd[pg] *= 1.0 + growth * i
        elif i < 11:
            # k^D = -M sum over the heads' and rows' q~: a large negative score for every row
            qt = torch.einsum("bhd,hed->bhe", q.float().view(5, 2, 4, 64).sum(2), Uk).mean(0)
            c.pool_kd[pg] = (-1e3 * qt / qt.norm(dim=-1, keepdim=True)).bfloat16()[:, None]
    got = dar.dar_attn_decode_shared(c, q, Uk, Uv, ints(group), ints(pages), dar.shared_decode_workspace(c, 8))
    torch.cuda.synchronize()
    check_outputs("bf16", c, full, q, Uk, Uv, got)


def test_shared_reads_only_the_first_members_entries_of_the_prefix():
    """filled_cache leaves -1 in the others' tables; entries that name other pages change nothing either."""
    lens, group, pages = [500, 520, 540], [0, 0, 0], [5]
    c, full = R.filled_cache(dar, 8, "bf16", 2, 16, 40, lens, group, pages)
    q, Uk, Uv = R.operands(9, "bf16", 3, 4, 2, 16)
    ws = dar.shared_decode_workspace(c, 4)
    a = dar.dar_attn_decode_shared(c, q, Uk, Uv, ints(group), ints(pages), ws)
    c.block_table[1:, :5] = c.block_table[0, 5]
    b = dar.dar_attn_decode_shared(c, q, Uk, Uv, ints(group), ints(pages), ws)
    assert torch.equal(a, b) and c.device_status() == 0


def test_shared_bad_groups_and_pages_are_reported():
    lens, group, pages = [500, 520, 540, 560], [0, 0, 0, 0], [5]
    c, full = R.filled_cache(dar, 8, "bf16", 2, 16, 40, lens)
    q, Uk, Uv = R.operands(9, "bf16", 4, 4, 2, 16)
    ws = dar.shared_decode_workspace(c, 4)
    for bad in (1, 7, -2, -2 ** 31, 2 ** 31 - 1):
        c.status.zero_()
        got = dar.dar_attn_decode_shared(c, q, Uk, Uv, ints([-1, -1, bad, -1]), ints(pages), ws)
        assert c.device_status() == dar.DAR_ERR_INVALID_ARG
        check_outputs("bf16", c, full, q, Uk, Uv, got)  # attended alone
    for bad in (-1, c.max_pages_per_seq + 1, 2 ** 31 - 1, -2 ** 31):
        c.status.zero_()
        got = dar.dar_attn_decode_shared(c, q, Uk, Uv, ints(group), ints([bad]), ws)
        assert c.device_status() == dar.DAR_ERR_CAPACITY
        check_outputs("bf16", c, full, q, Uk, Uv, got)
    good = c.block_table.clone()
    for bad in (-1, c.num_pages, 2 ** 31 - 1, -2 ** 31):
        c.status.zero_()
        c.block_table[2, 3] = bad
        got = dar.dar_attn_decode_shared(c, q, Uk, Uv, ints([-1] * 4), ints(pages), ws)
        assert c.device_status() == dar.DAR_ERR_CAPACITY
        c.block_table.copy_(good)
        keep = [0, 1, 3]  # the others are right
        want = dar.dar_attn_decode_shared(c, q, Uk, Uv, ints([-1] * 4), ints(pages), ws)
        assert torch.equal(got[keep], want[keep])
    for bad in (-1, c.max_pages_per_seq * 64 + c.w + 1, 2 ** 31 - 1):
        c.status.zero_()
        c.seq_lens[1] = bad
        got = dar.dar_attn_decode_shared(c, q, Uk, Uv, ints([-1] * 4), ints(pages), ws)
        assert c.device_status() == dar.DAR_ERR_CAPACITY
        assert torch.equal(got[[0, 2, 3]], want[[0, 2, 3]])
        c.seq_lens[1] = lens[1]


SCORED = [
    ("bf16", 8, 8, 16, 128, [101]),
    ("bf16", 4, 4, 16, 8, [0, 1, 7, 8, 9, 71, 72, 73, 136, 137]),
    ("bf16", 12, 12, 16, 128, [1300 + 7 * i for i in range(5)]),
    ("bf16", 8, 2, 16, 33, [700, 0, 4000, 1, 33, 650]),
    ("bf16", 20, 1, 16, 17, [300, 2100]),
    ("bf16", 16, 2, 8, 40, [1111, 3000]),
    ("bf16", 6, 2, 32, 40, [1111, 1200]),
    ("bf16", 4, 4, 64, 1000, [1111, 1200, 30]),
    ("bf16", 2, 2, 16, 1, [1, 2, 65, 66]),
    ("bf16", 70, 1, 16, 17, [300, 2100]),
    ("bf16", 16, 1, 8, 17, [300, 2100]),
    ("bf16", 12, 1, 32, 17, [300, 2100]),
    ("bf16", 1, 1, 16, 16, [40003]),
    ("f32", 8, 4, 16, 37, [20, 1501, 700]),
    ("f32", 4, 4, 8, 21, [500, 0, 90]),
    ("f32", 6, 2, 32, 21, [500, 510]),
    ("f32", 4, 4, 64, 50, [500, 90]),
]


@pytest.mark.parametrize("decay", [1.0, 0.0, 0.75])
@pytest.mark.parametrize("dtype,Hq,Hkv,dd,w,lens", SCORED)
def test_scored(dtype, Hq, Hkv, dd, w, lens, decay):
    c, full = R.filled_cache(dar, 13 * len(lens) + dd, dtype, Hkv, dd, w, lens)
    q, Uk, Uv = R.operands(dd + w, dtype, len(lens), Hq, Hkv, dd, q_std=2.0)
    weights = dar.attention_weights(c).uniform_(generator=torch.Generator("cuda").manual_seed(1))
    if decay == 0.0:
        weights.fill_(float("nan"))  # whatever was there is gone
    old = weights.cpu().double()
    got = dar.dar_attn_decode_scored(c, q, Uk, Uv, weights, dar.scored_decode_workspace(c, Hq), decay=decay)
    torch.cuda.synchronize()
    assert c.device_status() == 0
    wts = check_outputs(dtype, c, full, q, Uk, Uv, got)
    new = weights.cpu().double()
    for b, L in enumerate(lens):
        assert torch.equal(new[b, :, L:].nan_to_num(-1.0), old[b, :, L:].nan_to_num(-1.0))
        if L == 0:
            continue
        p, top = wts[b]
        p = p.view(Hkv, Hq // Hkv, L).sum(1)
        base = decay * old[b, :, :L] if decay else torch.zeros_like(p)
        err, tol = (new[b, :, :L] - (base + p)).abs(), R.weight_tolerance(p, base, top)
        assert (err <= tol).all(), (b, float((err / tol).max()))


def test_scored_sums_to_the_query_heads():
    """Each step adds weights that sum to the query heads per KV head, and steps accumulate."""
    c, _ = R.filled_cache(dar, 2, "bf16", 2, 16, 50, [400, 3, 2500])
    q, Uk, Uv = R.operands(3, "bf16", 3, 8, 2, 16)
    weights, ws = dar.attention_weights(c), dar.scored_decode_workspace(c, 8)
    for step in range(1, 4):
        dar.dar_attn_decode_scored(c, q, Uk, Uv, weights, ws)
        total = weights.double().sum(-1)
        # sums of p: each p is off by some 2^-18 at most, and so is their sum
        assert ((total - 4.0 * step).abs() <= 4.0 * step * 2.0 ** -17).all()


def test_scored_reports_bad_pages_and_lengths():
    c, full = R.filled_cache(dar, 8, "bf16", 2, 16, 40, [500, 520, 540])
    q, Uk, Uv = R.operands(9, "bf16", 3, 4, 2, 16)
    ws = dar.scored_decode_workspace(c, 4)
    good = c.block_table.clone()
    want = dar.dar_attn_decode_scored(c, q, Uk, Uv, dar.attention_weights(c), ws)
    for bad in (-1, c.num_pages):
        c.status.zero_()
        c.block_table[1, 2] = bad
        weights = dar.attention_weights(c)
        got = dar.dar_attn_decode_scored(c, q, Uk, Uv, weights, ws)
        assert c.device_status() == dar.DAR_ERR_CAPACITY
        assert torch.equal(got[[0, 2]], want[[0, 2]])
        assert torch.isfinite(weights[[0, 2]]).all()
        c.block_table.copy_(good)
    for bad in (-5, c.max_pages_per_seq * 64 + c.w + 1, 2 ** 31 - 1):
        c.status.zero_()
        c.seq_lens[1] = bad
        weights = torch.full_like(weights, 7.0)
        got = dar.dar_attn_decode_scored(c, q, Uk, Uv, weights, ws)
        assert c.device_status() == dar.DAR_ERR_CAPACITY
        assert torch.equal(got[[0, 2]], want[[0, 2]])
        assert (weights[1] == 7.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_same_bits_eager_captured_and_on_another_stream(dtype):
    lens, group, pages = [900, 950, 1000, 30], [0, 0, 0, 0], [12]
    c, _ = R.filled_cache(dar, 3, dtype, 2, 16, 40, lens, group, pages)
    q, Uk, Uv = R.operands(4, dtype, 4, 8, 2, 16)
    for b in (1, 2):
        c.block_table[b, :12] = c.block_table[0, :12]
    g, p = ints(group), ints(pages)
    sh, sc = dar.shared_decode_workspace(c, 8), dar.scored_decode_workspace(c, 8)
    weights = dar.attention_weights(c).fill_(9.0)  # entries behind a sequence's end keep this
    out1, out2 = torch.empty_like(q), torch.empty_like(q)

    def both(stream=None):
        dar.dar_attn_decode_shared(c, q, Uk, Uv, g, p, sh, out=out1, stream=stream)
        dar.dar_attn_decode_scored(c, q, Uk, Uv, weights, sc, decay=0.0, out=out2, stream=stream)

    both()
    torch.cuda.synchronize()
    want = [t.clone() for t in (out1, out2, weights)]
    s = torch.cuda.Stream()
    for t in (out1, out2, weights):
        t.fill_(9.0)
    s.wait_stream(torch.cuda.current_stream())
    both(stream=s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((out1, out2, weights), want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for _ in range(3):
        for t in (out1, out2, weights):
            t.fill_(9.0)
        sh.fill_(255)  # a workspace needs no initialisation
        sc.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((out1, out2, weights), want))


def test_a_cache_without_pages_and_an_empty_batch():
    c = dar.DarCache(3, 2, 16, 30, 0)
    k, v = (torch.randn((3, 2, 30, 64), device="cuda").bfloat16() for _ in range(2))
    D = torch.zeros((2, 64, 16), device="cuda")
    dar.dar_cache_append(c, k, v, D, D, n_per_seq=ints([30, 0, 7]))
    q, Uk, Uv = R.operands(4, "bf16", 3, 4, 2, 16)
    # (rows that were never written are zero here, not NaN: the cache is the library's own)
    got = dar.dar_attn_decode_shared(c, q, Uk, Uv, ints([0, 0, 0]), ints([0]), dar.shared_decode_workspace(c, 4))

    def empty_contents(b):
        L = int(c.seq_lens[b])
        none = torch.zeros((2, 0, 16), dtype=torch.float64)
        return none, none, c.win_k[b, :, :L].cpu().double(), c.win_v[b, :, :L].cpu().double()
    weights = dar.attention_weights(c)
    assert weights.shape == (3, 2, 30)
    same = dar.dar_attn_decode_scored(c, q, Uk, Uv, weights, dar.scored_decode_workspace(c, 4))
    for b in (0, 2):
        out, p, mag, top = R.attend(q[b].cpu().double(), *empty_contents(b), Uk.cpu().double(), Uv.cpu().double())
        tol = R.tolerances("bf16", out, mag, top)
        assert ((got[b].cpu().double() - out).abs() <= tol).all() and ((same[b].cpu().double() - out).abs() <= tol).all()
    assert not got[1].any() and not weights[1].any()
    dar.dar_cache_evict(c, weights, ints([0, 0, 0]), dar.evict_workspace(c))
    assert c.seq_lens.tolist() == [30, 0, 7] and c.device_status() == 0
    e = dar.DarCache(0, 2, 16, 30, 4)
    q0 = torch.zeros((0, 4, 64), dtype=torch.bfloat16, device="cuda")
    assert dar.dar_attn_decode_shared(e, q0, Uk, Uv, ints([]), ints([]), dar.shared_decode_workspace(e, 4)).shape == q0.shape
    dar.dar_attn_decode_scored(e, q0, Uk, Uv, dar.attention_weights(e), dar.scored_decode_workspace(e, 4))
    dar.dar_cache_evict(e, dar.attention_weights(e), ints([]), dar.evict_workspace(e))


def test_operands_are_checked():
    c, _ = R.filled_cache(dar, 3, "bf16", 2, 16, 40, [100, 200])
    q, Uk, Uv = R.operands(4, "bf16", 2, 4, 2, 16)
    ws, weights = dar.scored_decode_workspace(c, 4), dar.attention_weights(c)
    g, p = ints([0, 0]), ints([1])
    sh = dar.shared_decode_workspace(c, 4)
    bad = [
        lambda: dar.dar_attn_decode_shared(c, q[:1], Uk, Uv, g, p, sh),
        lambda: dar.dar_attn_decode_shared(c, q.float(), Uk, Uv, g, p, sh),
        lambda: dar.dar_attn_decode_shared(c, q, Uk[:1], Uv, g, p, sh),
        lambda: dar.dar_attn_decode_shared(c, q, Uk, Uv.bfloat16(), g, p, sh),
        lambda: dar.dar_attn_decode_shared(c, q, Uk, Uv, g[:1], p, sh),
        lambda: dar.dar_attn_decode_shared(c, q, Uk, Uv, g.long(), p, sh),
        lambda: dar.dar_attn_decode_shared(c, q, Uk, Uv, g.cpu(), p, sh),
        lambda: dar.dar_attn_decode_shared(c, q.transpose(0, 1).contiguous().transpose(0, 1), Uk, Uv, g, p, sh),
        lambda: dar.dar_attn_decode_scored(c, q, Uk, Uv, weights[..., :-1].contiguous(), ws),
        lambda: dar.dar_attn_decode_scored(c, q, Uk, Uv, weights.double(), ws),
        lambda: dar.dar_attn_decode_scored(c, q, Uk, Uv, weights.cpu(), ws),
    ]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    for call in (lambda: dar.dar_attn_decode_shared(c, q, Uk, Uv, g, ints([1, 1, 1]), sh),
                 lambda: dar.dar_attn_decode_shared(c, q, Uk, Uv, g, p, sh[:256]),
                 lambda: dar.dar_attn_decode_scored(c, q, Uk, Uv, weights, ws, decay=1.5),
                 lambda: dar.dar_attn_decode_scored(c, q, Uk, Uv, weights, ws, decay=float("nan")),
                 lambda: dar.dar_attn_decode_scored(c, q[:, :3].contiguous(), Uk, Uv, weights, ws)):
        with pytest.raises(dar.DarError):
            call()
    assert c.device_status() == 0


def test_the_largest_batch():
    """1024 sequences, some empty, in 40 groups in no order; f32 so that the comparison is sharp."""
    g = torch.Generator().manual_seed(4)
    B, pages = 1024, [int(x) for x in torch.randint(0, 3, (40,), generator=g)]
    group = [int(x) for x in torch.randint(-1, 40, (B,), generator=g)]
    lens = [0 if i % 97 == 5 else 5 + 64 * (pages[k] if k >= 0 else 1) + int(x)
            for i, (k, x) in enumerate(zip(group, torch.randint(0, 90, (B,), generator=g)))]
    c, full = R.filled_cache(dar, 6, "f32", 1, 8, 5, lens, group, pages)
    q, Uk, Uv = R.operands(7, "f32", B, 2, 1, 8)
    got = dar.dar_attn_decode_shared(c, q, Uk, Uv, ints(group), ints(pages), dar.shared_decode_workspace(c, 2))
    torch.cuda.synchronize()
    assert c.device_status() == 0
    check_outputs("f32", c, full, q, Uk, Uv, got)


def test_infinite_and_nan_inputs_stay_in_their_sequence():
    """A NaN query, an infinite key and an infinite value of one member reach nobody else's output."""
    lens, group, pages = [500, 520, 540, 45], [0, 0, 0, -1], [5]
    c, full = R.filled_cache(dar, 8, "bf16", 2, 16, 40, lens, group, pages)
    q, Uk, Uv = R.operands(9, "bf16", 4, 4, 2, 16)
    ws = dar.shared_decode_workspace(c, 4)
    want = dar.dar_attn_decode_shared(c, q, Uk, Uv, ints(group), ints(pages), ws)
    q[1, 0] = float("nan")
    c.win_v[1] = float("inf")
    c.pool_kd[full[1][6]] = float("inf")
    got = dar.dar_attn_decode_shared(c, q, Uk, Uv, ints(group), ints(pages), ws)
    assert torch.equal(got[[0, 2, 3]], want[[0, 2, 3]])
    assert torch.isnan(got[1]).all()


def test_calls_of_two_streams_with_workspaces_of_their_own():
    lens, group, pages = [2000 + i for i in range(16)], [0] * 16, [25]
    c, _ = R.filled_cache(dar, 8, "bf16", 2, 16, 40, lens, group, pages)
    q, Uk, Uv = R.operands(9, "bf16", 16, 4, 2, 16)
    for b in range(1, 16):
        c.block_table[b, :25] = c.block_table[0, :25]
    g, p = ints(group), ints(pages)
    want = dar.dar_attn_decode_shared(c, q, Uk, Uv, g, p, dar.shared_decode_workspace(c, 4))
    weights = [dar.attention_weights(c) for _ in range(3)]
    dar.dar_attn_decode_scored(c, q, Uk, Uv, weights[2], dar.scored_decode_workspace(c, 4))
    streams = [torch.cuda.Stream() for _ in range(2)]
    ws = [dar.shared_decode_workspace(c, 4) for _ in streams]
    wsc = [dar.scored_decode_workspace(c, 4) for _ in streams]
    outs = [torch.empty_like(q) for _ in streams]
    torch.cuda.synchronize()
    for _ in range(20):
        for i, s in enumerate(streams):
            dar.dar_attn_decode_shared(c, q, Uk, Uv, g, p, ws[i], out=outs[i], stream=s)
    for i, s in enumerate(streams):
        dar.dar_attn_decode_scored(c, q, Uk, Uv, weights[i], wsc[i], stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
    assert all(torch.equal(x, weights[2]) for x in weights[:2])
