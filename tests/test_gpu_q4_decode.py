"""dar_attn_decode_q4 against softmax attention over the values that the pages stand for, in 64 bits."""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)

from paper_2606_18587_gb300 import dar  # noqa: E402
from tests.helpers import q4_ref as Q  # noqa: E402
from tests.helpers import serving_ref as R  # noqa: E402


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


DECODE = [
    # dtype, Hq, Hkv, dd, w, lens
    ("bf16", 4, 4, 16, 8, [200, 0, 1, 7, 8, 9, 71, 72, 73, 136]),              # page and window edges, an empty one
    ("bf16", 2, 2, 16, 1, [130, 1, 2, 65, 66]),                                # window of one token
    ("bf16", 12, 12, 16, 128, [1300 + 7 * i for i in range(9)]),
    ("bf16", 8, 4, 16, 33, [700, 0, 400, 1, 33, 650]),                         # two query heads a KV head
    ("bf16", 6, 2, 16, 33, [700, 30, 400]),                                    # three
    ("bf16", 32, 8, 16, 256, [4500 + 13 * i for i in range(5)]),
    ("bf16", 10, 2, 16, 40, [411, 1500]),                                      # five
    ("bf16", 8, 1, 16, 64, [900, 500]),
    ("bf16", 9, 1, 16, 64, [900, 500]),                                        # two tiles of heads
    ("bf16", 20, 1, 16, 17, [300, 310, 16]),
    ("bf16", 4, 2, 8, 40, [1111, 1200, 41]),
    ("bf16", 8, 1, 8, 5, [1111, 70]),
    ("bf16", 6, 2, 32, 40, [1111, 1200, 41]),
    ("bf16", 8, 1, 32, 40, [1111, 1200, 41]),
    ("bf16", 4, 4, 64, 40, [1111, 1200, 41]),
    ("bf16", 16, 2, 64, 15, [999, 200]),
    ("bf16", 2, 2, 16, 500, [100, 400, 500, 501, 564, 565]),                   # windows that hold almost all
    ("bf16", 1, 1, 16, 16, [40000]),                                           # one head over all SMs
    ("bf16", 4, 2, 16, 64, [64 + 64 * i for i in range(12)]),                  # whole pages: one to eleven
    ("bf16", 2, 2, 64, 64, [64 + 64 * i + 1 for i in range(12)]),
    ("bf16", 2, 1, 8, 16, [3000, 17]),
    ("bf16", 1, 1, 32, 16, [3000, 17]),
    ("bf16", 8, 8, 16, 20, [20 + (i * 37) % 300 for i in range(70)]),          # many sequences
    ("f32", 4, 4, 16, 32, [230, 270, 0, 5]),
    ("f32", 8, 2, 8, 21, [500, 510, 90]),
    ("f32", 6, 2, 32, 21, [500, 510, 90]),
    ("f32", 5, 1, 64, 50, [500, 510, 51]),
    ("f32", 20, 1, 16, 17, [300, 17]),
]


def decode(c4, q, Uk, Uv, **kw):
    return dar.dar_attn_decode_q4(c4, q, Uk, Uv, dar.decode_q4_workspace(c4, q.shape[1]), **kw)


@pytest.mark.parametrize("dtype,Hq,Hkv,dd,w,lens", DECODE)
def test_decode(dtype, Hq, Hkv, dd, w, lens):
    c, full = R.filled_cache(dar, 11 * len(lens) + dd, dtype, Hkv, dd, w, lens)
    c4 = Q.beside(dar, c)
    dar.dar_cache_pack_q4(c, c4)
    q, Uk, Uv = R.operands(dd + w, dtype, len(lens), Hq, Hkv, dd)
    got = decode(c4, q, Uk, Uv)
    again = decode(c4, q, Uk, Uv)
    torch.cuda.synchronize()
    assert c4.device_status() == 0
    assert torch.equal(got, again)
    Q.check_outputs(dtype, Q.read_back(dar, c4), full, q, Uk, Uv, got)


def test_far_pages():
    """A pool of more than 4 GB whose last pages a sequence lists."""
    B, Hkv, dd, w, lens = 2, 8, 16, 16, [300, 77]
    c, full = R.filled_cache(dar, 6, "bf16", Hkv, dd, w, lens)
    n = (1 << 32) // (Hkv * dar.dar_q4_page_bytes(dd)) + 100
    table = torch.where(c.block_table >= 0, n - 1 - c.block_table, -1).cpu()
    c4 = dar.DarCacheQ4(B, Hkv, dd, w, c.max_pages_per_seq, n, block_table=table)
    for t, s in ((c4.win_k, c.win_k), (c4.win_v, c.win_v), (c4.seq_lens, c.seq_lens)):
        t.copy_(s)
    dar.dar_cache_pack_q4(c, c4)
    back = dar.DarCache(B, Hkv, dd, w, c.max_pages_per_seq, c.num_pages, block_table=c.block_table.cpu())
    dar.dar_cache_unpack_q4(c4, back)
    for t, s in ((back.win_k, c.win_k), (back.win_v, c.win_v), (back.seq_lens, c.seq_lens)):
        t.copy_(s)
    q, Uk, Uv = R.operands(6, "bf16", B, 16, Hkv, dd)
    Q.check_outputs("bf16", back, full, q, Uk, Uv, decode(c4, q, Uk, Uv))
    k, v = (torch.randn((B, Hkv, 3, 64), device="cuda").bfloat16() for _ in range(2))
    Dk, Dv = (torch.randn((Hkv, 64, dd), device="cuda") / 8 for _ in range(2))
    c4.seq_lens.sub_(3)
    plain = dar.DarCacheQ4.beside(back)
    plain.seq_lens.sub_(3)
    dar.dar_cache_append_q4(c4, k, v, Dk, Dv)
    dar.dar_cache_append_q4(plain, k, v, Dk, Dv)
    for b in range(B):
        for i, pg in enumerate(full[b]):
            if i == (lens[b] - w - 1) // 64:
                rows = dar.DarCache(B, Hkv, dd, w, c.max_pages_per_seq, c.num_pages, block_table=c.block_table.cpu())
                dar.dar_cache_unpack_q4(c4, rows, first=ints([max(0, L - w - 3) for L in lens]))
                other = dar.DarCache(B, Hkv, dd, w, c.max_pages_per_seq, c.num_pages, block_table=c.block_table.cpu())
                dar.dar_cache_unpack_q4(plain, other, first=ints([max(0, L - w - 3) for L in lens]))
                assert torch.equal(rows.pool_kd[pg], other.pool_kd[pg]) and rows.pool_kd[pg].any()
    assert c4.device_status() == 0


def test_scale_and_output():
    c, full = R.filled_cache(dar, 5, "bf16", 2, 16, 20, [300, 0, 5])
    c4 = Q.beside(dar, c)
    dar.dar_cache_pack_q4(c, c4)
    q, Uk, Uv = R.operands(6, "bf16", 3, 4, 2, 16)
    out = torch.full_like(q, math.nan)
    assert decode(c4, q, Uk, Uv, scale=0.3, out=out) is out
    Q.check_outputs("bf16", Q.read_back(dar, c4), full, q, Uk, Uv, out, scale=0.3)


@pytest.mark.parametrize("Hq", [2, 8, 16])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size,scale", [(1e-30, 0.125), (1e-30, 1e-30), (1.0, 1e-38), (1e-38, 1e-38), (0.0, 1e-38)])
def test_scores_that_vanish(dtype, size, scale, Hq):
    """Queries and scales whose product is no fp32 number: all weights are the same, and rows behind the last token
    still have none."""
    c, full = R.filled_cache(dar, 5, dtype, 2, 16, 20, [300, 21, 5])
    c4 = Q.beside(dar, c)
    dar.dar_cache_pack_q4(c, c4)
    q, Uk, Uv = R.operands(6, dtype, 3, Hq, 2, 16)
    q *= size
    Q.check_outputs(dtype, Q.read_back(dar, c4), full, q, Uk, Uv, decode(c4, q, Uk, Uv, scale=scale), scale=scale)


@pytest.mark.parametrize("std", [0.02, 12.0, 40.0])
@pytest.mark.parametrize("Hq", [2, 16])
def test_flat_and_peaked_scores(std, Hq):
    lens = [900, 950, 4000]
    c, full = R.filled_cache(dar, 3, "bf16", 2, 16, 40, lens)
    c4 = Q.beside(dar, c)
    dar.dar_cache_pack_q4(c, c4)
    q, Uk, Uv = R.operands(4, "bf16", 3, Hq, 2, 16, q_std=std)
    Q.check_outputs("bf16", Q.read_back(dar, c4), full, q, Uk, Uv, decode(c4, q, Uk, Uv))


@pytest.mark.parametrize("dd", [8, 16, 64])
@pytest.mark.parametrize("growth,values", [(3.0, 1.0), (40.0, 1.0), (1.0, 8.0), (0.5, 0.1), (-1.0, 1.0)])
def test_scores_and_scales_that_rise(dd, growth, values):
    """Keys that grow from page to page raise the scores again and again, values that grow or shrink by a factor
    move the weights' own reference; growth -1: the first pages score lowest."""
    lens = [900, 950, 70]
    c, full = R.filled_cache(dar, 3, "bf16", 2, dd, 40, lens)
    for b in range(3):
        for i, pg in enumerate(full[b]):
            c.pool_kd[pg] *= 1.0 + growth * i if growth > 0 else 1.0
            c.pool_vd[pg] *= values ** i
            if growth < 0 and i < 8:
                c.pool_kd[pg] = -300.0
    c4 = Q.beside(dar, c)
    dar.dar_cache_pack_q4(c, c4)
    q, Uk, Uv = R.operands(4, "bf16", 3, 8, 2, dd)
    if growth < 0:
        Uk.abs_()
        q.abs_()
    Q.check_outputs("bf16", Q.read_back(dar, c4), full, q, Uk, Uv, decode(c4, q, Uk, Uv))


@pytest.mark.parametrize("size", [1e-26, 1e-12, 1e12, 1e30])
@pytest.mark.parametrize("Hq", [2, 8, 16])
def test_values_of_every_size(size, Hq):
    """Values far from 1 (2^-90 to 2^100), in the ring too: sums stay finite and exact, relative to what they are made
    of."""
    lens = [300, 40, 700]
    c, full = R.filled_cache(dar, 3, "bf16", 2, 16, 40, lens)
    c.pool_vd *= size
    c.win_v *= size
    c4 = Q.beside(dar, c)
    dar.dar_cache_pack_q4(c, c4)
    q, Uk, Uv = R.operands(4, "bf16", 3, Hq, 2, 16)
    Q.check_outputs("bf16", Q.read_back(dar, c4), full, q, Uk, Uv, decode(c4, q, Uk, Uv))


@pytest.mark.parametrize("Hq", [2, 8, 16])
@pytest.mark.parametrize("where", ["key", "value"])
def test_nan_groups_stay_in_their_sequence(where, Hq):
    lens = [300, 300, 300]
    c, full = R.filled_cache(dar, 3, "bf16", 2, 16, 40, lens)
    (c.pool_kd if where == "key" else c.pool_vd)[full[1][2], 1, 5, 3] = math.inf
    c4 = Q.beside(dar, c)
    dar.dar_cache_pack_q4(c, c4)
    q, Uk, Uv = R.operands(4, "bf16", 3, Hq, 2, 16)
    got = decode(c4, q, Uk, Uv)
    bad = torch.zeros(got.shape[:2], dtype=torch.bool)
    bad[1, Hq // 2:] = True
    assert torch.equal(got.isnan().any(-1).cpu(), bad)
    assert got[1, Hq // 2:].isnan().all()


def test_errors():
    """Lengths and pages out of range are reported, and spoil no other sequence."""
    lens = [300, 300, 300, 300]
    c, full = R.filled_cache(dar, 2, "bf16", 2, 16, 8, lens)
    c4 = Q.beside(dar, c)
    dar.dar_cache_pack_q4(c, c4)
    q, Uk, Uv = R.operands(4, "bf16", 4, 8, 2, 16)
    want = decode(c4, q, Uk, Uv)
    table = c4.block_table.clone()
    for kind in ("long", "negative", "page", "minus"):
        c4.seq_lens.copy_(ints(lens))
        c4.block_table.copy_(table)
        c4.status.zero_()
        if kind == "long":
            c4.seq_lens[1] = c4.max_pages_per_seq * 64 + 9
        elif kind == "negative":
            c4.seq_lens[1] = -1
        else:
            c4.block_table[1] = c4.num_pages if kind == "page" else -1
        got = decode(c4, q, Uk, Uv)
        assert c4.device_status() == 3
        for b in (0, 2, 3):
            # (another length cuts the line of work elsewhere: the same up to the order of sums)
            assert (got[b].float() - want[b].float()).abs().max() <= 2.0 ** -7 * want[b].float().abs().max()


@pytest.mark.parametrize("n,per", [(1, None), (3, [3, 0, 1, 2]), (70, [70, 1, 64, 65])])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_step_equals_append_and_decode(dtype, n, per):
    lens, w, Hq = [300, 0, 39, 168], 40, 8
    c, full = R.filled_cache(dar, 2, dtype, 4, 16, w, [L + n for L in lens])
    c.seq_lens.copy_(ints(lens))
    a, b = (dar.DarCacheQ4(4, 4, 16, w, c.max_pages_per_seq, c.num_pages, dtype=c.dtype, block_table=c.block_table.cpu())
            for _ in range(2))
    for x in (a, b):
        x.pool.copy_(Q.beside(dar, c).pool)
        x.win_k.copy_(c.win_k)
        x.win_v.copy_(c.win_v)
        x.seq_lens.copy_(c.seq_lens)
        dar.dar_cache_pack_q4(c, x)
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn((4, 4, n, 64), device="cuda", generator=g).to(R.DT[dtype]) for _ in range(2))
    Dk, Dv = (torch.randn((4, 64, 16), device="cuda", generator=g) / 8 for _ in range(2))
    q, Uk, Uv = R.operands(4, dtype, 4, Hq, 4, 16)
    per_t = None if per is None else ints(per)
    dar.dar_cache_append_q4(a, k, v, Dk, Dv, n_per_seq=per_t)
    want = decode(a, q, Uk, Uv)
    got = dar.dar_decode_step_q4(b, k, v, Dk, Dv, q, Uk, Uv, dar.decode_q4_workspace(b, Hq), n_per_seq=per_t)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(a.pool, b.pool) and torch.equal(a.seq_lens, b.seq_lens)
    assert a.device_status() == 0 and b.device_status() == 0
    Q.check_outputs(dtype, Q.read_back(dar, b), full, q, Uk, Uv, got)


@pytest.mark.parametrize("dd", [8, 16, 32, 64])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (6, 3), (6, 2), (10, 2), (17, 1)])
def test_step_of_one_token(dd, Hq, Hkv):
    """Every width and number of heads, and units that leave warps of the first kernel over."""
    lens, w = [300, 0, 39, 168, 40], 40
    c, full = R.filled_cache(dar, 2, "bf16", Hkv, dd, w, [L + 1 for L in lens])
    c.seq_lens.copy_(ints(lens))
    a, b = (dar.DarCacheQ4(5, Hkv, dd, w, c.max_pages_per_seq, c.num_pages, block_table=c.block_table.cpu())
            for _ in range(2))
    for x in (a, b):
        x.pool.random_(0, 256)
        for t, u in ((x.win_k, c.win_k), (x.win_v, c.win_v), (x.seq_lens, c.seq_lens)):
            t.copy_(u)
        dar.dar_cache_pack_q4(c, x)
    b.pool.copy_(a.pool)
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn((5, Hkv, 1, 64), device="cuda", generator=g).bfloat16() for _ in range(2))
    Dk, Dv = (torch.randn((Hkv, 64, dd), device="cuda", generator=g) / 8 for _ in range(2))
    q, Uk, Uv = R.operands(4, "bf16", 5, Hq, Hkv, dd)
    dar.dar_cache_append_q4(a, k, v, Dk, Dv)
    want = decode(a, q, Uk, Uv)
    got = dar.dar_decode_step_q4(b, k, v, Dk, Dv, q, Uk, Uv, dar.decode_q4_workspace(b, Hq))
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(a.pool, b.pool) and torch.equal(a.seq_lens, b.seq_lens)
    assert a.device_status() == 0 and b.device_status() == 0
    Q.check_outputs("bf16", Q.read_back(dar, b), full, q, Uk, Uv, got)
