"""Pages in 4 bits: conversion, appends, and what they leave alone."""
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


def same(a, b):
    """Equal numbers, NaN in the same places."""
    return torch.equal(a.double().nan_to_num(nan=1e300), b.double().nan_to_num(nan=1e300)) and \
        torch.equal(a.isnan(), b.isnan())


def vectors(c, full, b):
    kd, vd, _, _ = R.contents(c, full, b)
    return kd, vd


CONVERT = [
    ("bf16", 3, 16, 8, [0, 1, 8, 9, 71, 72, 73, 74, 200, 137]),
    ("bf16", 1, 8, 1, [66, 2, 300]),
    ("bf16", 2, 32, 40, [500, 39, 168]),
    ("bf16", 5, 64, 100, [1000, 101, 230]),
    ("f32", 2, 8, 30, [300, 159]),
    ("f32", 4, 16, 7, [72, 199, 8]),
    ("f32", 2, 32, 9, [500, 75]),
    ("f32", 1, 64, 3, [333, 4]),
]


@pytest.mark.parametrize("dtype,Hkv,dd,w,lens", CONVERT)
def test_pack_and_unpack(dtype, Hkv, dd, w, lens):
    c, full = R.filled_cache(dar, 5 + dd, dtype, Hkv, dd, w, lens)
    c4 = Q.beside(dar, c)
    dar.dar_cache_pack_q4(c, c4)
    back = Q.read_back(dar, c4)
    torch.cuda.synchronize()
    assert c4.device_status() == 0 and back.device_status() == 0
    touched = torch.zeros_like(back.pool_kd, dtype=torch.bool)
    for b, L in enumerate(lens):
        n = max(0, L - w)
        for x, y in zip(vectors(c, full, b), vectors(back, full, b)):
            assert same(y, Q.held(x.to(R.DT[dtype])))
        for i in range(-(-n // 64)):
            touched[full[b][i], :, :min(64, n - 64 * i)] = True
    assert back.pool_kd[~touched].isnan().all() and back.pool_vd[~touched].isnan().all()  # rows behind the last token
    # what was read back is held by the same bytes
    again = dar.DarCacheQ4.beside(back)
    again.pool.copy_(c4.pool)
    dar.dar_cache_pack_q4(back, again)
    assert torch.equal(again.pool, c4.pool)


@pytest.mark.parametrize("dtype,dd", [("bf16", 16), ("bf16", 8), ("f32", 16), ("f32", 64)])
def test_special_values(dtype, dd):
    """Zeros of both signs, ties, infinities, NaN, the largest and the smallest numbers; a group is on its own."""
    w, L = 4, 4 + 64
    c, full = R.filled_cache(dar, 1, dtype, 1, dd, w, [L])
    x = c.pool_kd[full[0][0], 0]
    n = min(16, dd)
    x[0] = 0.0
    x[1] = -0.0
    x[2, 0] = math.inf
    x[3, 1] = -math.inf
    x[4, 2] = math.nan
    x[5] = 0.0
    x[5, 3] = -7.0                                             # s = 1: ties between codes
    x[5, 4:8] = torch.tensor([0.5, 1.5, -2.5, -0.5])
    x[6] = torch.finfo(R.DT[dtype]).max * torch.linspace(-1, 1, dd)
    x[7] = torch.finfo(R.DT[dtype]).tiny * torch.linspace(-1, 1, dd)
    x[8] = torch.finfo(R.DT[dtype]).tiny * torch.linspace(-40, 40, dd)
    x[9] = 2.0 ** -133 * torch.arange(dd)                      # subnormal
    x[10] = 2.0 ** -133
    for e in range(32):                                        # maxima all around the borders of s
        x[11 + e, :n] = torch.linspace(-1, 1, n) * 7 * (1 + e / 32) * 2.0 ** (e - 16)
    c.pool_vd.copy_(c.pool_kd)
    c4 = Q.beside(dar, c)
    dar.dar_cache_pack_q4(c, c4)
    back = Q.read_back(dar, c4)
    for a, y in zip(vectors(c, full, 0), vectors(back, full, 0)):
        assert same(y, Q.held(a.to(R.DT[dtype])))


@pytest.mark.parametrize("dtype,dd", [("bf16", 16), ("bf16", 8), ("bf16", 64), ("f32", 32)])
@pytest.mark.parametrize("cut", [1, 2, 63, 64, 65, 129, 300, 10000])
def test_convert_from_a_position(dtype, dd, cut):
    """Only tokens from first[b] on are written, by either way; those before keep their bytes."""
    w, lens = 11, [411, 140, 11, 64 + 11 + 1]
    c, full = R.filled_cache(dar, 2, dtype, 2, dd, w, lens)
    c4, whole = Q.beside(dar, c, seed=3), Q.beside(dar, c, seed=3)
    dar.dar_cache_pack_q4(c, whole)
    early = c.pool_kd.clone(), c.pool_vd.clone()
    first = ints([cut] * 4)
    # in two parts: first the tokens before the cut (of contexts that end there), then the others
    c.seq_lens.copy_(ints([min(L, w + cut) for L in lens]))
    dar.dar_cache_pack_q4(c, c4)
    c.seq_lens.copy_(ints(lens))
    for b, L in enumerate(lens):
        for i in range(min(cut, max(0, L - w))):               # these must not be read again
            for t in (c.pool_kd, c.pool_vd):
                t[full[b][i // 64], :, i % 64] = math.nan
    dar.dar_cache_pack_q4(c, c4, first=first)
    assert torch.equal(c4.pool, whole.pool)
    back = dar.DarCache(c.B, 2, dd, w, c.max_pages_per_seq, c.num_pages, dtype=c.dtype, block_table=c.block_table.cpu())
    dar.dar_cache_unpack_q4(c4, back, first=first)
    c.pool_kd.copy_(early[0])
    c.pool_vd.copy_(early[1])
    for b, L in enumerate(lens):
        n = max(0, L - w)
        back.seq_lens[b] = L
        for x, y in zip(vectors(c, full, b), vectors(back, full, b)):
            assert not y[:, :min(n, cut)].any()
            assert same(y[:, cut:], Q.held(x.to(R.DT[dtype]))[:, cut:])
    assert c4.device_status() == 0 and back.device_status() == 0


def test_convert_errors():
    """Bad lengths, positions and pages are reported to dst, and leave the others alone."""
    lens = [300, 300, 300, 300]
    c, full = R.filled_cache(dar, 2, "bf16", 2, 16, 8, lens)
    want = Q.beside(dar, c)
    dar.dar_cache_pack_q4(c, want)
    for kind, code in (("long", 3), ("negative", 3), ("first", 1), ("page", 3), ("page4", 3)):
        c4 = dar.DarCacheQ4(4, 2, 16, 8, c.max_pages_per_seq, c.num_pages, block_table=c.block_table.cpu())
        c4.pool.copy_(Q.beside(dar, c).pool)
        before, first = c4.pool.clone(), None
        c.seq_lens.copy_(ints(lens))
        table = c.block_table.clone()
        if kind == "long":
            c.seq_lens[1] = c.max_pages_per_seq * 64 + 9
        elif kind == "negative":
            c.seq_lens[1] = -1
        elif kind == "first":
            first = ints([0, -1, 0, 0])
        elif kind == "page":
            c.block_table[1] = c.num_pages
        else:
            c4.block_table[1] = -1
        dar.dar_cache_pack_q4(c, c4, first=first)
        assert c4.device_status() == code and c.device_status() == 0
        expect = want.pool.clone()
        expect[full[1]] = before[full[1]]
        assert torch.equal(c4.pool, expect), kind
        c.block_table.copy_(table)
        if kind == "page4":
            c4.seq_lens.copy_(ints(lens))
            dar.dar_cache_unpack_q4(c4, c)
            assert c.device_status() == code
            c.status.zero_()


APPEND = [
    # dtype, Hkv, dd, w, lengths before, n, n_per_seq
    ("bf16", 2, 16, 8, [0, 5, 7, 8, 9, 70, 71, 72, 135, 136], 1, None),
    ("bf16", 2, 16, 8, [0, 5, 7, 8, 9, 70, 71, 72, 135, 136], 2, [0, 1, 2, 2, 1, 2, 1, 2, 2, 0]),
    ("bf16", 3, 16, 128, [100, 128, 191, 192, 193, 1000], 7, [7, 7, 1, 2, 3, 6]),
    ("bf16", 12, 16, 128, [4096, 4095], 8, None),
    ("bf16", 2, 16, 8, [0, 20, 75], 9, [9, 8, 3]),
    ("bf16", 2, 16, 37, [0, 20, 75, 64 + 37, 63 + 37], 200, [200, 131, 0, 64, 65]),
    ("bf16", 1, 16, 1, [0, 1, 2, 65], 130, [130, 1, 64, 129]),
    ("bf16", 2, 8, 20, [0, 19, 84, 300], 5, [5, 3, 1, 4]),
    ("bf16", 2, 8, 20, [0, 19, 84, 300], 100, [100, 3, 1, 77]),
    ("bf16", 20, 32, 20, [0, 19, 84, 300], 3, [3, 2, 1, 3]),
    ("bf16", 2, 32, 20, [0, 19, 84, 300], 150, [150, 3, 1, 77]),
    ("bf16", 16, 64, 20, [0, 19, 84, 300], 3, [3, 2, 1, 3]),
    ("bf16", 2, 64, 20, [0, 19, 84, 300], 300, [300, 3, 1, 77]),
    ("f32", 4, 16, 8, [0, 5, 7, 8, 9, 70, 71, 72], 2, [0, 1, 2, 2, 1, 2, 1, 2]),
    ("f32", 4, 16, 37, [0, 20, 75, 101], 150, [150, 131, 0, 64]),
    ("f32", 2, 8, 20, [0, 19, 84, 300], 5, [5, 3, 1, 4]),
    ("f32", 1, 8, 20, [0, 19, 84, 300], 99, [99, 3, 1, 77]),
    ("f32", 2, 32, 20, [0, 19, 84, 300], 33, [33, 3, 1, 7]),
    ("f32", 2, 64, 20, [0, 19, 84, 300], 77, [77, 3, 1, 77]),
    ("f32", 40, 64, 20, [0, 19, 84], 2, [2, 1, 2]),
]


def grown_pair(dtype, Hkv, dd, w, lens, n, seed):
    """An ordinary cache of these contexts with pages for n more tokens, and one in 4 bits with the same tokens."""
    c, full = R.filled_cache(dar, seed, dtype, Hkv, dd, w, [L + n for L in lens])
    c.seq_lens.copy_(ints(lens))
    c4 = dar.DarCacheQ4(len(lens), Hkv, dd, w, c.max_pages_per_seq, c.num_pages, dtype=c.dtype,
                        block_table=c.block_table.cpu())
    c4.pool.copy_(Q.beside(dar, c, seed).pool)
    for t, s in ((c4.win_k, c.win_k), (c4.win_v, c.win_v), (c4.seq_lens, c.seq_lens)):
        t.copy_(s)
    dar.dar_cache_pack_q4(c, c4)
    return c, c4, full


def new_tokens(dtype, B, Hkv, n, dd, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    k, v = (torch.randn((B, Hkv, n, 64), device="cuda", generator=g).to(R.DT[dtype]) for _ in range(2))
    Dk, Dv = (torch.randn((Hkv, 64, dd), device="cuda", generator=g) / 8 for _ in range(2))
    return k, v, Dk, Dv


@pytest.mark.parametrize("dtype,Hkv,dd,w,lens,n,per", APPEND)
def test_append(dtype, Hkv, dd, w, lens, n, per):
    """Rings, lengths and vectors are those of dar_cache_append; the vectors are held as pack holds them, and
    what was held before keeps its bytes."""
    c, c4, full = grown_pair(dtype, Hkv, dd, w, lens, n, 7)
    k, v, Dk, Dv = new_tokens(dtype, len(lens), Hkv, n, dd, 8)
    per_t = None if per is None else ints(per)
    before = ints([max(0, L - w) for L in lens])
    expect = dar.DarCacheQ4.beside(c)
    expect.pool.copy_(c4.pool)
    dar.dar_cache_append(c, k, v, Dk, Dv, n_per_seq=per_t)
    dar.dar_cache_pack_q4(c, expect, first=before)
    dar.dar_cache_append_q4(c4, k, v, Dk, Dv, n_per_seq=per_t)
    torch.cuda.synchronize()
    assert c4.device_status() == 0 and c.device_status() == 0
    assert torch.equal(c4.seq_lens, c.seq_lens)
    assert torch.equal(c4.pool, expect.pool)
    for a, b in ((c4.win_k, c.win_k), (c4.win_v, c.win_v)):
        assert same(a, b)


@pytest.mark.parametrize("dtype,Hkv,dd,w,B,n", [
    ("bf16", 2, 16, 8, 400, 8), ("bf16", 12, 16, 20, 70, 7), ("bf16", 8, 64, 5, 60, 8), ("bf16", 6, 8, 20, 260, 8),
    ("bf16", 5, 32, 1, 90, 5), ("bf16", 90, 16, 3, 33, 4), ("f32", 4, 16, 8, 200, 8), ("f32", 6, 8, 20, 260, 8),
    ("f32", 48, 8, 20, 100, 6), ("f32", 8, 64, 5, 60, 8),
])
def test_append_to_many(dtype, Hkv, dd, w, B, n):
    """Few tokens each to many sequences, at every place of a page and with 0 to n of them: as test_append."""
    test_append(dtype, Hkv, dd, w, [(7 * b) % 213 for b in range(B)], n, [(5 * b + b // 9) % (n + 1) for b in range(B)])


@pytest.mark.parametrize("dtype,dd", [("bf16", 16), ("bf16", 8), ("f32", 32)])
def test_append_in_pieces(dtype, dd):
    """However a run of tokens is cut into calls, the cache ends with the same bytes."""
    Hkv, w, B, total = 2, 13, 3, 230
    k, v, Dk, Dv = new_tokens(dtype, B, Hkv, total, dd, 4)
    got = []
    for pieces in ([230], [1] * 230, [9, 1, 64, 65, 3, 2, 30, 8, 48], [100, 130]):
        c4 = dar.DarCacheQ4(B, Hkv, dd, w, 4, dtype=R.DT[dtype])
        at = 0
        for n in pieces:
            dar.dar_cache_append_q4(c4, k[:, :, at:at + n].contiguous(), v[:, :, at:at + n].contiguous(), Dk, Dv)
            at += n
        assert c4.device_status() == 0 and c4.seq_lens.tolist() == [total] * B
        got.append((c4.pool.clone(), c4.win_k.clone(), c4.win_v.clone()))
    for x in got[1:]:
        for a, b in zip(got[0], x):
            assert torch.equal(a, b)


@pytest.mark.parametrize("n", [2, 70])
def test_append_errors(n):
    """Sequences that do not fit, or ask for what there is not, are refused and left as they are."""
    lens = [100, 100, 100, 100, 100]
    c, c4, full = grown_pair("bf16", 2, 16, 8, lens, 100, 3)
    k, v, Dk, Dv = new_tokens("bf16", 5, 2, n, 16, 8)
    c4.seq_lens.copy_(ints([100, c4.max_pages_per_seq * 64 + 8, -3, 100, 100]))
    per = ints([n, n, n, n + 1, -1])
    state = c4.pool.clone(), c4.win_k.clone()
    dar.dar_cache_append_q4(c4, k, v, Dk, Dv, n_per_seq=per)
    assert c4.device_status() in (1, 3)
    assert c4.seq_lens.tolist() == [100 + n, c4.max_pages_per_seq * 64 + 8, -3, 100, 100]
    for b in range(1, 5):
        assert torch.equal(c4.pool[full[b]], state[0][full[b]])
        assert same(c4.win_k[b], state[1][b])
    assert not torch.equal(c4.pool[full[0]], state[0][full[0]])
    # a page that the table does not name
    c4.status.zero_()
    c4.seq_lens.copy_(ints(lens))
    c4.block_table[2] = -1
    c4.block_table[3] = c4.num_pages
    before = c4.pool.clone()
    dar.dar_cache_append_q4(c4, k, v, Dk, Dv)
    assert c4.device_status() == 3
    for b in (2, 3):
        assert torch.equal(c4.pool[full[b]], before[full[b]])


def test_binding_refuses():
    c = dar.DarCache(2, 2, 16, 8, 4)
    c4 = dar.DarCacheQ4.beside(c)
    k, v, Dk, Dv = new_tokens("bf16", 2, 2, 3, 16, 1)
    with pytest.raises(ValueError):
        dar.dar_cache_append_q4(c4, k.float(), v, Dk, Dv)
    with pytest.raises(ValueError):
        dar.dar_cache_append_q4(c4, k, v[:, :, :2], Dk, Dv)
    with pytest.raises(ValueError):
        dar.dar_cache_append_q4(c4, k, v, Dk[:1], Dv)
    with pytest.raises(ValueError):
        dar.dar_cache_append_q4(c4, k, v, Dk, Dv, n_per_seq=torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError):
        dar.dar_cache_append_q4(c4, k.transpose(0, 1), v, Dk, Dv)
    with pytest.raises(ValueError):
        dar.dar_cache_pack_q4(c, c4, first=torch.zeros(3, dtype=torch.int32, device="cuda"))
    with pytest.raises(dar.DarError):
        dar.DarCacheQ4(2, 2, 12, 8, 4)
    q, Uk, Uv = R.operands(1, "bf16", 2, 4, 2, 16)
    ws = dar.decode_q4_workspace(c4, 4)
    with pytest.raises(ValueError):
        dar.dar_attn_decode_q4(c4, q[:1], Uk, Uv, ws)
    with pytest.raises(ValueError):
        dar.dar_attn_decode_q4(c4, q, Uk.cpu(), Uv, ws)
    with pytest.raises(dar.DarError):
        dar.dar_attn_decode_q4(c4, q, Uk, Uv, ws[:256])
    with pytest.raises(dar.DarError):
        dar.decode_q4_workspace(c4, 3)
