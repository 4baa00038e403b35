"""Steps of two to eight tokens a sequence, which append and make the queries' part in one kernel: as an append and a
decode."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)

from paper_2606_18587_gb300 import dar  # noqa: E402
from tests.helpers import q4_ref as Q  # noqa: E402
from tests.helpers import serving_ref as R  # noqa: E402

W = 40
# B, Hkv, query heads a KV head, d_down, tokens: enough sequences for that many (or two, which always are)
CASES = [
    (4, 4, 1, 16, 2), (4, 2, 3, 8, 2), (5, 1, 8, 64, 2), (64, 2, 2, 16, 3), (200, 4, 1, 16, 8), (260, 6, 2, 8, 8),
    (200, 2, 5, 64, 8), (90, 5, 4, 32, 5),
    (64, 20, 1, 16, 6),   # more chains than threads
    (64, 90, 1, 16, 7),   # fewer rows in shared memory than tokens
]


@pytest.mark.parametrize("B,Hkv,G,dd,n", CASES)
@pytest.mark.parametrize("ragged", [False, True])
def test_step(B, Hkv, G, dd, n, ragged):
    rounds = -(-2 * Hkv * dd // 512)
    assert n * rounds <= 2 + B * 2 * Hkv * dd // 4096  # what append_is_few asks for
    lens = [(300, 0, 39, 168, 40, 64 + W - 1, 37)[b % 7] for b in range(B)]
    per = [(n, 0, 1, n - 1, n)[b % 5] for b in range(B)] if ragged else None
    g = torch.Generator(device="cuda").manual_seed(1)
    maxp = -(-(300 + n - W) // 64)
    a, b = (dar.DarCacheQ4(B, Hkv, dd, W, maxp) for _ in range(2))
    a.pool.random_(0, 256, generator=g)
    kd, vd = (torch.empty((B * maxp, Hkv, 64, dd), device="cuda").normal_(generator=g).bfloat16() for _ in range(2))
    c = dar.DarCache(B, Hkv, dd, W, maxp)
    c.pool_kd.copy_(kd)
    c.pool_vd.copy_(vd)
    c.seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))
    dar.dar_cache_pack_q4(c, a)
    for t in (a.win_k, a.win_v):
        t.normal_(generator=g)
    a.seq_lens.copy_(c.seq_lens)
    for x, y in ((b.pool, a.pool), (b.win_k, a.win_k), (b.win_v, a.win_v), (b.seq_lens, a.seq_lens)):
        x.copy_(y)
    k, v = (torch.randn((B, Hkv, n, 64), device="cuda", generator=g).bfloat16() for _ in range(2))
    Dk, Dv = (torch.randn((Hkv, 64, dd), device="cuda", generator=g) / 8 for _ in range(2))
    q, Uk, Uv = R.operands(4, "bf16", B, G * Hkv, Hkv, dd)
    per_t = None if per is None else torch.tensor(per, dtype=torch.int32, device="cuda")
    ws = dar.decode_q4_workspace(a, G * Hkv)
    dar.dar_cache_append_q4(a, k, v, Dk, Dv, n_per_seq=per_t)
    want = dar.dar_attn_decode_q4(a, q, Uk, Uv, ws)
    got = dar.dar_decode_step_q4(b, k, v, Dk, Dv, q, Uk, Uv, ws, n_per_seq=per_t)
    assert torch.equal(got, want) and torch.equal(a.pool, b.pool) and torch.equal(a.seq_lens, b.seq_lens)
    assert torch.equal(a.win_k, b.win_k) and torch.equal(a.win_v, b.win_v)
    assert a.seq_lens.tolist() == [L + (n if per is None else per[i]) for i, L in enumerate(lens)]
    assert a.device_status() == 0 and b.device_status() == 0
    if B <= 5:
        Q.check_outputs("bf16", Q.read_back(dar, b), b.block_table.cpu().tolist(), q, Uk, Uv, got)
