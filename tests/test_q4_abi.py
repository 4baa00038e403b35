"""The entry points of the cache in 4 bits refuse bad arguments on the host, with the documented codes and without a
launch; sizes of pages and workspaces; the definition of what a page holds."""
import ctypes
import math

import pytest

torch = pytest.importorskip("torch")

from tests.helpers import q4_ref  # noqa: E402


@pytest.fixture(scope="module")
def lib():
    from paper_2606_18587_gb300 import dar
    try:
        dar.load_library()
    except RuntimeError:
        from paper_2606_18587_gb300 import build
        build.build()
    return dar


def cache(lib, **kw):
    c = dict(dtype=lib.DAR_BF16, B=2, Hkv=2, d=64, d_down=16, w=8, max_pages_per_seq=4, num_pages=8, win_k=256,
             win_v=512, pool=768, block_table=1280, seq_lens=1536, status=1792)
    c.update(kw)
    return lib.dar_cache_q4(*[c[f] for f, _ in lib.dar_cache_q4._fields_])


def plain(lib, **kw):
    c = dict(dtype=lib.DAR_BF16, B=2, Hkv=2, d=64, d_down=16, w=8, max_pages_per_seq=4, num_pages=8, win_k=256,
             win_v=512, pool_kd=768, pool_vd=1024, block_table=1280, seq_lens=1536, status=1792)
    c.update(kw)
    return lib.dar_cache(*[c[f] for f, _ in lib.dar_cache._fields_])


P = 4096
BAD = [(dict(d=32), 2), (dict(d_down=12), 2), (dict(w=0), 1), (dict(Hkv=0), 1), (dict(dtype=7), 1), (dict(win_k=0), 1),
       (dict(pool=258), 1), (dict(pool=0), 1), (dict(B=5000), 2), (dict(B=-1), 1), (dict(block_table=0), 1),
       (dict(seq_lens=0), 1), (dict(status=0), 1), (dict(num_pages=0), 1)]


def test_page_bytes(lib):
    """Codes of 4 bits and a 16-bit scale for each group, keys and values."""
    for dd in (8, 16, 32, 64):
        assert lib.dar_q4_page_bytes(dd) == 2 * 64 * (dd // 2 + 2 * max(1, dd // 16))
        assert lib.dar_q4_page_bytes(dd) % 256 == 0
    assert [lib.dar_q4_page_bytes(dd) for dd in (0, -8, 12, 24, 128)] == [0] * 5


def test_append_refuses(lib):
    L = lib.load_library()

    def call(c=None, k=P, n=4, per=None, Dk=P):
        return L.dar_cache_append_q4(ctypes.byref(c or cache(lib)), k, P, n, per, Dk, P, None)
    for kw, code in BAD:
        assert call(cache(lib, **kw)) == code
        assert L.dar_last_error().decode()
    assert L.dar_cache_append_q4(None, P, P, 1, None, P, P, None) == 1
    assert call(n=-1) == 1
    assert call(k=0) == 1
    assert call(k=P + 2) == 1
    assert call(Dk=P + 4) == 1
    assert call(Dk=0) == 1
    assert call(cache(lib, B=4096, Hkv=64), n=2 ** 31 - 1) == 2   # more blocks than a grid has
    assert call(n=0) == 0
    assert call(cache(lib, B=0)) == 0
    assert L.dar_last_error().decode() == ""


def test_convert_refuses(lib):
    L = lib.load_library()

    def pack(t=None, c=None):
        return L.dar_cache_pack_q4(ctypes.byref(t or plain(lib)), None, ctypes.byref(c or cache(lib)), None)

    def unpack(t=None, c=None):
        return L.dar_cache_unpack_q4(ctypes.byref(c or cache(lib)), None, ctypes.byref(t or plain(lib)), None)
    for call in (pack, unpack):
        for kw, code in BAD:
            assert call(c=cache(lib, **kw)) == code
        assert call(t=plain(lib, d_down=12)) == 2
        assert call(t=plain(lib, pool_kd=0)) == 1
        for kw in (dict(B=3), dict(Hkv=4), dict(d_down=32), dict(w=9), dict(dtype=lib.DAR_F32)):
            assert call(t=plain(lib, **kw)) == 1
            assert "differ" in L.dar_last_error().decode()
        big = dict(max_pages_per_seq=2 ** 30, Hkv=2)
        assert call(plain(lib, **big), cache(lib, **big)) == 2
        assert call(plain(lib, B=0), cache(lib, B=0)) == 0
    assert L.dar_cache_pack_q4(None, None, ctypes.byref(cache(lib)), None) == 1
    assert L.dar_cache_pack_q4(ctypes.byref(plain(lib)), None, None, None) == 1
    assert L.dar_cache_unpack_q4(None, None, ctypes.byref(plain(lib)), None) == 1


def test_convert_refuses_a_batch_beyond_a_grid(lib):
    L, big = lib.load_library(), dict(B=65536)
    t, c = plain(lib, **big), cache(lib, **big)
    assert L.dar_cache_pack_q4(ctypes.byref(t), None, ctypes.byref(c), None) == 2
    assert L.dar_cache_unpack_q4(ctypes.byref(c), None, ctypes.byref(t), None) == 2


def test_decode_refuses(lib):
    L = lib.load_library()

    def call(c=None, Hq=4, q=P, Uk=P, out=P, ws=P, wsb=1 << 40):
        return L.dar_attn_decode_q4(ctypes.byref(c or cache(lib)), Hq, q, Uk, P, 0.0, out, ws, wsb, None)

    def step(c=None, Hq=4, n=1, k=P, q=P, wsb=1 << 40):
        return L.dar_decode_step_q4(ctypes.byref(c or cache(lib)), k, P, n, None, P, P, Hq, q, P, P, 0.0, P, P, wsb, None)
    for f in (call, step):
        for kw, code in BAD + [(dict(B=1025), 2)]:
            assert f(cache(lib, **kw)) == code
            assert L.dar_last_error().decode()
        assert f(Hq=3) == 1
        assert f(Hq=0) == 1
        assert f(q=0) == 1
        assert f(q=P + 8) == 1
        assert f(wsb=256) == 3
        assert "workspace" in L.dar_last_error().decode()
        assert f(cache(lib, w=2 ** 31 - 1)) == 2
        assert f(cache(lib, B=1024, Hkv=32, max_pages_per_seq=1 << 20), Hq=32) == 2
        assert f(cache(lib, B=0)) == 0
        assert f(cache(lib, B=1, Hkv=1 << 21, w=1, max_pages_per_seq=0), Hq=1 << 21) == 2   # 2.7 GB a page
    assert call(Uk=0) == 1
    assert call(Uk=P + 4) == 1
    assert call(out=P + 2) == 1
    assert call(ws=P + 8) == 1
    assert step(n=-1) == 1
    assert step(k=0) == 1
    n = L.dar_decode_q4_workspace_bytes(ctypes.byref(cache(lib)), 4)
    assert n > 0 and n % 256 == 0
    assert L.dar_decode_q4_workspace_bytes(ctypes.byref(cache(lib)), 5) == 0
    assert L.dar_decode_q4_workspace_bytes(ctypes.byref(cache(lib, w=0)), 4) == 0
    # independent of the capacity
    assert L.dar_decode_q4_workspace_bytes(ctypes.byref(cache(lib, max_pages_per_seq=4096)), 4) == n


@pytest.mark.parametrize("dd", [8, 16, 64])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_held_values(dd, dtype):
    """The definition itself: values are bf16 numbers within half a step, and held again by the same codes."""
    x = (torch.randn((300, dd), generator=torch.Generator().manual_seed(dd)) * torch.logspace(-30, 30, 300)[:, None]).to(dtype)
    v = q4_ref.held(x)
    assert torch.equal(v, v.to(torch.bfloat16).double())
    assert torch.equal(q4_ref.held(v.to(dtype)), v)
    a = x.double().unflatten(-1, (max(1, dd // 16), -1)).abs().amax(-1, keepdim=True)
    err = (v - x.double()).abs().unflatten(-1, (max(1, dd // 16), -1))
    # half a step, and the maximum lies at most 7 (1 + 2^-5) steps up, whose code is 7
    assert (err <= a / 7 * (1 + 2.0 ** -5) / 2 * (1 + 1e-12)).all()
    one = torch.zeros((4, dd), dtype=dtype)
    one[1, 0], one[2, 0], one[3, 0] = 3.0, math.inf, math.nan
    v = q4_ref.held(one)
    assert not v[0].any() and v[1, 0] != 0 and not v[1, 1:].any()
    n = min(dd, 16)
    assert v[2:, :n].isnan().all() and not v[2:, n:].any()
