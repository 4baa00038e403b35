"""The operators of the cache in 4 bits together, as a serving program uses them."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)

from paper_2606_18587_gb300 import dar  # noqa: E402
from tests.helpers import q4_ref as Q  # noqa: E402
from tests.helpers import serving_ref as R  # noqa: E402

Hq, Hkv, dd, w = 8, 2, 16, 48


def weights(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    Dk, Dv = (torch.randn((Hkv, 64, dd), device="cuda", generator=g) / 8 for _ in range(2))
    Uk, Uv = (torch.randn((Hkv, dd, 64), device="cuda", generator=g) / 4 for _ in range(2))
    return g, Dk, Dv, Uk, Uv


def tokens(g, B, n):
    return [torch.randn((B, h, n, 64), device="cuda", generator=g).bfloat16() for h in (Hq, Hkv, Hkv)]


def test_prompt_chat_and_resume():
    """A prompt enters an ordinary cache chunk by chunk, each packed as it is done; the chat goes on in 4 bits; its
    context is read back, and the next prompt is processed over it."""
    B = 3
    g, Dk, Dv, Uk, Uv = weights(1)
    c = dar.DarCache(B, Hkv, dd, w, 12)
    c4 = dar.DarCacheQ4.beside(c)
    full = c.block_table.cpu().tolist()
    done = torch.zeros(B, dtype=torch.int32, device="cuda")
    for n in (100, 77, 130):
        q, k, v = tokens(g, B, n)
        dar.dar_prefill_chunk(c, q, k, v, Dk, Uk, Dv, Uv)
        dar.dar_cache_pack_q4(c, c4, first=done)
        done.copy_((c.seq_lens - w).clamp(min=0))
    whole = dar.DarCacheQ4.beside(c)
    dar.dar_cache_pack_q4(c, whole)
    assert torch.equal(whole.pool, c4.pool)
    ws = dar.decode_q4_workspace(c4, Hq)
    # beside the chat, the ordinary cache of the same values takes the same steps: appended tokens leave the window
    # into it as they are, and are given the values of 4 bits then
    mirror = Q.read_back(dar, c4)
    for i in range(70):
        q, k, v = tokens(g, B, 1)
        q = q[:, :, 0].contiguous()
        out = dar.dar_decode_step_q4(c4, k, v, Dk, Dv, q, Uk, Uv, ws)
        dar.dar_cache_append(mirror, k, v, Dk, Dv)
        if i % 23 == 0 or i == 69:
            dar.dar_cache_unpack_q4(c4, mirror)
            Q.check_outputs("bf16", mirror, full, q, Uk, Uv, out)
    assert torch.equal(c4.win_k, mirror.win_k) and torch.equal(c4.seq_lens, mirror.seq_lens)
    # resumed: the ordinary cache has the ring and the lengths already
    dar.dar_cache_unpack_q4(c4, c)
    for b in range(B):
        for x, y in zip(R.contents(c, full, b), R.contents(mirror, full, b)):
            assert torch.equal(x, y)
    q, k, v = tokens(g, B, 65)
    a = dar.dar_prefill_chunk(c, q, k, v, Dk, Uk, Dv, Uv)
    m = dar.dar_prefill_chunk(mirror, q, k, v, Dk, Uk, Dv, Uv)
    assert torch.equal(a, m)
    assert c.device_status() == 0 and mirror.device_status() == 0


def test_captured_steps():
    """A step captured once and replayed follows the lengths on the device; two graphs share a workspace in turn."""
    B = 2
    g, Dk, Dv, Uk, Uv = weights(2)
    caches = [dar.DarCacheQ4(B, Hkv, dd, w, 6) for _ in range(3)]
    _, k0, v0 = tokens(g, B, 150)
    for c in caches:
        dar.dar_cache_append_q4(c, k0, v0, Dk, Dv)
    ws = dar.decode_q4_workspace(caches[0], Hq)
    q, k, v = tokens(g, B, 1)
    q = q[:, :, 0].contiguous()
    outs = [torch.empty_like(q) for _ in caches]
    graphs = []
    stream = torch.cuda.Stream()
    for i in (0, 1):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.stream(stream), torch.cuda.graph(graph, stream=stream):
            dar.dar_decode_step_q4(caches[i], k, v, Dk, Dv, q, Uk, Uv, ws, out=outs[i])
        graphs.append(graph)
    torch.cuda.synchronize()
    assert caches[0].seq_lens.tolist() == [150] * B  # captured, not run
    for i in range(40):
        qi, ki, vi = tokens(g, B, 1)
        q.copy_(qi[:, :, 0])
        k.copy_(ki)
        v.copy_(vi)
        for graph in graphs:
            graph.replay()
        dar.dar_decode_step_q4(caches[2], k, v, Dk, Dv, q, Uk, Uv, ws, out=outs[2])
        assert torch.equal(outs[0], outs[2]) and torch.equal(outs[1], outs[2]), i
    assert torch.equal(caches[0].pool, caches[2].pool)
    assert all(c.device_status() == 0 for c in caches)


def test_two_streams():
    """Two batches on two streams, each with a workspace of its own."""
    g, Dk, Dv, Uk, Uv = weights(3)
    runs = []
    for n in (900, 333):
        c = dar.DarCacheQ4(4, Hkv, dd, w, 20)
        _, k, v = tokens(g, 4, n)
        dar.dar_cache_append_q4(c, k, v, Dk, Dv)
        q = tokens(g, 4, 1)[0][:, :, 0].contiguous()
        runs.append((c, q, dar.decode_q4_workspace(c, Hq), torch.empty_like(q), torch.cuda.Stream()))
    want = [dar.dar_attn_decode_q4(c, q, Uk, Uv, ws) for c, q, ws, _, _ in runs]
    torch.cuda.synchronize()
    for _ in range(20):
        for c, q, ws, out, s in runs:
            dar.dar_attn_decode_q4(c, q, Uk, Uv, ws, out=out, stream=s)
    torch.cuda.synchronize()
    for (_, _, _, out, _), x in zip(runs, want):
        assert torch.equal(out, x)


def test_largest_batch():
    """DAR_DECODE_MAX_BATCH sequences of a few tokens, half of them empty."""
    B = 1024
    g, Dk, Dv, Uk, Uv = weights(4)
    c4 = dar.DarCacheQ4(B, Hkv, dd, 8, 2)
    _, k, v = tokens(g, B, 70)
    per = (torch.arange(B, device="cuda", dtype=torch.int32) % 71) * (torch.arange(B, device="cuda", dtype=torch.int32) % 2)
    dar.dar_cache_append_q4(c4, k, v, Dk, Dv, n_per_seq=per)
    q = tokens(g, B, 1)[0][:, :, 0].contiguous()
    out = dar.dar_attn_decode_q4(c4, q, Uk, Uv, dar.decode_q4_workspace(c4, Hq))
    assert c4.device_status() == 0
    c = Q.read_back(dar, c4)
    Q.check_outputs("bf16", c, c.block_table.cpu().tolist(), q, Uk, Uv, out)
