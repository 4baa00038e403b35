"""Samples of one prompt as a program serves them: the prompt enters one sequence, the others list its pages and copy
its ring; every step appends a token and attends over the shared prefix, every other one adds the attention weights;
when a sequence is over its budget it gives up what it attended to least, and serving goes on.  Each step against a
model in 64 bits that keeps the tokens by head."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)

from paper_2606_18587_gb300 import dar  # noqa: E402
from tests.helpers import serving_ref as R  # noqa: E402


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype,B,Hq,Hkv,dd,w,prompt,budget", [
    ("bf16", 3, 8, 2, 16, 24, 250, 215),
    ("bf16", 5, 2, 2, 32, 16, 209, 200),
    ("f32", 2, 4, 2, 8, 17, 150, 140),
])
def test_samples_of_a_prompt(dtype, B, Hq, Hkv, dd, w, prompt, budget):
    dt, steps, every = R.DT[dtype], 26, 5
    g = torch.Generator().manual_seed(B + dd)
    Dk, Dv = ((torch.randn((Hkv, 64, dd), generator=g) / 8).cuda() for _ in range(2))
    _, Uk, Uv = R.operands(3, dtype, B, Hq, Hkv, dd)
    P = (prompt - w) // 64
    maxp = (prompt + steps) // 64 + 2
    table = torch.full((B, maxp), -1, dtype=torch.int32)
    table[0] = torch.arange(maxp)
    for b in range(1, B):  # the prefix's pages are the first sequence's; the rest is each one's own
        table[b, :P] = table[0, :P]
        table[b, P:] = torch.arange(maxp - P) + maxp + (b - 1) * (maxp - P)
    c = dar.DarCache(B, Hkv, dd, w, maxp, int(table.max()) + 1, dtype=dt, block_table=table)
    k0, v0 = (torch.randn((B, Hkv, prompt, 64), generator=g).to(dt).cuda() for _ in range(2))
    dar.dar_cache_append(c, k0, v0, Dk, Dv, n_per_seq=ints([prompt] + [0] * (B - 1)))
    # the fork: ring, length and the pages that are not shared
    c.win_k[1:], c.win_v[1:] = c.win_k[0], c.win_v[0]
    c.seq_lens.fill_(prompt)
    for b in range(1, B):
        for p in range(P, maxp):
            for pool in (c.pool_kd, c.pool_vd):
                pool[table[b, p].item()] = pool[table[0, p].item()]
    down = [dar.dar_down_project(x[:1].contiguous(), D).cpu().double()[0] for x, D in ((k0, Dk), (v0, Dv))]
    n0 = prompt - w
    dist = [[[x[h, :n0].clone() for x in down] for h in range(Hkv)] for _ in range(B)]
    near = [[[x[0, h, n0:].cpu().double() for x in (k0, v0)] for h in range(Hkv)] for _ in range(B)]
    totals = [[[0.0] * prompt for _ in range(Hkv)] for _ in range(B)]

    weights, ws = dar.attention_weights(c), dar.shared_decode_workspace(c, Hq)
    wsc, we = dar.scored_decode_workspace(c, Hq), dar.evict_workspace(c)
    group, pages = ints([0] * B), ints([P])
    keep, protect = ints([budget] * B), ints([64 * P] * B)
    for step in range(steps):
        k1, v1 = (torch.randn((B, Hkv, 1, 64), generator=g).to(dt).cuda() for _ in range(2))
        q = (torch.randn((B, Hq, 64), generator=g) * 1.5).to(dt).cuda()
        leave = [[near[b][h][i][0].to(dt) for i in range(2)] for b in range(B) for h in range(Hkv)]
        left = [torch.stack([r[i] for r in leave]).view(B, Hkv, 1, 64).cuda() for i in range(2)]
        left = [dar.dar_down_project(x, D).cpu().double() for x, D in zip(left, (Dk, Dv))]
        dar.dar_cache_append(c, k1, v1, Dk, Dv)
        for b in range(B):
            for h in range(Hkv):
                for i, x in enumerate((k1, v1)):
                    dist[b][h][i] = torch.cat((dist[b][h][i], left[i][b, h]))
                    near[b][h][i] = torch.cat((near[b][h][i][1:], x[b, h].cpu().double()))
                totals[b][h].append(0.0)
        outs = [dar.dar_attn_decode_shared(c, q, Uk, Uv, group, pages, ws)]
        if step % 2:
            outs.append(dar.dar_attn_decode_scored(c, q, Uk, Uv, weights, wsc))
        outs.append(dar.dar_attn_decode(c, q, Uk, Uv, dar.decode_workspace(c, Hq)))
        torch.cuda.synchronize()
        assert c.device_status() == 0
        got = weights.cpu().double()
        for b in range(B):
            kd, vd, kk, vv = (torch.stack([src[b][h][i] for h in range(Hkv)]) for src, i in
                              ((dist, 0), (dist, 1), (near, 0), (near, 1)))
            assert int(c.seq_lens[b]) == kd.shape[1] + kk.shape[1]
            out, p, mag, top = R.attend(q[b].cpu().double(), kd, vd, kk, vv, Uk.cpu().double(), Uv.cpu().double())
            tol = R.tolerances(dtype, out, mag, top)
            for y in outs[:-1]:
                assert ((y[b].cpu().double() - out).abs() <= tol).all(), (step, b)
            if step % 2:
                p = p.view(Hkv, Hq // Hkv, -1).sum(1)
                for h in range(Hkv):
                    old = torch.tensor(totals[b][h], dtype=torch.float64)
                    new = got[b, h, :len(old)]
                    assert ((new - old - p[h]).abs() <= R.weight_tolerance(p[h], old, top)).all(), (step, b, h)
                    totals[b][h] = new.tolist()
                    assert not got[b, h, len(old):].any()
        # the unshared step of the library, which rounds the absorbed query where these two do not
        assert (outs[0].double() - outs[-1].double()).abs().max() <= (2e-2 if dtype == "bf16" else 1e-5)
        if step % every == every - 1:
            dar.dar_cache_evict(c, weights, keep, we, protect=protect)
            torch.cuda.synchronize()
            assert c.device_status() == 0
            for b in range(B):
                for h in range(Hkv):
                    kd, vd, _, _, t = R.evict(*dist[b][h], *near[b][h], totals[b][h], budget, 64 * P, w)
                    dist[b][h] = [kd[:budget], vd[:budget]]  # (the rows behind are nobody's any more)
                    totals[b][h] = t[:dist[b][h][0].shape[0] + w]
    assert int(c.seq_lens.max()) <= budget + w + every
