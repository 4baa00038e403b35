"""dar_attn_decode_shared, dar_attn_decode_scored and dar_cache_evict refuse bad arguments on the host, with the
documented codes and without a launch; and a host model of how their work is cut up."""
import ctypes
import random

import pytest


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
             win_v=512, pool_kd=768, pool_vd=1024, block_table=1280, seq_lens=1536, status=1792)
    c.update(kw)
    return lib.dar_cache(*[c[f] for f, _ in lib.dar_cache._fields_])


P = 4096
BAD_CACHES = [(dict(d=32), 2), (dict(d_down=12), 2), (dict(w=0), 1), (dict(Hkv=0), 1), (dict(dtype=7), 1),
              (dict(win_k=0), 1), (dict(pool_kd=258), 1), (dict(B=5000), 2), (dict(block_table=0), 1)]


def test_shared_refuses(lib):
    L = lib.load_library()

    def call(c=None, Hq=4, q=P, group=P, n=1, pages=P, out=P, ws=P, wsb=1 << 40):
        return L.dar_attn_decode_shared(ctypes.byref(c or cache(lib)), Hq, q, P, P, group, n, pages, 0.0, out, ws, wsb,
                                        None)
    for kw, code in BAD_CACHES + [(dict(B=1025), 2)]:
        assert call(cache(lib, **kw)) == code
        assert L.dar_last_error().decode()
    assert call(Hq=3) == 1
    assert call(Hq=0) == 1
    assert call(q=0) == 1
    assert call(q=P + 8) == 1
    assert call(out=P + 2) == 1
    assert call(n=-1) == 1
    assert call(n=3) == 1            # more groups than sequences
    assert call(group=0) == 1
    assert call(pages=0) == 1
    assert call(wsb=1024) == 3
    assert "workspace" in L.dar_last_error().decode()
    assert call(cache(lib, num_pages=2 ** 31 - 1, Hkv=64), Hq=64) == 2   # 2^37 lines of pages
    assert call(cache(lib, w=2 ** 31 - 1)) == 2
    assert call(cache(lib, B=1024, Hkv=32, max_pages_per_seq=1 << 20), Hq=32) == 2
    assert call(cache(lib, B=0), n=0) == 0
    n = L.dar_decode_shared_workspace_bytes(ctypes.byref(cache(lib)), 4)
    assert n > 0 and n % 256 == 0
    assert L.dar_decode_shared_workspace_bytes(ctypes.byref(cache(lib)), 5) == 0


def test_scored_refuses(lib):
    L = lib.load_library()

    def call(c=None, Hq=4, q=P, weights=P, decay=1.0, ws=P, wsb=1 << 40):
        return L.dar_attn_decode_scored(ctypes.byref(c or cache(lib)), Hq, q, P, P, 0.0, weights, decay, P, ws, wsb,
                                        None)
    for kw, code in BAD_CACHES + [(dict(B=1025), 2)]:
        assert call(cache(lib, **kw)) == code
    assert call(Hq=3) == 1
    assert call(q=P + 4) == 1
    assert call(weights=0) == 1
    assert call(weights=P + 4) == 1
    for bad in (-0.1, 1.01, float("nan"), float("inf"), -float("inf")):
        assert call(decay=bad) == 1
        assert "decay" in L.dar_last_error().decode()
    assert call(ws=0) == 1
    assert call(wsb=1024) == 3
    assert call(Hq=2 * 1025) == 2
    assert call(cache(lib, B=0)) == 0
    # 4 bytes per query head and position, beside the partial results
    a, b = (L.dar_decode_scored_workspace_bytes(ctypes.byref(cache(lib, max_pages_per_seq=m)), 4) for m in (4, 1028))
    assert b - a == 2 * 4 * 1024 * 64 * 4


def test_the_joining_kernels_blocks_are_counted_as_they_are_launched(lib):
    """One per output row, and of a scored step one per 2048 positions of a head: 2^31 of them are too many.  (None of
    these calls gets as far as a launch: what comes after the count is refused.)"""
    L = lib.load_library()

    def scored(c, Hq):
        return L.dar_attn_decode_scored(ctypes.byref(c), Hq, P, P, P, 0.0, P, 2.0, P, P, 1 << 42, None)

    def shared(c, Hq):
        return L.dar_attn_decode_shared(ctypes.byref(c), Hq, P, P, P, P, -1, P, 0.0, P, P, 1 << 42, None)
    small = dict(d_down=8, w=1, max_pages_per_seq=1)  # capacity: 65 positions
    # 2095000 heads, of 1024 rows and a block of weights each: 2^31 - 108648
    assert scored(cache(lib, B=1000, Hkv=2095, **small), 2095 * 1024) == 1
    assert "decay" in L.dar_last_error().decode()
    assert scored(cache(lib, B=1024, Hkv=2046, **small), 2046 * 1024) == 1   # 2^31 - 2048
    assert scored(cache(lib, B=1024, Hkv=2047, **small), 2047 * 1024) == 2   # 2^31 + 2^20 - 1024
    assert "blocks" in L.dar_last_error().decode()
    assert shared(cache(lib, B=1024, Hkv=2046, **small), 2046 * 1024) == 1   # rows alone: 2^31 - 2^21
    assert shared(cache(lib, B=1024, Hkv=2048, **small), 2048 * 1024) == 2   # 2^31


def test_evict_refuses(lib):
    L = lib.load_library()

    def call(c=None, weights=P, keep=P, protect=None, ws=P, wsb=1 << 40):
        return L.dar_cache_evict(ctypes.byref(c or cache(lib)), weights, keep, protect, ws, wsb, None)
    for kw, code in BAD_CACHES:
        assert call(cache(lib, **kw)) == code
    assert call(weights=0) == 1
    assert call(weights=P + 8) == 1
    assert call(keep=0) == 1
    assert call(ws=0) == 1
    assert call(ws=P + 1) == 1
    assert call(wsb=256) == 3
    assert "workspace" in L.dar_last_error().decode()
    assert call(cache(lib, Hkv=1 << 28)) == 2
    assert call(cache(lib, B=0)) == 0
    n = L.dar_cache_evict_workspace_bytes(ctypes.byref(cache(lib)))
    assert n > 0 and n % 256 == 0
    assert L.dar_cache_evict_workspace_bytes(ctypes.byref(cache(lib, w=0))) == 0


def owner(p, total, ctas):
    return ((p + 1) * ctas - 1) // total


UNIT = 2  # length of a unit's set-up, before its stages


@pytest.mark.parametrize("seed", range(60))
def test_every_stage_has_one_cta_and_every_cut_one_slot(seed):
    """The line of units: stages are dealt to CTAs by their place, a unit's cut by CTA k has the slot unit + k, and the
    joining kernel's first and last CTA of a unit, and all between them, have a cut of it."""
    rng = random.Random(seed)
    costs = rng.choice(((4,), (4, 5, 7, 8, 16)))
    units = [(rng.choice((0, 1, 1, 2, 3, 17, 200)), rng.choice(costs)) for _ in range(rng.randint(1, 400))]
    if rng.random() < 0.2:
        units = [(rng.randint(1, 3000), 4)]
    length = [UNIT + n * c if n else 0 for n, c in units]
    total = sum(length)
    grid = rng.choice((1, 2, 152, 304, 456, 480))
    ctas = max(1, min(grid, total // max(costs)))
    starts, at = [], 0
    for n in length:
        starts.append(at)
        at += n
    slots, seen = set(), {}
    for k in range(ctas):
        lo, hi = total * k // ctas, total * (k + 1) // ctas
        for u, (n, c) in enumerate(units):
            if n == 0 or starts[u] + length[u] <= lo or starts[u] >= hi:
                continue
            p, first = max(lo, starts[u]), starts[u] + UNIT
            st0 = 0 if p <= first else -(-(p - first) // c)
            st1 = 0 if hi <= first else min(n, -(-(hi - first) // c))
            if st0 >= st1:
                continue
            assert u + k not in slots and u + k < len(units) + grid
            slots.add(u + k)
            for st in range(st0, st1):
                assert (u, st) not in seen
                seen[u, st] = k
    for u, (n, c) in enumerate(units):
        place = [starts[u] + UNIT + st * c for st in range(n)]
        for st in range(n):
            assert seen[u, st] == owner(place[st], total, ctas)
        if n:
            k0, k1 = owner(place[0], total, ctas), owner(place[-1], total, ctas)
            assert {seen[u, st] for st in range(n)} == set(range(k0, k1 + 1))


@pytest.mark.parametrize("seed", range(40))
def test_holes_and_movers_in_slices_pair_up_in_order(seed):
    """Each block of a cluster lists the holes and movers of its slice of the candidates; hole i and mover i of the
    cluster are found from the slices' counts, also where the slices are shorter than the cluster is long."""
    rng = random.Random(seed)
    C = rng.choice((1, 2, 4, 8))
    n = rng.choice((1, 2, 5, 9, 100, 1000))
    first = rng.randint(0, n - 1)
    keep = rng.randint(first, n - 1)
    w = [rng.choice((0.0, 1.0, 2.0, rng.random())) for _ in range(n)]
    cand, need = w[first:], keep - first
    order = sorted(range(len(cand)), key=lambda i: (-cand[i], i))
    stays = {first + i for i in order[:need]}
    last = cand[order[need - 1]] if need else None
    left = need - sum(x > last for x in cand) if need else 0
    m, sl = len(cand), -(-len(cand) // C)
    holes, movers, eq = [], [], 0
    for r in range(C):
        i0 = min(m, r * sl)
        h, mv = [], []
        for i in range(i0, min(m, i0 + sl)):
            same = need and cand[i] == last
            st = bool(need) and (cand[i] > last or (same and eq < left))
            eq += bool(same)
            assert st == (first + i in stays)
            if not st and first + i < keep:
                h.append(first + i)
            if st and first + i >= keep:
                mv.append(first + i)
        holes.append(h)
        movers.append(mv)
    hb, mb = [0], [0]
    for r in range(C):
        hb.append(hb[-1] + len(holes[r]))
        mb.append(mb[-1] + len(movers[r]))
    assert hb[-1] == mb[-1]
    flat_h, flat_m = sum(holes, []), sum(movers, [])
    for i in range(hb[-1]):
        qh = sum(i >= hb[q] for q in range(1, C))
        qm = sum(i >= mb[q] for q in range(1, C))
        assert holes[qh][i - hb[qh]] == flat_h[i] and movers[qm][i - mb[qm]] == flat_m[i]
        assert flat_h[i] < keep <= flat_m[i]
    # the ring turns by two reflections, each a set of disjoint swaps
    W, e = rng.randint(1, 50), rng.randint(0, 200)
    ring = list(range(W))
    want = [ring[(s + e) % W] for s in range(W)]
    for c in (0, W - e % W) if e % W else ():
        for s in range(W):
            o = c - s + (W if c < s else 0)
            assert 0 <= o < W
            if s < o:
                ring[s], ring[o] = ring[o], ring[s]
    assert ring == want
