"""How the segments kernels deal a bf16 call's stages to thread blocks, restated: which cuts a call has, so that a test
can say how far into a pipeline it goes.  (It says nothing about results.)"""


def cuts(Hq, Hkv, dd, w, lens, group=None, pages=None, grid=480):
    """[(kind, block, stages of the ring, stages of pages, pages they span)] of every cut; 480 blocks are the most."""
    G, ring, page = Hq // Hkv, 64, 4096 // dd  # tokens of a stage
    pages = list(pages or [])
    group = list(group) if group else [-1] * len(lens)
    group = [g if g >= 0 and pages[g] and max(0, n - w) >= 64 * pages[g] else -1 for g, n in zip(group, lens)]
    count = [group.count(g) for g in range(len(pages))]
    units, most = [], 4  # (kind, ring stages, page stages, cost of a stage)
    for g, n in enumerate(count):
        if n >= 2:
            rows = n * G
            cost = max(4, (min(rows, 64) + 7) // 8)
            most = max(most, cost)
            units += [("prefix", 0, -(-64 * pages[g] // page), cost)] * (Hkv * -(-rows // 64))
    for n, g in zip(lens, group):
        shared = 64 * pages[g] if g >= 0 and count[g] >= 2 else 0
        near = min(n, w)
        units += [("private", -(-near // ring), -(-(n - near - shared) // page), 4)] * (Hkv * -(-G // 64))
    starts, total = [], 0
    for _, a, b, cost in units:
        starts.append(total)
        total += 2 + (a + b) * cost if a + b else 0
    ctas = max(1, min(grid, total // most))
    out, u = [], 0
    for k in range(ctas):
        lo, hi = total * k // ctas, total * (k + 1) // ctas
        while u > 0 and starts[u] > lo:
            u -= 1
        while u < len(units) and starts[u] < hi:
            kind, a, b, cost = units[u]
            first = starts[u] + 2
            s0 = min(a + b, max(0, -(-(lo - first) // cost)))
            s1 = min(a + b, max(0, -(-(hi - first) // cost)))
            if s0 < s1:
                r = max(0, min(s1, a) - s0)
                out.append((kind, k, r, s1 - s0 - r, -(-(s1 - s0 - r) * page // 64)))
            u += 1
        u = min(u, len(units) - 1)
    assert sum(r + p for _, _, r, p, _ in out) == sum(a + b for _, a, b, _ in units)
    return out
