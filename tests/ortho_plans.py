"""Plans that between them launch every kernel of the orthogonalisation's tiles: (one half, matrices, tiles of G, B and X).

"256c": tiles of 256 x 256, some of whose sums are cut into parts that another launch joins.  test_ortho_launches_cpu.py sees
that they are launched as listed, test_gpu_ortho_tiles.py what they compute.  Most sides are no multiples of their tiles."""

BLOCKS = [(768, 2304)] * 12 + [(768, 768)] * 12 + [(768, 2048)] * 24 + [(2048, 768)] * 12
PLANS = [
    (False, [(40, 967)], "64c 64 64"),
    (False, [(967, 40), (70, 33)], "64c 64 64"),
    (False, [(600, 2425), (68, 4851)], "64c 64 64"),
    (False, [(642, 577)] * 12, "128 128 128"),
    (False, [(68, 4851)] * 5, "64c 64 128"),
    (False, [(4851, 70)] * 5, "64c 64 128"),
    (False, [(5092, 1554)], "64 64 128c"),
    (False, [(2999, 3001)], "128 128 128c"),
    (False, [(3001, 2950)], "128 128 128c"),
    (False, [(4090, 4001)], "128c 128c 256"),
    (False, [(4096, 4096)], "128c 128c 256"),
    (False, [(200, 16300)] * 3, "64c 64 256"),
    (False, [(16300, 200)] * 3, "64c 64 256"),
    (False, [(2040, 8190)], "256c 128 256"),
    (False, [(1530, 4090)] * 3, "128 128 256c"),
    (False, [(4090, 1500)] * 3, "128 128 256c"),
    (False, [(2990, 3001)] * 3, "256 256 256"),
    (False, [(4000, 4090)] * 2, "256c 256c 256"),
    (False, BLOCKS, "128 128 256c"),
    (True, [(64, 3000)], "64c 64 64"),
    (True, [(3000, 61)], "64c 64 64"),
    (True, [(91, 1436)] * 12, "64 64 128"),
    (True, [(1436, 91)] * 12, "64 64 128"),
    (True, [(536, 532)] * 12, "128 128 128"),
    (True, [(128, 16300)] * 3, "128c 64 128"),
    (True, [(16300, 120)] * 3, "128c 64 128"),
    (True, [(3376, 2523), (238, 52)], "128 128 128c"),
    (True, [(2523, 3376), (52, 238)], "128 128 128c"),
    (True, [(4090, 4001)], "128c 128c 256"),
    (True, [(190, 8190)] * 5, "64c 64 256"),
    (True, [(8190, 190)] * 5, "64c 64 256"),
    (True, [(2048, 8192)], "128 128 256"),
    (True, [(1530, 16300)], "256c 64 256"),
    (True, [(2040, 2001)] * 5, "256 256 128"),
    (True, [(2999, 3001)] * 2, "256 256 256c"),
    (True, [(3001, 2950)] * 2, "256 256 256c"),
    (True, [(4000, 4090)] * 2, "256c 256c 256"),
    (True, BLOCKS, "128 128 256"),
]


def name(plan):
    half, mats, tiles = plan
    return f"{'one' if half else 'two'}-{mats[0][0]}x{mats[0][1]}*{len(mats)}-{tiles.replace(' ', '-')}"


def layout(mats, odd):
    """[(offset, rows, cols, row stride)] and the vector's length: odd offsets, every other matrix (from the first on if `odd`) in
    rows that lie apart."""
    out, at = [], 3
    for k, (r, c) in enumerate(mats):
        ld = c + (5 if (k + odd) % 2 else 0)
        out.append((at, r, c, ld))
        at += r * ld + 2
    return out, at
