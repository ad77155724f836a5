"""The plan of an attention call over pages, as the host and the kernel make it: rows of a tile, and how the work is dealt
out.  Tests name the path that they take with it."""
import paper_2606_20537_amd as cap

UNIT = 32
BEGIN = {64: 10, 128: 8, 256: 6}  # units that the beginning of a segment counts for


def places(d, tile):
    return 768 if d == 64 and tile > 16 else 65536 // d


def plan(d, Hkv, G, page, columns, n, T, window=0):
    """(rows of a tile, "whole" / "parts" / "runs", workgroups, units of a part): segments are not cut, or each into even
    parts, or the units of all are dealt out in equal runs."""
    capacity, tokens, n_seq = columns * page, sum(T), len(n)
    rows, seen = tokens * G, min(capacity, window + tokens) if window else capacity
    whole = seen <= (1024 if n_seq * Hkv >= places(d, 16) else {64: 768, 128: 512, 256: 256}[d])

    def fills(tile, units):
        segments = max(n_seq, rows // tile) * Hkv
        return segments >= places(d, tile) or segments * (seen // UNIT) >= units * places(d, tile)

    tile = 128 if rows > {64: 96, 128: 64, 256: 32}[d] * n_seq and fills(128, 6) else 32 if rows > 16 * n_seq and fills(32, 8) else 16
    units = min(-(-capacity // UNIT), seen // UNIT + 2) + BEGIN[d]
    most = (rows // tile + n_seq) * Hkv * (1 if whole else units)
    wgs = min(most, places(d, tile))
    if whole:
        return tile, "whole", wgs, 0
    segments = all_units = 0
    for m, t in zip(n, T):
        if t:
            lo = max(0, m - t + 1 - window) if window else 0
            of = -(-t * G // tile) * Hkv
            segments += of
            all_units += of * max(1, -(-min(m, capacity) // UNIT) - lo // UNIT)
    if segments < wgs and all_units < 33 * wgs:
        cut = max(4, all_units // (wgs - segments) + 1)
        if cut <= 32:
            return tile, "parts", wgs, cut
    return tile, "runs", wgs, 0


def plan_of(step, G, window=0):
    """That of a Step's call; its tile is what the workspace says."""
    p = plan(step.d, step.Hkv, G, step.page, step.table.shape[1], step.n, step.T, window)
    heads = step.Hkv * G
    has = cap.kvp_attend_workspace_bytes(step.cache, step.tokens, heads, window)
    assert has == (0 if p[1] == "whole" else p[2] * 2 * p[0] * (step.d + 2) * 4 + step.tokens * heads * 8)
    return p
