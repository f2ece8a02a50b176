"""Calls of dash_paged4_attend whose tiles of 128 rows are cut in each of the ways that there are, and the dealing's rules as far as the host has them."""

# (head dimension, kv-heads, group, tokens of each sequence, new ones, way): `once` and `twice`: a sequence's items in as many parts each as there are places for, or twice
# that; `whole`: one item a CU stays whole, the others fill up; `fine`: more parts than places, of unequal items; `even`: as many as places; `none`: not cut
DEALS = [
    (128, 32, 1, [2000], [1100], "twice"), (64, 32, 1, [2300], [1600], "twice"), (128, 8, 4, [3500], [1100], "twice"),
    (128, 32, 1, [3900], [1400], "whole"), (64, 48, 1, [3900], [1400], "whole"),
    (128, 32, 1, [1300], [500], "once"), (64, 16, 2, [1500], [700], "once"),
    (128, 32, 1, [2000, 700, 40], [1100, 48, 1], "twice"), (64, 32, 1, [2300, 33], [1600, 9], "twice"),
    (128, 32, 1, [2100, 1900, 900, 30], [200, 200, 200, 20], "even"), (64, 16, 1, [1500, 1400, 1300], [300, 200, 300], "even"), (64, 32, 2, [2600, 60, 500, 1800], [100, 60, 200, 300], "fine"),
    (128, 32, 1, [1200, 1100], [1200, 900], "none"),
    # all resident, the later ones taken from the other end
    (128, 32, 1, [1200], [1200], "none"), (64, 32, 1, [2100], [2100], "none"), (128, 32, 1, [700, 1100, 20], [700, 650, 2], "none"),
]


def room(d, h_kv, g, lens, news):
    """parts at most, places, gain of the launch of 128-row tiles, and (tiles, cost) of every sequence that it has."""
    slots, tokens = max((512 if d == 128 else 768) // h_kv, 1), 128 // g
    rows = sum(news)
    most = min(rows // tokens + min(len(lens), rows), rows)
    wgs = slots if most < 2 * slots else 0
    if wgs and most * 4 >= slots:
        wgs = most + slots * 3 // 2
    few = 48 // g if len(lens) > 1 else 0
    seqs = [(-(-m // tokens) if m > few else 0, max((n + 63) // 64, 1)) for n, m in zip(lens, news)]
    return wgs, slots, 0.65 if rows * g < 64 * most else 0.9, seqs


def way(four, wgs, slots, cut, seqs):
    """Of a cut as the library makes it (size, whole, parts); see above."""
    size, whole, parts = cut
    items = sum(t for t, _ in seqs)
    if parts == items:
        return "none"
    if whole:
        return "whole"
    if four and items <= slots and len({c for t, c in seqs if t}) == 1:
        return "twice" if parts > slots else "once"
    return "fine" if parts > slots else "even"
