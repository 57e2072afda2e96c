"""How the cross attention's forward and dQ deal out their work, restated: a unit is 128 query rows of a key head, a step one of its key
tiles; either a workgroup has one unit, or all steps are cut into equal shares, one a workgroup."""
from paper_2509_01085_amd import binding as B

UNIT = 128


def rows_deal(s):
    """(shares?, workgroups, keys of a tile, units of an entry)"""
    bf16 = s.dtype == B.BF16
    tile = 64 if bf16 and s.d <= 128 else 32
    rows = s.Hkv * -(-(s.H // s.Hkv * s.Lq) // UNIT)
    units, tiles = rows * s.B, -(-s.S // tile)
    slots, worth, least = 512 if bf16 and s.d <= 128 else 256, 12 if bf16 else 4, 4 if bf16 else 1
    idle = (-units % slots) * tiles
    shares = units < (2 * slots if bf16 else slots // 2) and idle > worth * slots
    return shares, min(slots, max(1, units * tiles // least)) if shares else units, tile, rows


def pieces(s, lens):
    """The pieces of every workgroup in order: (entry, unit, first step, steps of the piece, steps of the unit)."""
    shares, grid, tile, rows = rows_deal(s)
    steps = [(b, u, -(-min(max(n, 0), s.S) // tile)) for b, n in enumerate(lens) for u in range(rows)]
    if not shares:
        return [[(b, u, 0, n, n)] for b, u, n in steps]
    per = -(-sum(n for *_, n in steps) // grid)
    out, room = [[]], per
    for b, u, n in steps:
        at = 0
        while at < n:
            if room == 0:
                out.append([])
                room = per
            k = min(room, n - at)
            out[-1].append((b, u, at, k, n))
            at, room = at + k, room - k
    return out


def short_units_behind_others(s, lens, steps=2):
    """Whole units of `steps` steps that are not their workgroup's first piece."""
    return sum(p[3] == p[4] == steps for w in pieces(s, lens) for p in w[1:])
