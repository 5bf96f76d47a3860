"""A model in whole numbers of the plan that plora_attn_plan makes of a step: its sets of
rows, how they are cut, and how many items and partial rows that takes."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                    "paper_2608_05483_amd", "csrc", "paged")
TEXT = "".join(open(os.path.join(CSRC, f)).read() for f in ("attn_plan.h", "attn_plan.hip"))


def constant(name):
    return int(re.search(rf"\b{name} = (\d+)[,;]", TEXT).group(1))


FEW, TILE, FEW_STEP, TILE_STEP = (constant(n) for n in ("kFew", "kTile", "kFewStep", "kTileStep"))
FEW_TARGET, TILE_TARGET = constant("kFewTarget"), constant("kTileTarget")
MIN_FEW, MIN_TILE = constant("kMinFew"), constant("kMinTile")
SLOTS, START = constant("kTileSlots"), constant("kTileStart")
TRY = [int(x) for x in re.search(r"kTry\[kTries\] = \{([^}]*)\}", TEXT).group(1).split(",")]
SHARE_ROWS, MAX_KEYS = 128, 1 << 30


def per_piece(work, target, kv_heads, least, step):
    c = min(max(-(-work // -(-target // kv_heads)), least), MAX_KEYS)
    return min(-(-c // step) * step, MAX_KEYS)


def cut(rows, keys, few_keys, tile_keys):
    """Tiles, pieces, keys of a piece."""
    few = rows <= FEW
    n = (keys - 1) // (few_keys if few else tile_keys) + 1
    step = FEW_STEP if few else TILE_STEP
    per = ((keys - 1) // n + step) // step * step
    return 1 if few else -(-rows // TILE), (keys - 1) // per + 1, per


def sets_of(past, new, r, page, group=None, prefix=()):
    """(rows, keys, whether its rows always leave partials): prefixes by group, then
    requests."""
    B = len(past)
    u, lead = [0] * B, []
    if group is not None:
        for g in sorted(set(int(x) for x in group if 0 <= x < len(prefix))):
            length = max(int(prefix[g]), 0) // page * page
            mem = [b for b in range(B) if group[b] == g and new[b] > 0 and length > 0 and
                   new[b] * r <= SHARE_ROWS and past[b] >= length]
            if len(mem) >= 2:
                for b in mem:
                    u[b] = length
                lead.append((sum(int(new[b]) for b in mem) * r, length, True))
    own = [(int(new[b]) * r, int(past[b] + new[b]) - u[b], u[b] > 0) for b in range(B)]
    return lead + [s for s in own if s[0] > 0]


def plan(sets, kv_heads):
    """few, tiles, part_rows, few_keys, tile_keys, later: the header's words."""
    tiles_of = lambda rows: 1 if rows <= FEW else -(-rows // TILE)
    work = [sum(tiles_of(n) * k for n, k, _ in sets if (n <= FEW) == f) for f in (True, False)]
    few_keys = per_piece(work[0], FEW_TARGET, kv_heads, MIN_FEW, FEW_STEP)
    tile_keys = MAX_KEYS
    if work[1]:
        best = None
        for t in TRY:
            per = per_piece(work[1], t, kv_heads, MIN_TILE, TILE_STEP)
            cuts = [cut(n, k, few_keys, per) for n, k, _ in sets if n > FEW]
            items = sum(a * b for a, b, _ in cuts)
            cost = -(-items * kv_heads // SLOTS) * (max(c for _, _, c in cuts) + START)
            if best is None or cost < best:
                best, tile_keys = cost, per
    few = tiles = later = parts = 0
    for rows, keys, always in sets:
        t, pieces, per = cut(rows, keys, few_keys, tile_keys)
        if rows > FEW:
            tiles += t * pieces
        elif pieces == 1 and per <= few_keys // 2:
            later += 1
        else:
            few += pieces
        parts += rows * pieces if always or pieces > 1 else 0
    return few, tiles, parts, few_keys, tile_keys, later
