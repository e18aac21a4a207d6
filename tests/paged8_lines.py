"""How chunks of prompts are cut on the paged cache of 8-bit floating point, as the kernel cuts them: asked so that tests know what they reach."""


def line(kv, gqa, rows, lengths, max_rows, table_tokens):
    """(tiles and leads of a workgroup's share, pieces that each unit is cut into, longest run of tiles that a workgroup has of one unit)."""
    heads, tiles = len(rows) * kv, table_tokens // 32
    most = max_rows * gqa
    groups = min(256, (-(-most // 256) * (tiles + 8 + max_rows // 32) * heads // 16 + 8) & ~7)
    at, units = 0, []
    for r, n in zip(rows, lengths):
        n, blocks = min(n, table_tokens), -(-r * gqa // 256) if r * gqa > 64 else 0
        seen, growth = max(0, n - r) / 32, 256 / 64 / gqa
        place = [int(b * (b + 1) * growth + b * seen) + 8 * b for b in range(blocks + 1)]
        for _ in range(kv):
            for b in range(blocks):
                last = min(r * gqa, (b + 1) * 256) - 1
                units.append((at + place[b], place[b + 1] - place[b], -(-max(0, n - r + last // gqa + 1) // 32)))
            at += place[-1]
    share = max(16, -(-at // groups))
    pieces = [(u + length - 1) // share - u // share + 1 for u, length, _ in units]
    return share, pieces, max(min(t, -(-share * t // length)) for _, length, t in units)
