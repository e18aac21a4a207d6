"""How chunks of prompts are cut on the paged cache of 8-bit floating point, as the kernel cuts them: asked so that tests know what they reach."""


def sums(kv, gqa, rows, lengths, max_rows, n_rows, table_tokens):
    """(length of the line on which all blocks lie, workgroups) and of every unit (its place on the line, its length there, its tiles)."""
    tiles, n = table_tokens // 32, len(rows)
    most, length = max_rows * gqa, table_tokens // 32 + 16 + max_rows // 64
    blocks = -(-most // 256) * n
    if blocks * length * kv > 1 << 30:
        blocks = min(blocks, n_rows * gqa // 256 + n)
    groups = min(256, (blocks * length * kv // 16 + 8) & ~7)
    at, units = 0, []
    for r, held in zip(rows, lengths):
        held, blocks = min(held, table_tokens), -(-r * gqa // 256) if r * gqa > 64 else 0
        seen, growth = max(0, held - r) / 32, 256 / 64 / gqa
        place = [int(b * (b + 1) * growth + b * seen) + 8 * b for b in range(blocks + 1)]
        for _ in range(kv):
            for b in range(blocks):
                last = min(r * gqa, (b + 1) * 256) - 1
                units.append((at + place[b], place[b + 1] - place[b], -(-max(0, held - r + last // gqa + 1) // 32)))
            at += place[-1]
    return at, groups, units


def line(kv, gqa, rows, lengths, max_rows, table_tokens):
    """(tiles and leads of a workgroup's share, pieces that each unit is cut into, longest run of tiles that a workgroup has of one unit)."""
    total, groups, units = sums(kv, gqa, rows, lengths, max_rows, sum(rows), table_tokens)
    share = max(16, -(-total // groups))
    pieces = [(u + length - 1) // share - u // share + 1 for u, length, _ in units]
    return share, pieces, max(min(t, -(-share * t // length)) for _, length, t in units)
