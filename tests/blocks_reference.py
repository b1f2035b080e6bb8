"""Counts, tables and pairs of tutti_blocks_fork, _free and _compact from their definitions, entry by entry.  Test infrastructure only."""
NONE = 0xffffffff
BAD_BLOCK, BAD_EXTENT, NO_FREE, BAD_USES = 1, 16, 64, 128


def fork(uses, table, records, max_entries, max_pairs):
    """records: (src_off, dst_off, n_shared, n_copied, n_new).  Changes uses and table; returns pairs and the status bits."""
    free = [b for b, u in enumerate(uses) if u == 0]
    before, status, pairs, number, over = list(table), 0, [], 0, False
    for src, dst, shared, copied, new in records:
        n = shared + copied + new
        if n > max_entries or dst + n > len(table) or (shared + copied and src + shared + copied > len(table)):
            status |= BAD_EXTENT
            continue
        over = over or len(pairs) + copied > max_pairs
        if over:
            status |= BAD_EXTENT
            continue
        for e in range(n):
            old = before[src + e] if e < shared + copied else None
            if old is not None and old >= len(uses):
                status |= BAD_BLOCK if old != NONE else 0
                old = NONE
            block = old
            if e >= shared:
                block = free[number] if number < len(free) else NONE
                if old == NONE:
                    block = NONE
                elif block == NONE:
                    status |= NO_FREE
                number += 1
                if old is not None:
                    pairs.append((old, block) if block != NONE else (NONE, NONE))
            table[dst + e] = block
            if block != NONE:
                uses[block] += 1
    return pairs, status


def free(uses, table, ranges, max_entries):
    status = 0
    for off, n in ranges:
        if n > max_entries or off + n > len(table):
            status |= BAD_EXTENT
            continue
        for e in range(off, off + n):
            b, table[e] = table[e], NONE
            if b == NONE:
                continue
            if b >= len(uses):
                status |= BAD_BLOCK
            elif uses[b] == 0:
                status |= BAD_USES
            else:
                uses[b] -= 1
    return status


def compact(uses, table, max_pairs):
    """Returns pairs, how many blocks are used, and the status bits."""
    n = sum(u != 0 for u in uses)
    holes = [b for b in range(n) if uses[b] == 0]
    movers = [b for b in range(len(uses) - 1, n - 1, -1) if uses[b] != 0]
    pairs = list(zip(movers, holes))[:max_pairs]
    to = dict(pairs)
    for a, b in pairs:
        uses[b], uses[a] = uses[a], 0
    status = 0
    for e, b in enumerate(table):
        if b >= len(uses):
            status |= BAD_BLOCK if b != NONE else 0
        else:
            table[e] = to.get(b, b)
    return pairs, n, status
