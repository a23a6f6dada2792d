"""Oracle of the page tables that follow their sequences' lengths: plain Python, one sequence and one page after the other."""


def resize(table, lengths, ring, at, page_size, wanted, rows=None):
    """Changes table (list of lists), lengths, ring and at ([first, how many]) in place; returns (row offsets, positions, slots) of the new
    positions. rows: how many of them there may be (None: any number)."""
    n, width = len(ring), len(table[0])
    first, free = at[0] % n, min(max(at[1], 0), n)
    pages_of = lambda positions: -(-positions // page_size)
    taken = given = listed = 0
    open_ = True                                   # until the first sequence that does not fit
    off, positions, slots = [0], [], []
    gone = []
    for b, want in enumerate(wanted):
        old = min(max(lengths[b], 0), width * page_size)
        new = want if 0 <= want <= width * page_size else old
        if new > old:
            need = pages_of(new) - pages_of(old)
            if not open_ or need > free - taken or (rows is not None and new - old > rows - listed):
                open_, new = False, old
            for j in range(pages_of(old), pages_of(new)):
                table[b][j] = ring[(first + taken) % n]
                taken += 1
            for p in range(old, new):
                page = table[b][p // page_size]
                positions.append(p)
                slots.append(page * page_size + p % page_size if 0 <= page < n else -1)
            listed += new - old
        for j in range(pages_of(new), pages_of(old)):
            if 0 <= table[b][j] < n:
                gone.append(table[b][j])
            table[b][j] = -1
        lengths[b] = new
        off.append(listed)
    for page in gone:
        if given < n - free:                       # more than there is room for only where a page was in two places
            ring[(first + free + given) % n] = page
            given += 1
    at[0], at[1] = (first + taken) % n, free - taken + given
    return off, positions, slots
