"""Pages of the KV cache, block by block in Python -- oracle, test infrastructure only.

caches: arrays [num_blocks][..]; table [rows][max_blocks], lens [rows], refs [num_blocks]; changed in place.
"""
PAGE = 16


def _used(table, lens, row):
    return min((max(int(lens[row]), 0) + PAGE - 1) // PAGE, table.shape[1])


def copy_blocks(caches, src, dst):
    blocks = caches[0].shape[0]
    for s, d in zip(src, dst):
        if 0 <= s < blocks and 0 <= d < blocks:
            for c in caches:
                c[d] = c[s]


def fork(caches, table, lens, refs, parents, children, new_blocks):
    rows, blocks = len(lens), caches[0].shape[0]
    for p, c, new in zip(parents, children, new_blocks):
        if not (0 <= p < rows and 0 <= c < rows) or p == c:
            continue
        n = min(max(int(lens[p]), 0), table.shape[1] * PAGE)
        whole = n // PAGE
        if n % PAGE:
            old = table[p, whole]
            if not (0 <= old < blocks and 0 <= new < blocks):
                continue
            for x in caches:
                x[new] = x[old]
            table[c, whole] = new
            refs[new] += 1
        for e in range(whole):
            table[c, e] = table[p, e]
            if 0 <= table[p, e] < blocks:
                refs[table[p, e]] += 1
        lens[c] = n


def free(table, lens, refs, sequences):
    for s in sequences:
        if 0 <= s < len(lens):
            for e in range(_used(table, lens, s)):
                if 0 <= table[s, e] < len(refs):
                    refs[table[s, e]] -= 1
            lens[s] = 0


def compact(caches, table, lens, refs):
    """Two fingers: the lowest free block takes the highest one in use until they meet."""
    live, moved = int((refs > 0).sum()), {}
    low, high = 0, len(refs) - 1
    while True:
        while low < live and refs[low] > 0:
            low += 1
        while high >= live and refs[high] <= 0:
            high -= 1
        if low >= live or high < live:
            break
        for c in caches:
            c[low] = c[high]
        moved[high] = low
        refs[low], refs[high] = refs[high], 0
    for r in range(len(lens)):
        for e in range(_used(table, lens, r)):
            table[r, e] = moved.get(int(table[r, e]), table[r, e])
    return live
