"""Plain implementations of the operators for requests that share pages, in Python integers, on the host.  Written from the definitions; shares
no code with the library."""
import numpy as np


def kv_fork(lengths, source, rows, table, free, state, page_size, pages, table_out):
    """(table, lengths, copies, ring, ring state) after the call; one request after the other."""
    R, wide = table.shape
    out, ring, F = table_out.copy(), np.array(free).copy(), len(free)
    first = int(state[0]) if 0 <= state[0] < F else 0
    available = min(max(int(state[1]), 0), F)
    have = [min(max(int(n), 0), wide * page_size) for n in lengths]
    taken_over, kept, asked, used = set(), set(), 0, 0
    out_len, copies = [], []
    for r, s in enumerate(int(x) for x in source):
        n = have[s] if 0 <= s < R else 0
        if rows is not None:
            n = min(n, max(int(rows[r]), 0))
        whole, rest = n // page_size, n % page_size
        copy = (-1, -1, 0)
        if rest:
            if n // page_size == have[s] // page_size and s not in taken_over:
                taken_over.add(s)
                whole += 1
            else:
                asked += 1
                copy = (int(table[s, whole]), -1, rest)
                if asked > available:
                    out_len.append(0)
                    copies.append(copy)
                    continue
                out[r, whole] = free[(first + used) % F]
                copy = (copy[0], int(out[r, whole]), rest)
                used += 1
        for j in range(whole):
            out[r, j] = table[s, j]
            kept.add(int(table[s, j]))
        out_len.append(n)
        copies.append(copy)
    held = {int(table[s, j]) for s in range(R) for j in range(-(-have[s] // page_size))}
    back = sorted(p for p in held - kept if 0 <= p < pages)
    for i, p in enumerate(back[:F - available]):
        ring[(first + available + i) % F] = p
    return out, out_len, copies, ring, [(first + used) % F, available - used + min(len(back), F - available)]


def shared_rows(table, lengths, offsets, page_size):
    R, wide = table.shape
    at = [min(max(int(x), 0), R) for x in offsets]
    out = []
    for a, b in zip(at, at[1:]):
        mine = [r for r in range(a, b) if lengths[r] > 0]
        n = 0
        while mine and n < wide and all(lengths[r] >= (n + 1) * page_size and table[r, n] == table[mine[0], n] for r in mine):
            n += 1
        out.append(n * page_size)
    return out
