"""Plain forms of the calls around a wave's attention, on the CPU: page tables, sequence by sequence."""

import numpy as np

EINVAL, ESIZE = -1, -5


def reserve(new, kv, pages, free, n_free, P, T):
    """off, kv, n_free, taken, slots, positions, pages, status of fate_kv_reserve from lists and arrays."""
    pages, kv = pages.copy(), list(kv)
    B, width, n_pages = len(new), pages.shape[1], len(free)
    usable = n_free if 0 <= n_free <= n_pages else 0
    off, taken, slots, positions, status = [0], [0], [], [], [0] * B
    asked = rows = given = 0
    for b in range(B):
        if new[b] < 0 or kv[b] < 0 or kv[b] + new[b] > width * P:
            status[b] = EINVAL
        else:
            more = -(-(kv[b] + new[b]) // P) - -(-kv[b] // P)
            asked, rows = asked + more, rows + new[b]
            if (more and asked > usable) or rows > T:
                status[b] = ESIZE
            else:
                for x in range(more):
                    pages[b, -(-kv[b] // P) + x] = free[usable - 1 - given - x]
                given += more
                for at in range(kv[b], kv[b] + new[b]):
                    page = int(pages[b, at // P])
                    positions.append(at)
                    slots.append(page * P + at % P if 0 <= page < n_pages else -1)
                    if not 0 <= page < n_pages:
                        status[b] = EINVAL
                kv[b] += new[b]
        off.append(len(positions))
        taken.append(given)
    rest = [-1] * (T - len(slots))
    return (np.array(off), np.array(kv, np.int64).reshape(-1), np.array([n_free - given]), np.array(taken),
            np.array(slots + rest, np.int64), np.array(positions + rest, np.int64), pages, np.array(status, np.int64))


def trim(keep, kv, pages, free, n_free, P):
    """kv, n_free, given, free, status of fate_kv_trim."""
    free, kv = np.array(free), list(kv)
    B, width, n_pages = len(keep), pages.shape[1], len(free)
    given, status, total, asked = [0], [0] * B, 0, 0
    for b in range(B):
        stay = min(keep[b], kv[b])
        ok = keep[b] >= 0 and 0 <= kv[b] <= width * P
        mine = pages[b, -(-stay // P):-(-kv[b] // P)] if ok else []
        ok = ok and all(0 <= p < n_pages for p in mine)
        if ok and len(mine):
            asked += len(mine)
            ok = 0 <= n_free <= n_pages and n_free + asked <= n_pages
        if ok:
            free[n_free + total:n_free + total + len(mine)] = mine
            total += len(mine)
            kv[b] = stay
        else:
            status[b] = EINVAL
        given.append(total)
    return np.array(kv, np.int64).reshape(-1), np.array([n_free + total]), np.array(given), free, np.array(status, np.int64)
