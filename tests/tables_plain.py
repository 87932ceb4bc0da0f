"""What lrqk_pages_advance does, one sequence after the other in plain Python, and what lrqk_rotate does, in float64: what the
tests compare with.  Written from the definitions; neither the HIP library nor its plain torch forms are called."""
from __future__ import annotations

import numpy as np

OK, LONG, SHARED, PAGES, ROWS = range(5)


def pages(n, page):
    return -(-n // page)


def advance(refs, table, kv_len, keep, n_new, *, page, n_max, l_max, T):
    """Lists and arrays of the state (not changed) -> dict of what the call leaves."""
    refs, table, kv_len = refs.copy(), table.copy(), kv_len.copy()
    B, n_pages = len(kv_len), len(refs)
    kept = []
    for b in range(B):
        old = min(max(int(kv_len[b]), 0), l_max)
        k = old if keep is None else min(max(int(keep[b]), 0), old)
        kept.append(k)
        for i in range(pages(k, page), pages(old, page)):
            if 0 <= table[b, i] < n_pages:
                refs[table[b, i]] -= 1
            table[b, i] = -1
    free = [p for p in range(n_pages) if refs[p] <= 0]
    status, start, asked_pages, asked_rows, given = [], [0], 0, 0, 0
    for b in range(B):
        k, n = kept[b], max(int(n_new[b]), 0)
        st, need = OK, 0
        if n > 0:
            last = int(table[b, pages(k, page) - 1]) if k % page else -1
            if n > n_max or k + n > l_max:
                st = LONG
            elif k % page and 0 <= last < n_pages and refs[last] > 1:
                st = SHARED
            else:
                need = pages(k + n, page) - pages(k, page)
                asked_pages += need
                asked_rows += n
                if need and asked_pages > len(free):
                    st = PAGES
                elif asked_rows > T:
                    st = ROWS
        if st != OK:
            n = need = 0
        for i in range(need):
            p = free[given]
            given += 1
            refs[p] = 1
            table[b, pages(k, page) + i] = p
        kv_len[b] = k + n
        status.append(st)
        start.append(start[-1] + n)
    seq, pos, slot = (np.full(T, -1, np.int32) for _ in range(3))
    for b in range(B):
        for i in range(start[b + 1] - start[b]):
            t, p = start[b] + i, kept[b] + i
            seq[t], pos[t] = b, p
            pg = int(table[b, p // page])
            slot[t] = pg * page + p % page if 0 <= pg < n_pages else -1
    return dict(refs=refs, table=table, kv_len=kv_len.astype(np.int32), start=np.array(start, np.int32),
                status=np.array(status, np.int32), seq=seq, pos=pos, slot=slot)


PLAIN, LINEAR, BASE, BANDS, RAMP = range(5)


def frequencies(rot, scaling, base, factor=1.0, low=1.0, high=4.0, l_orig=8192):
    """Radians a position of each pair, and the amplitude."""
    f = []
    for j in range(rot // 2):
        b = base * factor ** (rot / (rot - 2)) if scaling == BASE and rot > 2 else base
        x = b ** (-2 * j / rot)
        turns = l_orig * x / (2 * np.pi)
        s = 1.0
        if scaling == LINEAR:
            s = 0.0
        elif scaling == BANDS:
            s = (turns - low) / (high - low)
        elif scaling == RAMP:
            index = lambda n: rot * np.log(l_orig / (2 * np.pi * n)) / (2 * np.log(base))  # noqa: E731
            j0, j1 = max(int(np.floor(index(high))), 0), min(int(np.ceil(index(low))), rot // 2 - 1)
            s = 1.0 - (j - j0) / max(j1 - j0, 0.001)
        s = min(max(s, 0.0), 1.0)
        f.append(x if scaling in (PLAIN, BASE) else x * (s + (1 - s) / factor))
    return np.array(f), 0.1 * np.log(factor) + 1.0 if scaling == RAMP and factor > 1 else 1.0


def turned(x, pos, f, amplitude, pairs, back):
    """Rows x [T,H,128] float64 at positions pos -> y and |x_u| + |x_v| of each element's pair (0: not turned)."""
    y, mass = x.copy(), np.zeros_like(x)
    half = len(f)
    a = pos.astype(np.float64)[:, None] * f          # |p f| < 2^31: off by 2^-22 at most, far less below 2^24
    a = np.where(back, -a, a)
    c, s = np.cos(a)[:, None], np.sin(a)[:, None]
    u, v = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if pairs else (slice(0, half), slice(half, 2 * half))
    with np.errstate(invalid="ignore"):
        y[..., u], y[..., v] = amplitude * (x[..., u] * c - x[..., v] * s), amplitude * (x[..., v] * c + x[..., u] * s)
    mass[..., u] = mass[..., v] = np.abs(x[..., u]) + np.abs(x[..., v])
    return y, mass
