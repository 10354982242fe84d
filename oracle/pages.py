"""Reference moves of the paged cache: kept tokens to the front, sequences that continue others.

Test infrastructure; see oracle/__init__.py.  One token and one table entry at a time.
"""
import numpy as np

from .cache import DECODE, PAGE, encode, scale_of


def keep(k, v, ks, vs, table, lens, path, kept, counts):
    """k [P, H, 64, d], v [P, H, d, 64] uint8 codes and ks, vs [P, H]: updated in place."""
    def page_of(b, slot):
        p = slot // PAGE
        return int(table[b, p]) if p < table.shape[1] and 0 <= table[b, p] < k.shape[0] else -1

    for b in range(len(lens)):
        nodes = min(int(counts[b]), int(lens[b]))
        first = int(lens[b]) - nodes
        n = min(int(kept[b]), nodes)
        for lp in range(first // PAGE, (first + n - 1) // PAGE + 1 if n > 0 else 0):
            page = page_of(b, lp * PAGE)
            if page < 0:
                continue
            moves = []   # (slot in the page, source page, slot in it)
            for i in range(max(lp * PAGE - first, 0), min((lp + 1) * PAGE - first, n)):
                u = int(path[b, i])
                if i < u < nodes and page_of(b, first + u) >= 0:
                    moves.append((first + i - lp * PAGE, page_of(b, first + u), (first + u) % PAGE))
            live = min(first + n - lp * PAGE, PAGE)
            for h in range(k.shape[1]):
                for codes, scale in ((k[:, h], ks), (v[:, h].swapaxes(-1, -2), vs)):
                    x = [(o, codes[p, s].copy(), float(scale[p, h]), p) for o, p, s in moves]
                    was = now = float(scale[page, h])
                    for _, c, s, p in x:
                        if p != page:
                            a = np.abs(DECODE[c] * s)
                            a = a[np.isfinite(a)]
                            now = max(now, scale_of(a.max() if a.size else 0.0))
                    with np.errstate(invalid="ignore"):
                        if now != was:
                            codes[page, :live] = encode(DECODE[codes[page, :live]] * (was / now))
                        for o, c, s, _ in x:
                            codes[page, o] = c if s == now else encode(DECODE[c] * (s / now))
                    scale[page, h] = now


def fork(table, lens, refs, src, room, pages):
    """(table [N, width], lens [N], refs, missing [N], copies [(from, to)])."""
    B, width = table.shape
    N = len(src)
    refs = np.array(refs, np.int64)
    rows, out_lens, missing, copies = np.full((N, width), -1, np.int64), np.zeros(N, np.int64), np.zeros(N, np.int64), []
    for b in range(B):
        for p in table[b]:
            if 0 <= p < pages:
                refs[p] -= 1
    ask, first = [], set()
    for n in range(N):
        b = int(src[n]) if 0 <= src[n] < B else -1
        length = min(max(int(lens[b]), 0), PAGE * width) if b >= 0 else 0
        leads = b >= 0 and b not in first
        first.add(b)
        want = max(0 if room is None else int(room[n]), length)
        out_lens[n] = length
        for i in range(min((want + PAGE - 1) // PAGE, width)):
            p = int(table[b, i]) if b >= 0 and 0 <= table[b, i] < pages else -1
            if p >= 0 and (leads or i < length // PAGE):
                rows[n, i] = p
                refs[p] += 1
            elif p >= 0 or i * PAGE >= length:
                ask.append((n, i, p if i * PAGE < length else -1))
    free = [p for p in range(pages) if refs[p] == 0]
    for x, (n, i, of) in enumerate(ask):
        if x < len(free):
            rows[n, i] = free[x]
            refs[free[x]] = 1
            if of >= 0:
                copies.append((of, free[x]))
        else:
            missing[n] += 1
            if of >= 0:
                out_lens[n] = i * PAGE
    return rows, out_lens, refs, missing, copies
