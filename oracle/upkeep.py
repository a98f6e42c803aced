"""Reference of the operators between two steps (TEST INFRASTRUCTURE ONLY):
attention weights of cached tokens, eviction by them, pages given back, beam
search's selection and the beams' rows of the page table.

Pinned by ``tests/test_upkeep.py`` (hand-worked cases and invariants). Plain
Python and numpy in 64 bits, from the definitions, on token arrays and lists of
page ids; where tokens lie in a pool is ``paged_kv``'s and ``paged_kvq``'s.
"""

import numpy as np

PAGE = 16


def pages_of(n):
    return (n + PAGE - 1) // PAGE


def weights(keys, q, lse, sees, scale, old, start, decay):
    """Weights [H, T] after one sequence's rows: keys [T, H, D], q [R, Hq, D], lse
    [R, Hq], sees [R] (how many tokens a row sees), old [H, T]; tokens from `start`
    on have no old weight. Also returns, for error bounds, the sum over rows of
    p * scale * sum |q_i k_i| and of p * (|s| + |lse|), both [H, T]."""
    T, H, _ = keys.shape
    G = q.shape[1] // H if len(q) else 1
    w, products, sizes = (np.zeros((H, T)) for _ in range(3))
    for h in range(H):
        k = keys[:, h]
        for r in range(len(q)):
            n = min(int(sees[r]), T)
            for g in range(h * G, (h + 1) * G):
                if n <= 0 or lse[r, g] == -np.inf:
                    continue
                s = scale * (k[:n] @ q[r, g])
                p = np.exp(s - lse[r, g])
                w[h, :n] += p
                products[h, :n] += p * scale * (np.abs(k[:n]) @ np.abs(q[r, g]))
                sizes[h, :n] += p * (np.abs(s) + abs(lse[r, g]))
        if decay:
            n = min(max(start, 0), T)
            w[h, :n] += decay * old[h, :n]
    return w, products, sizes


def evict(weights_row, length, budget, trigger, sinks, recent):
    """The tokens that one head of a sequence keeps (None: all): the first `sinks`,
    the last `recent`, and the heaviest of the others; equal weights: the earlier
    one; a NaN is less than any number."""
    if length <= trigger:
        return None

    def rank(t):
        x = float(weights_row[t])
        return (1, 0.0, t) if x != x else (0, -x, t)

    others = sorted(range(sinks, length - recent), key=rank)[:budget - sinks - recent]
    return sorted([*range(sinks), *others, *range(length - recent, length)])


def release(table, seq_len, new_len, free_pages, free_next):
    """(free list, free_next, flagged) after the pages of each row past its new
    length have gone back."""
    gone, flagged = [], False
    for row, a, b in zip(table, seq_len, new_len):
        if b < 0 or a < b or a > PAGE * len(row):
            flagged = True
            continue
        gone += [int(p) for p in row[pages_of(b):pages_of(a)]]
    out = list(free_pages)
    if not 0 <= free_next <= len(out) or len(gone) > free_next:
        return out, free_next, True
    out[free_next - len(gone):free_next] = gone
    return out, free_next - len(gone), flagged


def log_sum_exp(x):
    top = np.max(x)
    if not np.isfinite(top):
        return top
    return top + np.log(np.sum(np.exp(x - top)))


def select(logits, scores, ended, end_token, best):
    """(scores, tokens, parents) of one item: logits [W, V], scores [W]."""
    found = []
    for b, row in enumerate(np.asarray(logits, np.float64)):
        if not np.isfinite(scores[b]):
            continue
        if ended is not None and ended[b]:
            found.append((-float(scores[b]), b, end_token))
            continue
        if np.isnan(row).any() or (row == np.inf).any() or (row == -np.inf).all():
            continue
        # (from the largest logit, in whose size ln sum exp may be lost)
        top = np.max(row)
        value = ((row - top) - log_sum_exp(row - top)) + float(scores[b])
        live = np.flatnonzero(row > -np.inf)
        # (a beam's candidates past its own best `best` are none of the item's)
        order = live[np.lexsort((live, -row[live]))][:best]
        found += [(-float(value[t]), b, int(t)) for t in order]
    found = sorted(found)[:best]
    found += [(np.inf, -1, -1)] * (best - len(found))
    return [-v for v, _, _ in found], [t for _, _, t in found], [b for _, b, _ in found]


def beam_tables(items, beams, parents, seq_len, table, free_pages, free_next):
    """(table, lengths, free list, free_next, copy_src, copy_dst, flagged); rows of
    the table as lists of their pages alone."""
    flagged = False
    width = len(table[0]) if len(table) else 0
    parents = [[int(p) for p in row[:beams]] for row in parents]
    have = [pages_of(n) if 0 <= n <= PAGE * width else 0 for n in seq_len]
    for i in range(items):
        rows = range(i * beams, (i + 1) * beams)
        if any(not -1 <= p < beams for p in parents[i]) or any(not 0 <= seq_len[r] <= PAGE * width for r in rows):
            flagged = True
            parents[i] = list(range(beams))

    def step(parents):
        new, lengths, src, dst, taken, gone = [], [], [], [], 0, []
        for i in range(items):
            seen, kept = set(), set()
            for p in parents[i]:
                row = i * beams + p
                pages = [] if p < 0 else [int(x) for x in table[row][:have[row]]]
                lengths.append(0 if p < 0 else int(seq_len[row]))
                src.append(-1)
                dst.append(-1)
                if p >= 0 and p in seen and lengths[-1] % PAGE:
                    src[-1] = pages[-1]
                    at = free_next + taken
                    dst[-1] = pages[-1] = int(free_pages[at]) if 0 <= at < len(free_pages) else None
                    taken += 1
                seen.add(p)
                kept |= set(enumerate(pages))
                new.append(pages)
            done = set()
            for c in range(width):
                for b in range(beams):
                    row = i * beams + b
                    if c < have[row]:
                        page = (c, int(table[row][c]))
                        if page not in kept and page not in done:
                            gone.append(page[1])
                            done.add(page)
        return new, lengths, src, dst, taken, gone

    new, lengths, src, dst, taken, gone = step(parents)
    inside = 0 <= free_next <= len(free_pages)
    if not inside or free_next + taken > len(free_pages) or free_next + taken < len(gone):
        flagged = True
        new, lengths, src, dst, taken, gone = step([list(range(beams))] * items)
    out = list(free_pages)
    end = free_next + taken
    if inside:
        out[end - len(gone):end] = gone
    return new, lengths, out, end - len(gone), src, dst, flagged
