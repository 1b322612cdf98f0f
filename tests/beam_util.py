"""Beam search's choice, and the bookkeeping of a paged cache, in plain numpy and Python, for
their tests.  Sums of masses are in 80 bits, scores in 64."""
import numpy as np


def log_sum(l, T):
    """(maximum, ln of the sum of masses) of a row (float64); None if it has none."""
    if np.isnan(l).any() or (l == np.inf).any() or not np.isfinite(l).any():
        return None
    m = l.max()
    return m, float(np.log(np.exp(((l - m) / T).astype(np.longdouble)).sum()))


def select(logits, scores, k, T=1.0, ended=None, end_token=-1):
    """(parent, token, score in 64 bits) of one sequence, [W, V] float64 logits and [W] scores;
    None where a row or a score is out of its range.  T: a number or one a beam."""
    W, V = logits.shape
    T = np.broadcast_to(np.asarray(T, dtype=np.float32).astype(np.float64), (W,))
    found = []
    for w in range(W):
        s = float(scores[w])
        if np.isnan(s) or s == np.inf:
            return None
        if s == -np.inf:
            continue
        if ended is not None and ended[w]:
            found.append((-s, w, 0.0, end_token))
            continue
        ml = log_sum(logits[w], T[w])
        if ml is None:
            return None
        order = np.lexsort((np.arange(V), -logits[w]))[:k]
        for j in order[np.isfinite(logits[w][order])]:
            found.append((-(((logits[w, j] - ml[0]) / T[w] - ml[1]) + s), w, -logits[w, j], int(j)))
    found.sort()
    found = found[:k]
    none = k - len(found)
    return ([x[1] for x in found] + [-1] * none, [x[3] for x in found] + [-1] * none,
            [-x[0] for x in found] + [-np.inf] * none)


# what a score may be off besides its rounding: see test_gpu_beam
SUM_ERROR = 2.0e-6


def close_scores(got, want):
    got, want = np.asarray(got, dtype=np.float64), np.asarray(want, dtype=np.float64)
    with np.errstate(over="ignore"):
        same = want.astype(np.float32) == got
    fine = np.isfinite(want) & np.isfinite(got)
    off = np.abs(np.where(fine, got, 0.0) - np.where(fine, want, 0.0))
    return (same | (fine & (off <= np.abs(np.where(fine, want, 0.0)) * 2.0 ** -24 + SUM_ERROR))).all()


OK, BAD_PARAM, BAD_PAGE, NO_ROOM = 0, 10, 11, 12


def plan(kept, added, held, table, free, count, P, T):
    """resispec_plan_cache, request by request.  table (list of lists) and free are changed."""
    R, M, pages = len(kept), len(table[0]) if table else 1, len(free)
    status, want, starts, granted = [OK] * R, [0] * R, [0], [False] * R
    count_ok = 0 <= count <= pages
    at = 0
    for r in range(R):
        k, n, h = kept[r], added[r], held[r]
        if k < 0 or n < 0 or not 0 <= h <= M or k + n > M * P:
            status[r] = BAD_PARAM
            starts.append(at)
            continue
        want[r] = -(-(k + n) // P)
        if n > 0 and at + n > T:
            status[r] = NO_ROOM
        elif want[r] != h and not count_ok:
            status[r] = BAD_PARAM
        at += n
        starts.append(at)
    top, given = count, 0
    for r in range(R):
        if status[r] == OK and held[r] > want[r]:
            given += held[r] - want[r]
            if count + given > pages:
                status[r] = BAD_PARAM
                continue
            for e in range(want[r], held[r]):
                free[top] = table[r][e]
                top += 1
    avail, need, taken = top, 0, 0
    for r in range(R):
        if status[r] == OK and want[r] > held[r]:
            need += want[r] - held[r]
            if need > avail:
                status[r] = NO_ROOM
                continue
            for e in range(held[r], want[r]):
                top -= 1
                table[r][e] = free[top]
                taken += 1
    slots, positions, requests = [-1] * T, [-1] * T, [-1] * T
    for r in range(R):
        if status[r] != OK:
            continue
        for i in range(added[r]):
            t, p = starts[r] + i, kept[r] + i
            page = table[r][p // P]
            positions[t], requests[t] = p, r
            if 0 <= page < pages:
                slots[t] = page * P + p % P
            else:
                status[r] = BAD_PAGE
    out_held = [want[r] if status[r] in (OK, BAD_PAGE) else held[r] for r in range(R)]
    return slots, positions, requests, starts, out_held, avail - taken, status


def accepted_path(parent, token, tokens, length):
    """One sequence's path, or None."""
    N = len(parent)
    ways = {0: [0]}
    for n in range(1, N):
        way = ways.get(parent[n])
        if way is not None and len(way) <= length and token[n] == tokens[len(way) - 1]:
            ways[n] = way + [n]
    ends = [n for n, way in ways.items() if len(way) == length + 1]
    return ways[min(ends)] if ends else None
