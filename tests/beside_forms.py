"""Plain forms, in 64 bits and one row at a time, of the operators beside the verification (drafts, beams, states, pages)."""
import numpy as np

ROW_OK, ROW_BAD, ROW_NO_ROOM = 0, 3, 4


def softmax_mass(x, T):
    """Masses of a row of logits (any total); nothing where every entry is masked."""
    x = np.asarray(x, np.float64)
    top = x.max()
    return np.exp((x - top) / T) if np.isfinite(top) else np.zeros_like(x)


def draft_support(x, k):
    """Ids of the k largest entries of x that are worth drawing, ascending (ties: lower id)."""
    order = np.argsort(-np.asarray(x, np.float64), kind="stable")
    return np.sort(order[:k] if 0 < k < len(x) else order)


def draw(mass, ids, uniforms):
    """(token, distance of u from the nearest border of the CDF) of every uniform."""
    cdf = np.cumsum(mass)
    last = np.flatnonzero(mass > 0)[-1]
    out = []
    for u in np.asarray(uniforms, np.float64):
        at = min(int(np.searchsorted(cdf, u * cdf[-1], side="right")), int(last))
        out.append((int(ids[at]), float(np.abs(cdf / cdf[-1] - u).min())))
    return out


def beam_select(logits, scores, M, T=1.0, finished=None, eos=-1):
    """One sequence: logits [K, V], scores [K].  Lists of (score, parent, token), best first, at most M."""
    found = []
    K, V = logits.shape
    for b in range(K):
        s = float(scores[b])
        if s == -np.inf:
            continue
        if finished is not None and finished[b]:
            found.append((s, b, 0.0, eos))
            continue
        x = logits[b].astype(np.float64)
        mass = softmax_mass(x, T)
        if not mass.any():
            continue
        log_sum = np.log(mass.sum())
        best = np.argsort(-x, kind="stable")[:M]
        found += [(s + ((x[v] - x.max()) / T - log_sum), b, x[v], int(v)) for v in best if x[v] > -np.inf]
    found.sort(key=lambda f: (-f[0], f[1], -f[2], f[3]))
    return [(f[0], f[1], f[3]) for f in found[:M]]


def reorder(state, parent, first=None, length=None, table=None):
    """state [O, rows, H, T, D] (numpy), or [O, blocks, H, block, D] with a table."""
    S, K = parent.shape
    T = state.shape[3]
    new = state.copy()
    for s in range(S):
        lo = 0 if first is None else max(0, int(first[s]))
        most = T if table is None else T * table.shape[1]
        hi = most if length is None else min(most, int(length[s]))
        for b in range(K):
            p = int(parent[s, b])
            if p < 0 or p >= K or p == b:
                continue
            if table is None:
                if hi > lo:
                    new[:, s * K + b, :, lo:hi] = state[:, s * K + p, :, lo:hi]
                continue
            for j in range(lo // T, (hi + T - 1) // T if hi > lo else 0):
                a, c = int(table[s * K + p, j]), int(table[s * K + b, j])
                if a == c or not (0 <= a < state.shape[1] and 0 <= c < state.shape[1]):
                    continue
                t0, t1 = max(lo - j * T, 0), min(hi - j * T, T)
                new[:, c, :, t0:t1] = state[:, a, :, t0:t1]
    return new


def page_update(lengths, new_lengths, table, free_blocks, free_count, block, slots):
    """(lengths, free_count, starts, status, slots, table, free stack) after the call; requests one after the other."""
    R, width = table.shape
    table, slots = table.copy(), slots.copy()
    stack = [int(x) for x in free_blocks[:free_count]]
    out, status = [int(x) for x in lengths], [ROW_OK] * R
    up = lambda x: -(-int(x) // block)  # noqa: E731
    fits = [0 <= a <= width * block and 0 <= b <= width * block for a, b in zip(lengths, new_lengths)]
    for r in range(R):
        if not fits[r]:
            status[r] = ROW_BAD
        elif new_lengths[r] <= lengths[r]:
            stack += [int(x) for x in table[r, up(new_lengths[r]):up(lengths[r])]]
            out[r] = int(new_lengths[r])
    starts, short = [0], False
    for r in range(R):
        grow = fits[r] and new_lengths[r] > lengths[r]
        if grow:
            need, more = up(new_lengths[r]) - up(lengths[r]), int(new_lengths[r]) - int(lengths[r])
            short = short or need > len(stack) or starts[-1] + more > len(slots)
            if short:
                status[r], grow = ROW_NO_ROOM, False
        if grow:
            for j in range(up(lengths[r]), up(new_lengths[r])):
                table[r, j] = stack.pop()
            for i, t in enumerate(range(int(lengths[r]), int(new_lengths[r]))):
                page = int(table[r, t // block])
                slots[starts[-1] + i] = page * block + t % block if page >= 0 else -1
            out[r] = int(new_lengths[r])
        starts.append(starts[-1] + (int(new_lengths[r]) - int(lengths[r]) if grow else 0))
    return np.array(out), len(stack), np.array(starts), np.array(status), slots, table, np.array(stack, np.int64)
