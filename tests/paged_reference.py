"""The paged-cache operators written out in 64 bits on the CPU (numpy), request by request, for the tests."""
import numpy as np


def extend(lengths, n_new, owned, table, free, count, page, max_rows):
    """(status, row_start, positions, slots, lengths, owned, count, table), as lists and an array."""
    n, width = table.shape
    status = 0
    if not 0 <= count <= len(free) or any(x < 0 for x in [*lengths, *n_new, *owned]) or any(x > width for x in owned):
        status = 1
    need = [-(-(a + b) // page) for a, b in zip(lengths, n_new)]
    # the checks of a request stop at its first fault
    faults = [1 if a < 0 or b < 0 or c < 0 or c > width else 2 if x > width else 0
              for a, b, c, x in zip(lengths, n_new, owned, need)]
    found = [f for f in faults if f] + ([1] if status else [])
    good = [i for i in range(n) if not faults[i]]
    fresh = [max(0, need[i] - owned[i]) if not faults[i] else 0 for i in range(n)]
    if sum(n_new[i] for i in range(n) if faults[i] != 1) > max_rows:
        found.append(3)
    if sum(fresh[i] for i in good) > count:
        found.append(4)
    if found:
        return min(found), [0] * (n + 1), [0] * max_rows, [-1] * max_rows, list(lengths), list(owned), count, table.copy()
    table = table.copy()
    positions, slots, row_start = [0] * max_rows, [-1] * max_rows, [0]
    left = count
    for i in range(n):
        for j in range(fresh[i]):
            left -= 1
            table[i, owned[i] + j] = free[left]
        for t in range(n_new[i]):
            pos, r = lengths[i] + t, row_start[-1] + t
            positions[r] = pos
            slots[r] = int(table[i, pos // page]) * page + pos % page
        row_start.append(row_start[-1] + n_new[i])
    return (0, row_start, positions, slots, [a + b for a, b in zip(lengths, n_new)], [a + b for a, b in zip(owned, fresh)], left, table)


def rotate(x, positions, theta):
    """x [rows, heads, D] in float64."""
    half = x.shape[-1] // 2
    angle = np.asarray(positions, np.float64)[:, None] * np.float64(theta) ** (-np.arange(half, dtype=np.float64) / half)
    c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
    a, b = x[..., :half], x[..., half:]
    return np.concatenate([a * c - b * s, b * c + a * s], -1)


def attention(q, k_pool, v_pool, table, row_start, lengths, scale, page):
    """(out, sum_j p_j |v_j|, sum_i |q_i k_i| at its largest), rows outside the batch NaN.  Pools [block, head, slot, D], float64."""
    rows, H, D = q.shape
    n_blocks, Hkv = k_pool.shape[:2]
    out, size = np.full((rows, H, D), np.nan), np.full((rows, H, D), np.nan)
    most = 0.0
    for i in range(len(lengths)):
        m = row_start[i + 1] - row_start[i]
        for t in range(m):
            last = min(lengths[i] - m + t, table.shape[1] * page - 1)
            at = np.arange(last + 1)
            block = table[i, at // page]
            there = (block >= 0) & (block < n_blocks)
            at, block = at[there], block[there]
            r = row_start[i] + t
            for g in range(Hkv):
                heads = slice(g * (H // Hkv), (g + 1) * (H // Hkv))
                if not len(at):
                    out[r, heads] = size[r, heads] = 0.0
                    continue
                k, v = k_pool[block, g, at % page], v_pool[block, g, at % page]
                s = q[r, heads] @ k.T * scale
                most = max(most, float((np.abs(q[r, heads]) @ np.abs(k).T).max()) * scale)
                p = np.exp(s - s.max(-1, keepdims=True))
                p /= p.sum(-1, keepdims=True)
                out[r, heads], size[r, heads] = p @ v, p @ np.abs(v)
    return out, size, most


def verify(tokens, target, draft, row_start, u_accept, u_sample, lengths):
    """(n_accepted, next_token, emitted, lengths); probabilities in float64."""
    accepted, following, emitted, after = [], [], [-2] * len(tokens), []
    vocab = target.shape[1]
    for i in range(len(row_start) - 1):
        begin, end = row_start[i], row_start[i + 1]
        if begin == end:
            accepted.append(0), following.append(-1), after.append(lengths[i])
            continue
        row = begin
        while row + 1 < end:
            x = tokens[row + 1]
            if not 0 <= x < vocab or not float(u_accept[row]) * (draft[row, x] if draft is not None else 1.0) < target[row, x]:
                break
            row += 1
        w = target[row].copy()
        if row + 1 < end:
            if draft is not None:
                w = w - draft[row]
            elif 0 <= tokens[row + 1] < vocab:
                w[tokens[row + 1]] = 0.0
        with np.errstate(invalid="ignore"):
            def clean(x):
                return np.where((x > 0) & np.isfinite(x), x, 0.0)
            w = clean(w)
            if row + 1 < end and not w.any():
                w = clean(target[row])
        if not w.any():
            x = -1
        else:
            total = np.cumsum(w)
            u = float(u_sample[i])
            over = np.nonzero(total > (max(u, 0.0) * total[-1] if u == u else np.inf))[0]
            over = over[w[over] > 0]
            x = int(over[0]) if len(over) else int(np.nonzero(w)[0][-1])
        accepted.append(row - begin), following.append(x), after.append(lengths[i] + 1 + row - begin)
        for r in range(begin, end):
            emitted[r] = tokens[r + 1] if r < row else x if r == row else -1
    return accepted, following, emitted, after
