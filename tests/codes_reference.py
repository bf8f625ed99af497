"""Pools in 8 bits, the selection of a beam search and the reordering of tables, written out on the CPU (numpy), for the tests."""
import numpy as np

INT8, E4M3 = "int8", "e4m3"
TOP = {INT8: 127.0, E4M3: 448.0}
LEAST = 2.0 ** -100


def e4m3_values():
    """What the 256 codes of e4m3 stand for, in float64."""
    out = np.empty(256)
    for code in range(256):
        sign, exponent, fraction = (-1.0 if code >> 7 else 1.0), (code >> 3) & 15, code & 7
        out[code] = sign * (fraction * 2.0 ** -9 if exponent == 0 else (8 + fraction) * 2.0 ** (exponent - 10))
        if code & 127 == 127:
            out[code] = np.nan
    return out


def numbers(codes, kind):
    """codes: an array of bytes."""
    return codes.view(np.int8).astype(np.float64) if kind == INT8 else e4m3_values()[codes]


def nearest(y, kind):
    """The bytes of the codes nearest to y, ties to even."""
    if kind == INT8:
        return np.rint(y).astype(np.int8).view(np.uint8)
    y = np.asarray(y, np.float64)
    with np.errstate(divide="ignore"):
        exponent = np.where(y == 0, -6, np.floor(np.log2(np.abs(np.where(y == 0, 1, y)))))
    step = 2.0 ** (np.maximum(exponent, -6) - 3)
    value = np.minimum(np.rint(np.abs(y) / step) * step, 448.0)
    magnitudes = e4m3_values()[:127]
    code = np.searchsorted(magnitudes, value)
    assert (magnitudes[code] == value).all()
    return (code + 128 * np.signbit(y)).astype(np.uint8)


def quantise(x, kind):
    """(bytes, scales) of x [..., D] in float32, operation by operation as the definition says."""
    x = np.asarray(x, np.float32)
    m = np.maximum(np.abs(x).max(-1), np.float32(LEAST)).astype(np.float32)
    top = np.float32(TOP[kind])
    bad = ~np.isfinite(m)
    with np.errstate(invalid="ignore", divide="ignore"):
        y = np.where(bad[..., None], np.float32(0), x * (top / m)[..., None])
        scale = np.where(bad, np.float32("nan"), m / top).astype(np.float32)
    return nearest(y, kind), scale


def beam_select(logits, scores, keep, end_token, ended):
    """(parents, tokens, scores, ended) of logits [n, B, V] and scores [n, B] in float64."""
    n, B, V = logits.shape
    parents, tokens, best, over = (np.full((n, keep), -1), np.full((n, keep), -1), np.full((n, keep), -np.inf), np.zeros((n, keep), int))
    for i in range(n):
        value, beam, token = [], [], []
        for b in range(B):
            if not np.isfinite(scores[i, b]):
                continue
            if ended is not None and ended[i, b]:
                value.append([scores[i, b]]), beam.append([b]), token.append([end_token])
                continue
            x = logits[i, b]
            ok = np.nonzero(np.isfinite(x))[0]
            if not len(ok):
                continue
            top = x[ok].max()
            s = scores[i, b] + (x[ok] - (top + np.log(np.exp(x[ok] - top).sum())))
            value.append(s), beam.append(np.full(len(ok), b)), token.append(ok)
        if not value:
            continue
        value, beam, token = map(np.concatenate, (value, beam, token))
        order = np.lexsort((token, beam, -value))[:keep]
        m = len(order)
        parents[i, :m], tokens[i, :m], best[i, :m] = i * B + beam[order], token[order], value[order]
        over[i, :m] = [(ended is not None and bool(ended[i, b])) or (t == end_token >= 0) for b, t in zip(beam[order], token[order])]
    return parents, tokens, best, over


def reorder(parents, table, lengths, owned, free, count, page, width, held=None):
    """A dict of what comes out; table a list of rows."""
    n_in, old_width, n_out, n_free = len(lengths), len(table[0]) if len(table) else 0, len(parents), len(free)
    status = 0 if 0 <= count <= n_free else 1
    need = [-(-x // page) for x in lengths]
    for p in parents:
        if p == -1:
            continue
        if not 0 <= p < n_in or lengths[p] < 0 or not 0 <= owned[p] <= old_width or need[p] > owned[p]:
            status = 1
        elif need[p] > width and status == 0:
            status = 2
    empty = dict(table=[[-1] * width for _ in parents], lengths=[0] * n_out, owned=[0] * n_out, free_blocks=list(free), free_count=count,
                 copy_from=[-1] * n_out, copy_to=[-1] * n_out)
    copied = [p != -1 and 0 <= p < n_in and lengths[p] % page != 0 and p in parents[:i] for i, p in enumerate(parents)]
    if status == 0 and sum(copied) > count:
        status = 4
    if status:
        return dict(empty, status=status)
    out = dict(empty, status=0)
    left = count
    for i, p in enumerate(parents):
        if p == -1:
            continue
        out["lengths"][i], out["owned"][i] = lengths[p], need[p]
        out["table"][i][:need[p]] = table[p][:need[p]]
        if copied[i]:
            left -= 1
            full = lengths[p] // page
            out["copy_from"][i], out["copy_to"][i] = table[p][full], free[left]
            out["table"][i][full] = free[left]
    before = {b for row, n in zip(table, owned) for b in row[:max(0, min(n, old_width))]}
    after = {b for row in out["table"] for b in row}
    for b in sorted(before - after):
        if 0 <= b < n_free and not (held is not None and held[b]) and left < n_free:
            out["free_blocks"][left] = b
            left += 1
    out["free_count"] = left
    return out
