"""The paged key-value cache in float64: append with norm and rotation, and
attention over the pages, from their definitions (include/gvc.h).

Plain NumPy, one row at a time; arrays are float64 except the int32 lists.
"""
import numpy as np


def rope_norm(x, position, pairs, theta, gain=None, eps=1e-5):
    """One head vector x with norm (if gain) and rotation; position[axis]."""
    x = np.array(x, dtype=np.float64)
    if gain is not None:
        x = x / np.sqrt(np.mean(x * x) + eps) * gain
    n = sum(pairs)
    out = x.copy()
    i = 0
    for axis, count in enumerate(pairs):
        for _ in range(count):
            a = float(position[axis]) * float(theta) ** (-i / n)
            out[i] = x[i] * np.cos(a) - x[i + n] * np.sin(a)
            out[i + n] = x[i + n] * np.cos(a) + x[i] * np.sin(a)
            i += 1
    return out


def place(table, n_pages, page, seq, slot):
    """(page id, offset) of a slot, or None where there is none."""
    if not 0 <= seq < table.shape[0] or slot < 0 or slot // page >= table.shape[1]:
        return None
    pid = int(table[seq, slot // page])
    return (pid, slot % page) if 0 <= pid < n_pages else None


def seen_slots(last, window, sinks):
    """The slots that a row sees whose last slot is `last`, before pages are looked up."""
    return [j for j in range(last + 1) if window == 0 or j > last - window or j < sinks]


def attend_row(q, seq, last, k_pages, v_pages, table, scale, window=0, sinks=0):
    """Output [heads][dh] of one row q [heads][dh], and with it sum_j p_j |v_j|
    and max_j scale sum_i |q_i k_ji| per head, which error bounds are made of."""
    n_pages, kv, page, dh = k_pages.shape
    heads = q.shape[0]
    last = min(last, table.shape[1] * page - 1)
    at = [place(table, n_pages, page, seq, j) for j in seen_slots(last, window, sinks)]
    at = [x for x in at if x is not None]
    out, mag, top = np.zeros((heads, dh)), np.zeros((heads, dh)), np.zeros(heads)
    if not at:
        return out, mag, top, 0
    pid, off = np.array([x[0] for x in at]), np.array([x[1] for x in at])
    for h in range(heads):
        g = h // (heads // kv)
        k, v = k_pages[pid, g, off], v_pages[pid, g, :, off]
        with np.errstate(invalid="ignore", over="ignore"):
            s = k @ q[h] * scale
            p = np.exp(s - s.max())
            p = p / p.sum()
            out[h], mag[h] = p @ v, p @ np.abs(v)
            top[h] = scale * (np.abs(k) @ np.abs(q[h])).max()
    return out, mag, top, len(at)
