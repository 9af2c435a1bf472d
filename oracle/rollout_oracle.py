"""fp64 definitions of the rollout operators: rotary positions, new tokens entering a paged cache, attention over it."""
import numpy as np


def frequencies(rot_dim, base=10000.0, scaling=0, factor=1.0, original_len=0.0, low=1.0, high=32.0):
    """Angle per position of each pair (radians) and the factor on the rotated values."""
    theta = np.array([base ** (-2.0 * i / rot_dim) for i in range(rot_dim // 2)])
    if scaling == 1:
        return theta / factor, 1.0
    if scaling == 2:
        return np.array([(base * factor ** (rot_dim / (rot_dim - 2.0))) ** (-2.0 * i / rot_dim) for i in range(rot_dim // 2)]), 1.0
    if scaling == 3:
        turns = original_len * theta / (2.0 * np.pi)
        keep = np.clip((turns - low) / (high - low), 0.0, 1.0)
        return keep * theta + (1.0 - keep) * theta / factor, 0.1 * np.log(factor) + 1.0
    return theta, 1.0


def rotary(x, pos, theta, interleaved=False, amplitude=1.0, inverse=False):
    """x [n][heads][dim] turned by pos theta, as products of complex numbers."""
    x = np.array(x, dtype=np.float64)
    m = len(theta)
    turn = np.exp((-1j if inverse else 1j) * np.asarray(pos, dtype=np.float64)[:, None, None] * np.asarray(theta))
    a, b = (slice(0, 2 * m, 2), slice(1, 2 * m, 2)) if interleaved else (slice(0, m), slice(m, 2 * m))
    z = (x[..., a] + 1j * x[..., b]) * turn * amplitude
    x[..., a], x[..., b] = z.real, z.imag
    return x


def sequences(seq_len, q_off, n):
    """(first row, position of its first token, number of rows) of each sequence."""
    if q_off is None:
        q_off = np.arange(n + 1)
    return [(int(a), int(length) - (int(b) - int(a)), int(b) - int(a)) for a, b, length in zip(q_off[:-1], q_off[1:], seq_len)]


def append(k, v, k_pages, v_pages, table, seq_len, q_off):
    """Copies of the pages [n_pages][page][heads][dim] with the new tokens' (rotated) keys and values in their slots."""
    k_pages, v_pages = np.array(k_pages, dtype=np.float64), np.array(v_pages, dtype=np.float64)
    page = k_pages.shape[1]
    for s, (row, first, count) in enumerate(sequences(seq_len, q_off, len(k))):
        for i in range(count):
            j = first + i
            if j >= 0:
                at = table[s][j // page], j % page
                k_pages[at], v_pages[at] = k[row + i], v[row + i]
    return k_pages, v_pages


def seen(pos, length, window, sinks):
    j = np.arange(length)
    m = j <= pos
    if window:
        m &= (j > pos - window) | (j < sinks)
    return m


def attend(q, k_pages, v_pages, table, seq_len, q_off, scale, window=0, sinks=0):
    """out [n][heads][dim], lse [n][heads], and two sums that bound rounding: sum_j p_j |v_j| (as out) and
    max_j scale sum_d |q_d k_jd| (as lse).  Rows of no sequence are NaN."""
    n, heads, dim = q.shape
    page, kv = k_pages.shape[1], k_pages.shape[2]
    group = heads // kv
    out, mass = np.full(q.shape, np.nan), np.full(q.shape, np.nan)
    lse, reach = np.full((n, heads), np.nan), np.full((n, heads), np.nan)
    for s, (row, first, count) in enumerate(sequences(seq_len, q_off, n)):
        for i in range(count):
            m = np.flatnonzero(seen(first + i, max(0, int(seq_len[s])), window, sinks))
            r = row + i
            if m.size == 0:
                out[r], mass[r], lse[r], reach[r] = 0.0, 0.0, -np.inf, 0.0
                continue
            pages = np.asarray(table[s])[m // page]
            k, v = k_pages[pages, m % page].astype(np.float64), v_pages[pages, m % page].astype(np.float64)    # [keys][kv][dim]
            for h in range(heads):
                kh, vh, qh = k[:, h // group], v[:, h // group], q[r, h].astype(np.float64)
                z = scale * (kh @ qh)
                top = z.max()
                e = np.exp(z - top)
                p = e / e.sum()
                out[r, h], mass[r, h] = p @ vh, p @ np.abs(vh)
                lse[r, h], reach[r, h] = top + np.log(e.sum()), scale * (np.abs(kh) @ np.abs(qh)).max()
    return out, lse, mass, reach
