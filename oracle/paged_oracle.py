"""Plain implementations of the operators over a paged key-value cache, in Python integers and 64-bit floats, on the host.
Written from the definitions; shares no code with the library."""
import numpy as np


def kv_pages(lengths, new, table, free, state, page_size, tokens):
    """(lengths, granted, token offsets, ring state, slots, positions, table, ring) after the call; one request after the other."""
    R, wide = table.shape
    table, ring, F = table.copy(), np.array(free).copy(), len(free)
    first, available = int(state[0]), int(state[1])
    out_len, granted, offsets, slots, positions = [], [], [0], [], []
    asked = taken = back = 0
    for r in range(R):
        length, n = max(int(lengths[r]), 0), int(new[r])
        held = -(-length // page_size)
        offsets.append(offsets[-1] + max(n, 0))
        ok = n > 0 and length + n <= wide * page_size
        need = -(-(length + n) // page_size) - held if ok else 0
        asked += need
        ok = ok and (need == 0 or asked <= available) and offsets[-1] <= tokens
        if n < 0:
            for j in range(min(held, wide)):
                ring[(first + available + back) % F] = table[r, j]
                back += 1
        if ok:
            for j in range(need):
                table[r, held + j] = free[(first + taken + j) % F]
            taken += need
        for i in range(max(n, 0)):
            if offsets[-2] + i >= tokens:
                break
            row = length + i if ok else -1
            slots.append(int(table[r, row // page_size]) * page_size + row % page_size if ok else -1)
            positions.append(row)
        out_len.append(0 if n < 0 else length + n if ok else length)
        granted.append(n if ok else 0)
    pad = [-1] * (tokens - len(slots))
    return out_len, granted, offsets, [(first + taken) % F, available - taken + back], slots + pad, positions + pad, table, ring


def rows(x, weight, eps, positions, frequencies, interleaved):
    """Norm and rotation of x [..., tokens, heads, d]; and, of the same shape, |a| + |b| of the pair that each element comes from (|x| where
    it is not turned), which bounds the rounding of intermediate results."""
    x = np.asarray(x, dtype=np.float64).copy()
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(weight, dtype=np.float64)
    size = np.abs(x)
    half = 0 if frequencies is None else len(frequencies)
    if half:
        i = np.arange(half)
        ia, ib = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        # longdouble: the product is exact to far below the tolerance at any 32-bit position
        angle = np.asarray(positions, dtype=np.longdouble)[..., None, None] * np.asarray(frequencies, dtype=np.longdouble)
        cos, sin = np.cos(angle).astype(np.float64), np.sin(angle).astype(np.float64)
        a, b = x[..., ia].copy(), x[..., ib].copy()
        x[..., ia], x[..., ib] = a * cos - b * sin, a * sin + b * cos
        size[..., ia] = size[..., ib] = np.abs(a) + np.abs(b)
    return x, size


def decode(q, k, v, scale, lengths, window=0):
    """q [R, H, d]; k, v: per request [>= length, KH, d].  Returns O and, of the same shape, sum_j p_j |v_j| and, [R, H], the largest sum of
    |q_i k_i| of a visible row: what the rounding of scores and probabilities scales with."""
    R, H, d = q.shape
    o, size, score = np.zeros((R, H, d)), np.zeros((R, H, d)), np.zeros((R, H))
    for r in range(R):
        n = int(lengths[r])
        low = max(0, n - window) if window else 0
        if n <= 0:
            continue
        kr, vr = np.asarray(k[r][low:n], dtype=np.float64), np.asarray(v[r][low:n], dtype=np.float64)
        G = H // kr.shape[1]
        for h in range(H):
            s = kr[:, h // G] @ q[r, h].astype(np.float64) * scale
            p = np.exp(s - s.max())
            p /= p.sum()
            o[r, h], size[r, h] = p @ vr[:, h // G], p @ np.abs(vr[:, h // G])
            score[r, h] = (np.abs(kr[:, h // G]) @ np.abs(q[r, h].astype(np.float64))).max()
    return o, size, score
