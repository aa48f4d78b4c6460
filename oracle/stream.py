"""Rotary positions and the paged 8-bit K/V cache (oracle side; test infrastructure).

Plain numpy in 64 bits, written from the definitions:

* rotary positions: pair i of an axis of d channels turns by pos * theta^(-2 i / d);
* the page allocator: a queue of free pages, streams served in order;
* the store: a run of tokens appended to a page, one power-of-two scale per page and head;
* attention of a stream's newest tokens over its cached ones.

Shares nothing with the GPU library.
"""

import numpy as np

from .fp8 import E4M3_MAX, e4m3_decode, e4m3_encode

EXP_MIN = -100


# ---- rotary positions -------------------------------------------------------


def rope_angles(ids, H, W, dims, origin, theta):
    """Angles [tokens, pairs] of token ids (int64); a negative id gives zeros."""
    ids = np.asarray(ids, dtype=np.int64)
    safe = np.maximum(ids, 0)
    pos = (origin[0] + safe // (H * W), origin[1] + safe // W % H, origin[2] + safe % W)
    cols = []
    for p, d in zip(pos, dims):
        freq = float(theta) ** (-2.0 * np.arange(d // 2) / d) if d else np.zeros(0)
        cols.append(p[:, None].astype(np.float64) * freq[None, :])
    return np.where(ids[:, None] < 0, 0.0, np.concatenate(cols, axis=1))


def rope_ref(x, angles, halves, inverse=False):
    """x [..., tokens, 128] (fp64) with its first 2 * pairs channels turned."""
    x = np.asarray(x, dtype=np.float64)
    r = 2 * angles.shape[-1]
    c, s = np.cos(angles), np.sin(angles) * (-1.0 if inverse else 1.0)
    y = x.copy()
    u_at = slice(0, r // 2) if halves else slice(0, r, 2)
    v_at = slice(r // 2, r) if halves else slice(1, r, 2)
    u, v = x[..., u_at], x[..., v_at]
    y[..., u_at], y[..., v_at] = u * c - v * s, u * s + v * c
    return y


# ---- pages ------------------------------------------------------------------


def plan_ref(held, fresh, state, ring, table, page, tokens):
    """(kv_len, q_start, slots, ids, state_out, table, ring) of one plan; inputs are not changed."""
    ring, table = list(ring), np.array(table)
    cap, width = len(ring), table.shape[1]
    head, count = int(state[0]), int(state[1])
    pages = lambda n: -(-n // page)  # noqa: E731
    kv_len, q_start, slots, ids = [], [0], [], []
    taken = wanted = refused = 0
    back = []
    for s, (n, add) in enumerate(zip(map(int, held), map(int, fresh))):
        if add < 0:
            kv_len.append(0)
            q_start.append(q_start[-1])
            back += [int(p) for p in table[s, : pages(n)]]
            continue
        need = pages(n + add) - pages(n)
        q_start.append(q_start[-1] + add)
        ok = n + add <= width * page
        if ok:
            wanted += need
            ok = need == 0 or wanted <= count
        if not ok:
            refused += 1
            kv_len.append(n)
            slots += [-1] * add
            ids += [-1] * add
            continue
        for i in range(need):
            table[s, pages(n) + i] = ring[(head + taken) % cap]
            taken += 1
        kv_len.append(n + add)
        for p in range(n, n + add):
            slots.append(int(table[s, p // page]) * page + p % page)
            ids.append(p)
    for i, p in enumerate(back):
        ring[(head + count + i) % cap] = p
    pad = [-1] * max(0, tokens - len(slots))
    out = [(head + taken) % cap, count - taken + len(back), refused]
    return (np.array(kv_len), np.array(q_start), np.array((slots + pad)[:tokens]), np.array((ids + pad)[:tokens]),
            np.array(out), table, np.array(ring))


# ---- store ------------------------------------------------------------------


def page_exponent(amax):
    """Smallest e >= EXP_MIN with amax <= 448 * 2^e."""
    if amax == 0:
        return EXP_MIN
    e = int(np.ceil(np.log2(amax / E4M3_MAX)))
    while np.ldexp(amax, -e) > E4M3_MAX:
        e += 1
    while np.ldexp(amax, -(e - 1)) <= E4M3_MAX:
        e -= 1
    return max(e, EXP_MIN)


def store_ref(x, slots, codes, exps):
    """x [rows, heads, 128] into copies of codes [pages, heads, page, 128] and exps [pages, heads]."""
    x = np.asarray(x, dtype=np.float64)
    codes, exps = np.array(codes), np.array(exps)
    page = codes.shape[2]
    runs = {}
    for r, s in enumerate(np.asarray(slots).ravel()):
        if 0 <= s < codes.shape[0] * page:
            runs.setdefault(int(s) // page, []).append((r, int(s) % page))
    for p, got in runs.items():
        rows, offs = [r for r, _ in got], [o for _, o in got]
        for h in range(codes.shape[1]):
            v = x[rows, h]
            e = page_exponent(np.abs(v).max())
            first = offs[0]
            if first:
                e = max(e, int(exps[p, h]))
                if e != exps[p, h]:
                    old = e4m3_decode(codes[p, h, :first])
                    codes[p, h, :first] = e4m3_encode(np.ldexp(old, int(exps[p, h]) - e))
            codes[p, h, offs] = e4m3_encode(np.ldexp(v, -e))
            exps[p, h] = e
    return codes, exps


def cached(codes, exps, table_row, n):
    """Values [n, heads, 128] of a stream's first n cached tokens."""
    page = codes.shape[2]
    pages = np.asarray(table_row[: -(-n // page)], dtype=np.int64)
    v = np.ldexp(e4m3_decode(codes[pages]), np.asarray(exps)[pages][:, :, None, None])
    return v.transpose(0, 2, 1, 3).reshape(-1, codes.shape[1], codes.shape[3])[:n]


# ---- attention --------------------------------------------------------------


def visible_keys(kv_len, q_len, i, frame, window):
    """[lo, hi) of row i."""
    p = kv_len - q_len + i
    end = (p // frame + 1) * frame if frame else kv_len
    return (max(0, end - window) if window else 0), min(end, kv_len)


def attn_ref(q, k, v, frame=0, window=0, scale=None):
    """(O, mass, reach) of one stream: q [rows, heads, 128], k, v [keys, kv heads, 128]. mass[i, h, d] is
    sum_j p_j |v_jd| and reach[i, h] the largest (sum_d |q_d k_jd| + max_d |q_d| sum_d |k_jd| / 16) * scale over visible
    keys: what rounding errors of P and of the scores are bounded with."""
    m, H, d = q.shape
    n, KH = k.shape[:2]
    scale = d ** -0.5 if scale is None else scale
    O, mass, reach = np.zeros((m, H, d)), np.zeros((m, H, d)), np.zeros((m, H))
    bounds = np.array([visible_keys(n, m, i, frame, window) for i in range(m)]).reshape(m, 2)
    sees = bounds[:, 1] > bounds[:, 0]
    if not sees.any():
        return O, mass, reach
    j = np.arange(n)
    hidden = (j < bounds[sees, :1]) | (j >= bounds[sees, 1:])
    for h in range(H):
        kk, vv, qq = k[:, h // (H // KH)], v[:, h // (H // KH)], q[sees, h]
        s = np.where(hidden, -np.inf, qq @ kk.T * scale)
        w = np.exp(s - s.max(-1, keepdims=True))
        w /= w.sum(-1, keepdims=True)
        O[sees, h], mass[sees, h] = w @ vv, w @ np.abs(vv)
        top = np.abs(qq).max(-1, keepdims=True) / 16 * np.abs(kk).sum(-1)
        reach[sees, h] = np.where(hidden, 0, np.abs(qq) @ np.abs(kk).T + top).max(-1) * scale
    return O, mass, reach


def attn_tolerance(O, mass, reach, half_step=2.0**-8):
    """Largest element error of attention with P and O rounded to a type of that half step and scores accumulated in
    fp32: |dO| <= half_step |O| (the output) + half_step mass (every P) + 2 ds mass (every score, numerator and
    denominator) with ds <= 128 * 2^-24 * reach from the sum of 128 products, 2^-20 * reach more for the scale, the
    base-2 argument and the exponential (the 2^-17 of reach's second term is what two E4M3 codes leave of Q: at most
    2^-21 of a row's largest element in every channel), and 2^-18 of both for the sums over keys."""
    ds = (2.0**-17 + 2.0**-20) * reach[..., None] + 2.0**-18
    return half_step * np.abs(O) + (half_step + 2 * ds) * mass + 1e-30
