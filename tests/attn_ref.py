"""Plain 64-bit forms of the paged-cache operators (numpy), and bounds on the
kernels' rounding derived from their arithmetic."""
import numpy as np

# unit roundoff of the element types (8 and 11 significant bits)
UNIT = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}


def kv_map(ctx, new, table, page, free, head, n_tok):
    """Sequential statement of cf_kv_map's rules on Python integers."""
    table = np.array(table, np.int64)
    row_tokens = table.shape[1] * page
    q_start, kv_len, status = [0], [], []
    slots, pos = np.full(n_tok, -1, np.int64), np.zeros(n_tok, np.int64)
    at, head = max(int(head), 0), max(int(head), 0)
    for i, (c, m) in enumerate(zip(ctx, new)):
        c, m, first = int(c), int(m), q_start[-1]
        st = 0
        if c < 0 or m < 0 or c + m > row_tokens or first + m > n_tok:
            st = 1
        else:
            have, want = -(-c // page), -(-(c + m) // page)
            if want > have:
                at += want - have
                if at > len(free):
                    st = 2
                else:
                    table[i, have:want] = free[at - (want - have):at]
                    head = at
        for j in range(max(m, 0)):
            if first + j < n_tok:
                pos[first + j] = min(c + j, 2 ** 31 - 1)
                if st == 0:
                    p = table[i, (c + j) // page]
                    slots[first + j] = -1 if p < 0 else p * page + (c + j) % page
        q_start.append(first + max(m, 0))
        kv_len.append(c + m if st == 0 else 0)
        status.append(st)
    return dict(table=table, q_start=q_start, kv_len=kv_len, slots=slots, pos=pos, head=[head], status=status)


def attend(q, k, v, sees, scale, kind):
    """Attention of one sequence in 64 bits: q [n][H][D], k and v [m][Hkv][D], query j seeing
    keys 0 .. sees[j] - 1.  Returns out, lse and a bound on |kernel - out| and |kernel - lse|.

    The bound.  A score is an fp32 sum of exact products, off by at most (D + 4) 2^-24 sum
    |q_d k_d| scale =: e (the scale's and the base-2 factor's roundings among the 4 units), and
    exp2 by a few 2^-23: each weight is off by a factor within 1 +- (2 e + 2^-20).  Weights are
    rounded to the element type for the product with v (unit u; below the fp16 normal range by at
    most 2^-25, the row's largest weight being 1 or more), sums over m keys are fp32, and the output is rounded once: with A = sum p |v| /
    sum p, |error| <= (2 u + 2 (2 e + 2^-20) + (m + 64) 2^-23) A, the subnormal terms, and 2^-24
    for an output below the fp16 normal range."""
    n, H, D = q.shape
    m, Hkv, _ = k.shape
    out, lse = np.zeros((n, H, D)), np.full((n, H), -np.inf)
    tol, ltol = np.zeros((n, H, D)), np.zeros((n, H))
    u = UNIT[kind]
    for h in range(H):
        kh, vh = k[:, h * Hkv // H].astype(np.float64), v[:, h * Hkv // H].astype(np.float64)
        for j in range(n):
            s = min(max(int(sees[j]), 0), m)
            if s == 0:
                continue
            qj = q[j, h].astype(np.float64) * scale
            e = (np.abs(kh[:s]) @ np.abs(qj)).max() * (D + 4) * 2.0 ** -24
            x = kh[:s] @ qj
            top = x.max()
            p = np.exp(x - top)
            l = p.sum()
            out[j, h] = p @ vh[:s] / l
            lse[j, h] = top + np.log(l)
            rel = 2 * e + 2.0 ** -20
            A = p @ np.abs(vh[:s]) / l
            sub = 2.0 ** -25 * np.abs(vh[:s]).sum(0) / l if kind == "fp16" else 0.0
            tol[j, h] = (2 * u + 2 * rel + (m + 64) * 2.0 ** -23) * A + sub + 2.0 ** -24
            ltol[j, h] = rel + (m + 64) * 2.0 ** -23 + abs(lse[j, h]) * 2.0 ** -22 + 2.0 ** -20
    return out, lse, tol, ltol
