"""Causal attention of packed sequences, a cache of 4-bit blocks with the attention
over it, and log-probabilities of tokens, as plain float64 loops (what surrounds the
MoE layer of Sec. 2.1 in the blocks of the models the paper runs).

Queries without keys give zeros and a log-sum-exp of -inf."""
import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def softmax_rows(s, v):
    """One query: scores s [n], values v [n, D] -> (out [D], lse)."""
    if len(s) == 0 or not (s > -np.inf).any() and not np.isnan(s).any():
        return np.zeros(v.shape[1]), -np.inf
    p = np.exp(s - s.max())
    return p @ v / p.sum(), s.max() + np.log(p.sum())


def prompt_attention(q, k, v, q_offsets, k_offsets, scale, out=None, lse=None):
    """q [N, Hq, D], k and v [M, Hkv, D]; offsets [B+1]. Rows of no sequence keep what
    out and lse (zeros and -inf) hold."""
    q, k, v = (np.asarray(a, dtype=np.float64) for a in (q, k, v))
    N, Hq, D = q.shape
    n_q = Hq // k.shape[1]
    out = np.zeros((N, Hq, D)) if out is None else np.array(out, dtype=np.float64)
    lse = np.full((N, Hq), -np.inf) if lse is None else np.array(lse, dtype=np.float64)
    for b in range(len(q_offsets) - 1):
        n, m = q_offsets[b + 1] - q_offsets[b], k_offsets[b + 1] - k_offsets[b]
        for i in range(n):
            keys = slice(k_offsets[b], k_offsets[b] + max(0, m - n + i + 1))
            for h in range(Hq):
                at = (q_offsets[b] + i, h)
                out[at], lse[at] = softmax_rows(scale * (k[keys, h // n_q] @ q[at]),
                                                v[keys, h // n_q])
    return out, lse


def kv4_encode(x):
    """x [..., D] float -> (codes [..., D/2], scales [..., D/32]) uint8."""
    x = np.asarray(x, dtype=np.float64)
    y = x.reshape(x.shape[:-1] + (x.shape[-1] // 32, 32))
    codes = np.zeros(y.shape, dtype=np.uint8)
    scales = np.zeros(y.shape[:-1], dtype=np.uint8)
    for at in np.ndindex(scales.shape):
        b = y[at]
        if not np.isfinite(b).all():
            scales[at] = 255
            continue
        e = -124
        while e < 125 and np.abs(b).max() > 7 * 2.0 ** e:
            e += 1
        scales[at] = e + 127
        d = np.abs(np.abs(b)[:, None] / 2.0 ** e - E2M1)     # exact: a power of two
        for i in range(32):
            near = np.flatnonzero(d[i] == d[i].min())        # two of a tie: the even one
            c = near[0] if len(near) == 1 else near[near % 2 == 0][0]
            codes[at + (i,)] = c + 8 * int(np.signbit(b[i]))
    codes = codes.reshape(x.shape)
    return codes[..., 0::2] | codes[..., 1::2] << 4, scales


def kv4_decode(codes, scales):
    c = np.stack([codes & 15, codes >> 4], -1).reshape(codes.shape[:-1] + (2 * codes.shape[-1],))
    unit = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return np.where(c & 8, -1.0, 1.0) * E2M1[c & 7] * np.repeat(unit, 32, axis=-1)


def kv4_attention(q, cache, cache_row, lens, scale):
    """q [R, Hq, D]; cache (k_codes, k_scales, v_codes, v_scales) of [C, S, Hkv, .]."""
    q = np.asarray(q, dtype=np.float64)
    R, Hq, D = q.shape
    n_q = Hq // cache[0].shape[2]
    out, lse = np.zeros((R, Hq, D)), np.full((R, Hq), -np.inf)
    for r in range(R):
        if not 0 <= cache_row[r] < len(cache[0]):
            continue
        k, v = (kv4_decode(cache[2 * j][cache_row[r], :lens[r]],
                           cache[2 * j + 1][cache_row[r], :lens[r]]) for j in range(2))
        for h in range(Hq):
            out[r, h], lse[r, h] = softmax_rows(scale * (k[:, h // n_q] @ q[r, h]), v[:, h // n_q])
    return out, lse


def token_logprobs(logits, tokens, n_top):
    """logits [R, V], tokens [R, m] -> (logprobs, entropy, top tokens, their logprobs)."""
    z = np.asarray(logits, dtype=np.float64)
    R, V = z.shape
    logp = np.full(tokens.shape, -np.inf)
    entropy = np.zeros(R)
    top = np.full((R, n_top), -1, dtype=np.int64)
    top_logp = np.full((R, n_top), -np.inf)
    for r in range(R):
        inside = [(j, t) for j, t in enumerate(tokens[r]) if 0 <= t < V]
        if np.isnan(z[r]).any() or (z[r] == np.inf).any():
            entropy[r] = np.nan
            for j, _ in inside:
                logp[r, j] = np.nan
            continue
        live = z[r] > -np.inf
        if not live.any():
            continue
        m = z[r].max()
        total = np.sum(np.exp(z[r, live] - m))
        lp = z[r] - m - np.log(total)
        p = np.exp(lp[live])
        entropy[r] = -np.sum(p[p > 0] * lp[live][p > 0])
        for j, t in inside:
            logp[r, j] = lp[t]
        order = [v for v in np.argsort(-z[r], kind="stable")[:n_top] if live[v]]
        top[r, :len(order)], top_logp[r, :len(order)] = order, lp[order]
    return logp, entropy, top, top_logp
