"""Attention of rows that share a prefix of keys and values, each with a suffix of
its own, as plain loops in float64: softmax(scale q K^T) V over the keys of both
(the attention of the blocks that Sec. 2.1's MoE layer stands in). A row without
keys gives zeros and a log-sum-exp of -inf."""
import numpy as np


def prefix_attention(q, k_prefix, v_prefix, prefix_len, k_suffix, v_suffix, suffix_len, offsets,
                     scale, out=None, lse=None):
    """q [R, Hq, D]; prefix [G, P, Hkv, D], suffix [R, S, Hkv, D]; offsets [G+1]:
    rows of no group keep what out and lse (zeros and -inf) hold."""
    q = np.asarray(q, dtype=np.float64)
    R, Hq, D = q.shape
    Hkv = k_prefix.shape[2]
    out = np.zeros((R, Hq, D)) if out is None else np.array(out, dtype=np.float64)
    lse = np.full((R, Hq), -np.inf) if lse is None else np.array(lse, dtype=np.float64)
    for g in range(len(offsets) - 1):
        for r in range(offsets[g], offsets[g + 1]):
            for h in range(Hq):
                c = h // (Hq // Hkv)
                n, m = prefix_len[g], suffix_len[r]
                k = np.concatenate([k_prefix[g, :n, c], k_suffix[r, :m, c]]).astype(np.float64)
                v = np.concatenate([v_prefix[g, :n, c], v_suffix[r, :m, c]]).astype(np.float64)
                if len(k) == 0:
                    out[r, h], lse[r, h] = 0.0, -np.inf
                    continue
                s = scale * (k @ q[r, h])
                p = np.exp(s - s.max())
                out[r, h] = p @ v / p.sum()
                lse[r, h] = s.max() + np.log(p.sum())
    return out, lse
