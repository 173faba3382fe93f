"""Beam search's selection and the reordering of the beams' states, as plain
loops over float64 scores (the decode step of the encoder-decoder models the
paper runs on translation and summarisation, Sec. 4.1).

c(b, v) = score_b + logits[b, v] - ln sum_u exp logits[b, u]; a finished beam
continues only with the end token, at its score. Candidates that are NaN or
-inf do not count; equal ones go to the lower beam. Within a beam the order is that
of the logits, then of the tokens (the lower first), also where float64 sums of
different logits are equal."""
import numpy as np


def beam_select(logits, scores, n_out, finished=None, eos=None):
    """logits [B, K, V], scores [B, K]. Returns (parent [B, n_out] as rows
    b*K + beam, token, score, finished); -1, -1, -inf, 0 where none is left."""
    logits = np.asarray(logits, dtype=np.float64)
    scores = np.asarray(scores, dtype=np.float64)
    B, K, V = logits.shape
    parent = np.full((B, n_out), -1, dtype=np.int64)
    token = np.full((B, n_out), -1, dtype=np.int64)
    score = np.full((B, n_out), -np.inf)
    done = np.zeros((B, n_out), dtype=np.int64)
    for b in range(B):
        cand = []
        for k in range(K):
            s = scores[b, k]
            if finished is not None and finished[b, k]:
                if s > -np.inf:
                    cand.append((-s, k, 0.0, eos))
                continue
            z = logits[b, k]
            if not np.isfinite(s) and not s > 0:           # -inf, NaN
                continue
            if np.isnan(z).any() or (z == np.inf).any() or not (z > -np.inf).any():
                continue
            m = z.max()
            lse = m + np.log(np.sum(np.exp(z - m)))
            c = s + (z - lse)
            # the n_out best of a row are enough; a stable sort keeps low tokens first
            for v in np.argsort(-z, kind="stable")[:n_out]:
                if c[v] > -np.inf:
                    cand.append((-c[v], k, -z[v], int(v)))
        cand.sort()
        for j, (c, k, _, v) in enumerate(cand[:n_out]):
            parent[b, j], token[b, j], score[b, j] = b * K + k, v, -c
            if eos is not None:
                done[b, j] = int(v == eos or bool(finished is not None and finished[b, k]))
    return parent, token, score, done


def beam_reorder(cache, parent, K, lens=None):
    """cache [L, R, S, ...], R = B*K rows. Returns (new cache, new lens, bad):
    row r holds the first lens[parent[r]] positions of row parent[r] of the old
    cache; a parent of -1 keeps the row, one outside the request too (bad)."""
    cache = np.asarray(cache)
    out = cache.copy()
    R, S = cache.shape[1:3]
    lens = np.full(R, S) if lens is None else np.asarray(lens)
    new_lens = lens.copy()
    bad = False
    for r in range(R):
        p = int(parent[r])
        if p == -1:
            continue
        if p < 0 or p >= R or p // K != r // K:
            bad = True
            continue
        n = min(max(int(lens[p]), 0), S)
        out[:, r, :n] = cache[:, p, :n]
        new_lens[r] = lens[p]
    return out, new_lens, bad
