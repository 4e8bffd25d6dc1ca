"""The beams' choice in 64 bits, straight from its definition (test infrastructure)."""
import math

import numpy as np


def beam_step(logits, K, W, mask_id, score, done=None, done_token=-1):
    """token, parent, score [B, W] of float64 logits [B K, V]."""
    R, V = logits.shape
    token, parent = np.full((R // K, W), -1, np.int64), np.full((R // K, W), -1, np.int64)
    out = np.full((R // K, W), -np.inf)
    for b in range(R // K):
        cand = []
        for r in range(b * K, b * K + K):
            s = float(score[r])
            if not (-math.inf < s < math.inf):
                continue
            if done is not None and done[r]:
                cand.append((-s, r, 0.0, done_token))
                continue
            ids = np.array([v for v in range(V) if v != mask_id], np.int64)
            l = logits[r][ids]
            if np.isnan(l).any() or (l == np.inf).any():
                continue
            ids, l = ids[l > -np.inf], l[l > -np.inf]
            if len(l) == 0:
                continue
            below = l - l.max()   # relative, so that logits of 1e38 keep the score's bits
            lse = np.log(np.exp(below).sum())
            best = np.argsort(-l, kind="stable")[:W]
            cand += [(-(s + (below[i] - lse)), r, -l[i] + 0.0, int(ids[i])) for i in best]
        for i, (s, r, _, v) in enumerate(sorted(cand)[:W]):
            token[b, i], parent[b, i], out[b, i] = v, r, -s
    return token, parent, out
