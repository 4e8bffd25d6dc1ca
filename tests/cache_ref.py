"""Plain 64-bit references of the sampling and paged-cache operators (test infrastructure)."""
import math

import numpy as np
import torch


# ---- sampling ----------------------------------------------------------------------------------
def sample_row(l, mask_id, T, u, top_k=0, top_p=1.0, min_p=0.0):
    """(token, confidence) of one row of float64 logits, straight from the definition."""
    l = np.asarray(l, np.float64)
    ids = np.array([v for v in range(len(l)) if v != mask_id], dtype=np.int64)
    nan = bool(np.isnan(l[ids]).any()) if len(ids) else False
    ids = ids[~np.isnan(l[ids]) & (l[ids] > -np.inf)]
    if len(ids) == 0:
        return -1, (math.nan if nan else 0.0)
    order = ids[np.argsort(-l[ids], kind="stable")]
    top = l[order[0]]
    with np.errstate(invalid="ignore"):
        d = np.where(l[order] == top, 0.0, l[order] - top)
    pick = 0
    if T > 0:
        with np.errstate(invalid="ignore"):
            w = np.where(d == -np.inf, 0.0, np.exp(np.maximum(d, -1e300) / T))
        if top_k > 0:
            w = w[:top_k]
        n, c = len(w), np.cumsum(w)
        if top_p < 1:
            n = min(n, 1 + int(np.sum(c < top_p * c[-1])))
        if min_p > 0:
            n = min(n, max(1, int(np.sum(w >= min_p))))
        pick = min(int(np.sum(c[:n] <= u * c[n - 1])), n - 1)
    e = np.exp(d)
    return int(order[pick]), (math.nan if nan else float(e[pick] / e.sum()))


# ---- pages --------------------------------------------------------------------------------------
def k_offset(p, d, hd):
    k = p % 32
    return (p // 32) * 32 * hd + (k // 4 % 2) * 16 * hd + (d // 32) * 512 + (d // 8 % 4) * 128 \
        + (4 * (k // 8) + k % 4) * 8 + d % 8


def v_offset(p, d, hd):
    k = p % 32
    return (p // 32) * 32 * hd + (d // 16) * 512 + (k // 8) * 128 + (d % 16) * 8 + k % 8


def offsets(page, hd):
    p, d = np.arange(page)[:, None], np.arange(hd)[None, :]
    return (torch.from_numpy(k_offset(p, d, hd) + 0 * d).long(),
            torch.from_numpy(v_offset(p, d, hd) + 0 * d).long())


def natural(pages, offs):
    """[..., page * hd] in operand order -> [..., page, hd]."""
    return pages[..., offs.reshape(-1).to(pages.device)].reshape(*pages.shape[:-1], *offs.shape)


def operand(nat, offs):
    """The inverse of natural."""
    out = torch.empty(*nat.shape[:-2], offs.numel(), dtype=nat.dtype, device=nat.device)
    out[..., offs.reshape(-1).to(nat.device)] = nat.reshape(*nat.shape[:-2], -1)
    return out


class Plan:
    """The planner's state on the host, request by request."""

    def __init__(self, batch, max_pages, n_pages, page):
        self.table = np.full((batch, max_pages), -1, np.int64)
        self.len = np.zeros(batch, np.int64)
        self.free = list(range(n_pages - 1, -1, -1))
        self.n_pages, self.page, self.max_pages, self.B = n_pages, page, max_pages, batch

    def step(self, start, count, rows, reset=False):
        P = self.page
        if reset:
            self.len[:] = 0
            self.free = list(range(self.n_pages - 1, -1, -1))
        for b in range(self.B):
            if count[b] < 0:
                n = -(-int(self.len[b]) // P)
                self.free += [int(x) for x in self.table[b, :n]]
                self.len[b] = 0
        cu, pos, slots, status = [0], [], [], np.zeros(self.B, np.int64)
        n_free, asked_pages, asked_rows = len(self.free), 0, 0
        for b in range(self.B):
            s, c = int(start[b]), max(int(count[b]), 0)
            if c > 0:
                if s < 0 or s > self.len[b] or s + c > self.max_pages * P:
                    status[b] = -1
                else:
                    have = -(-int(self.len[b]) // P)
                    need = max(0, -(-(s + c) // P) - have)
                    asked_pages += need
                    asked_rows += c
                    if need > 0 and asked_pages > n_free:
                        status[b] = -3
                    elif asked_rows > rows:
                        status[b] = -2
                    else:
                        for j in range(have, have + need):
                            self.table[b, j] = self.free.pop()
                        self.len[b] = max(self.len[b], s + c)
                        for p in range(s, s + c):
                            pos.append(p)
                            slots.append(int(self.table[b, p // P]) * P + p % P)
            cu.append(len(pos))
        pad = [-1] * (rows - len(pos))
        return {"cu": cu, "positions": pos + pad, "slots": slots + pad, "status": status}


# ---- attention -----------------------------------------------------------------------------------
def attend(q, k, v, lens, start, cu, group, causal, scale):
    """q [T, H, hd], k and v lists of [len, Hkv, hd], all float64.  Returns the output, the sum of
    p |v| behind each element and a bound on the error that fp32 scores put on a term."""
    out = torch.zeros_like(q)
    mag = torch.zeros_like(q)
    dev = torch.zeros(q.shape[:2], dtype=torch.float64, device=q.device)
    hd = q.shape[-1]
    for b, n in enumerate(lens):
        rows = range(cu[b], cu[b + 1])
        for h in range(q.shape[1]):
            if len(rows) == 0:
                continue
            qq = q[cu[b]:cu[b + 1], h]
            kk, vv = k[b][:n, h // group], v[b][:n, h // group]
            s = qq @ kk.T * scale
            if causal:
                lim = start[b] + torch.arange(len(rows), device=q.device)
                s = s.masked_fill(torch.arange(n, device=q.device)[None, :] > lim[:, None], -math.inf)
            if n == 0:
                continue
            top = s.amax(dim=1, keepdim=True)
            e = torch.exp(s - torch.where(top == -math.inf, torch.zeros_like(top), top))
            p = e / e.sum(dim=1, keepdim=True).clamp_min(1e-300)
            out[cu[b]:cu[b + 1], h] = p @ vv
            mag[cu[b]:cu[b + 1], h] = p @ vv.abs()
            # fp32: hd products and sums, then scale and max: each 2^-24 of the sum of magnitudes
            dev[cu[b]:cu[b + 1], h] = (qq.abs() @ kk.abs().T * scale).amax(dim=1) * (hd + 4) * 2.0 ** -24
    return out, mag, dev


def attend_tolerance(out, mag, dev):
    """Terms rounded to bf16 (2^-8 of each), their exponents off by dev above and below the
    division and by 2^-21 in the hardware's exponential, the result rounded to bf16."""
    return 2.0 ** -8 * (mag + out.abs()) + mag * (2 * dev[..., None] + 2.0 ** -20) + 1e-30
