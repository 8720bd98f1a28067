"""Plain 64-bit forms of the operators on caches and logits, and the bounds that
the kernels' 32-bit arithmetic keeps to them."""
import math

import numpy as np
import torch


def chain_masks(rows):
    return [[(2 << i) - 1 for i in range(r)] for r in rows]


def tree_masks(rows, rng):
    """Random trees: each row sees itself and its ancestors."""
    out = []
    for r in rows:
        m = []
        for i in range(r):
            p = int(rng.integers(-1, i)) if i else -1
            m.append((1 << i) | (m[p] if p >= 0 else 0))
        out.append(m)
    return out


def mask_tensor(masks, device="cuda"):
    flat = np.array([m for ms in masks for m in ms], dtype=np.uint64)
    return torch.from_numpy(flat.view(np.int64)).to(device)


def seen_matrix(L, masks):
    """bool [rows][L + rows]."""
    r = len(masks)
    s = np.zeros((r, L + r), dtype=bool)
    s[:, :L] = True
    for i, m in enumerate(masks):
        for j in range(r):
            s[i, L + j] = bool((m >> j) & 1)
    return torch.from_numpy(s)


def scores(q, k, seen, scale):
    """(scaled scores, -inf where not seen; bound of their 32-bit error), both
    [n_kv][rows][G][keys].  q [rows][n_q][d], k [n_kv][keys][d] in double."""
    r, nq, d = q.shape
    nkv = k.shape[0]
    qg = q.view(r, nkv, nq // nkv, d).permute(1, 0, 2, 3)
    vis = seen.to(q.device)[None, :, None, :]
    k0 = torch.where(seen.any(0).to(q.device)[None, :, None], k, torch.zeros_like(k))
    s = torch.einsum("gihd,gtd->giht", qg, k0) * scale
    # d products added in 32 bits, each addition off by at most 2^-23 of the sum
    # of magnitudes (truncating adders); queries as two bf16 parts: 2^-16
    mag = torch.einsum("gihd,gtd->giht", qg.abs(), k0.abs()) * scale
    return s.masked_fill(~vis, -math.inf), mag * (d * 2.0 ** -23 + 2.0 ** -16)


def attention(q, k, v, seen, scale):
    """(out [rows][n_q][d], its bound, lse [rows][n_q], its bound) in double for
    one request."""
    r, nq, d = q.shape
    nkv, n = k.shape[0], k.shape[1]
    s, ds = scores(q, k, seen, scale)
    some = seen.any(1).to(q.device)[None, :, None]
    lse = torch.where(some, torch.logsumexp(s, -1), torch.full_like(s[..., 0], -math.inf))
    p = torch.where(s == -math.inf, torch.zeros_like(s), torch.exp(s - torch.where(some, lse, torch.zeros_like(lse))[..., None]))
    v0 = torch.where(seen.any(0).to(q.device)[None, :, None], v, torch.zeros_like(v))
    out = torch.einsum("giht,gtd->gihd", p, v0)
    mag = torch.einsum("giht,gtd->gihd", p, v0.abs())
    worst = torch.where(s == -math.inf, torch.zeros_like(s), ds).amax(-1)
    # a weight is off by twice the scores' error, the exponential's 2^-20 (of
    # arguments up to 2^5) and its parts' 2^-15; the sums of n terms by n 2^-23 each
    rel = 2 * worst + 2.0 ** -20 + 2.0 ** -15 + 2 * n * 2.0 ** -23
    pack = lambda x: x.permute(1, 0, 2, 3).reshape(r, nq, -1)  # noqa: E731
    return (pack(out), pack(mag * rel[..., None]), pack(lse[..., None])[..., 0],
            pack((worst + 2.0 ** -20 + n * 2.0 ** -23 + lse.nan_to_num(0, 0, 0).abs() * 2.0 ** -22)[..., None])[..., 0])


def weights(q, k, seen, scale, lse):
    """(weights [n_kv][keys], bound) of one request in double; lse [rows][n_q]."""
    r, nq, d = q.shape
    nkv = k.shape[0]
    s, ds = scores(q, k, seen, scale)
    lg = lse.view(r, nkv, nq // nkv).permute(1, 0, 2)[..., None]
    p = torch.where(s == -math.inf, torch.zeros_like(s), torch.exp(s - torch.where(lg == -math.inf, 0.0, lg)))
    rel = torch.where(s == -math.inf, torch.zeros_like(s), ds) + 2.0 ** -20 + lg.nan_to_num(0, 0, 0).abs() * 2.0 ** -22
    n = r * nq // nkv
    return p.sum((1, 2)), (p * rel).sum((1, 2)) + p.sum((1, 2)) * n * 2.0 ** -23


def evict(k, v, w, lens, keep, recent):
    """In place on numpy arrays [layers][batch][n_kv][cap](...); new lengths."""
    new = list(lens)
    for b, (n, most) in enumerate(zip(lens, keep)):
        if n <= most or n < 0 or n > w.shape[3]:
            continue
        new[b] = most
        late = min(recent, most)
        for layer in range(w.shape[0]):
            for g in range(w.shape[2]):
                x = w[layer, b, g]
                old = n - late
                order = sorted(range(old), key=lambda t: (math.isnan(x[t]), -x[t] if not math.isnan(x[t]) else 0.0, t))
                at = np.array(sorted(order[:most - late]) + list(range(old, n)), dtype=np.int64)
                for a in (k, v, w):
                    a[layer, b, g, :most] = a[layer, b, g, at]
    return new


def accept(probs, draft, cand, ks, u):
    """(n_accepted, token) lists from float64 arrays of the given floats."""
    ns, toks, r, c = [], [], 0, 0
    V = probs.shape[1]
    for k in ks:
        n = 0
        while n < k:
            t = cand[c + n]
            if not 0 <= t < V:
                break
            q = draft[c + n, t] if draft is not None else 1.0
            if not u[r + n] * q < probs[r + n, t]:
                break
            n += 1
        p = probs[r + n].copy()
        x = p.copy()
        if n < k:
            if draft is not None:
                x = x - draft[c + n]
            elif 0 <= cand[c + n] < V:
                x[cand[c + n]] = 0.0
        tok = -1
        for y in (x, p):
            y = np.where(y > 0, y, 0.0)
            if y.sum() > 0:
                cdf = np.cumsum(y)
                tok = int(np.searchsorted(cdf, u[r + k] * cdf[-1], side="right"))
                break
        ns.append(n)
        toks.append(tok)
        r, c = r + k + 1, c + k
    return ns, toks
