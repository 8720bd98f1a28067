"""Plain 64-bit forms of the operators between a projection and its attention, and
the bounds that the kernels' arithmetic keeps to them."""
import math

import numpy as np
import torch


def scale_values():
    """The value of each of the 256 scale bytes."""
    byte = np.arange(256)
    v = np.where(byte < 8, byte * 2.0 ** -17, (1 + byte % 8 / 8) * 2.0 ** (byte // 8 - 15))
    return np.minimum(v, 896.0)


def pack(x):
    """(codes [.., d / 2] uint8, scale bytes [.., d / 16] uint8) of a double tensor."""
    x = torch.as_tensor(x).double()
    b = x.unflatten(-1, (x.shape[-1] // 16, 16))
    b = torch.where(b.isnan(), torch.zeros_like(b), b)
    table = torch.from_numpy(scale_values()[:0xC7]).to(x.device)
    # seven times a scale against the largest magnitude: no division, no rounding
    most = b.abs().amax(-1).contiguous()
    borders = 3.5 * (table[1:] + table[:-1])
    byte = torch.searchsorted(borders, most, right=False)
    at = byte.clamp(max=len(borders) - 1)
    byte = torch.where((byte < len(borders)) & (borders[at] == most) & (byte % 2 == 1), byte + 1, byte)
    s = table[byte][..., None]
    c = torch.where(s > 0, b / torch.where(s > 0, s, torch.ones_like(s)), torch.zeros_like(b))
    c = c.clamp(-7, 7).round().long() + 8
    nibble = torch.tensor([0, 4, 1, 5, 2, 6, 3, 7], device=x.device)  # of dim 0 .. 7 of a word
    w = (c.flatten(-2).unflatten(-1, (x.shape[-1] // 8, 8)) << (4 * nibble)).sum(-1)
    codes = torch.stack([(w >> (8 * i)) & 255 for i in range(4)], -1).flatten(-2)
    return codes.to(torch.uint8), byte.to(torch.uint8)


def unpack(codes, scales):
    """The values in double."""
    w = codes.long().unflatten(-1, (codes.shape[-1] // 4, 4))
    w = sum(w[..., i] << (8 * i) for i in range(4))
    c = torch.stack([(w >> (4 * n)) & 15 for n in (0, 4, 1, 5, 2, 6, 3, 7)], -1).flatten(-2) - 8
    s = torch.from_numpy(scale_values()).to(codes.device)[scales.long()]
    return c * s.repeat_interleave(16, -1)


def finish(x, gain, positions, rotary, eps, theta):
    """Rows [n][heads][d] normed and rotated in double, and twice that is no number: the
    values and the magnitudes |y_j| + |y_j'| that their errors go by."""
    x = x.double()
    if gain is not None:
        x = x / (x.pow(2).mean(-1, keepdim=True) + eps).sqrt() * gain.double()
    h = rotary // 2
    angle = positions.double()[:, None] * theta ** (-torch.arange(h, device=x.device).double() / max(h, 1))
    cos, sin = angle.cos()[:, None], angle.sin()[:, None]
    a, b, c = x[..., :h], x[..., h:rotary], x[..., rotary:]
    mag = torch.cat([a.abs() + b.abs()] * 2 + [c.abs()], -1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin, c], -1), mag


# Of 32-bit rows: a sum of squares in a chain of 12 additions and the root halve to 6 roundings
# of 2^-24, the division, the mean, eps and two products add 5, sines and cosines are off by 2^-21
# (two steps, and an angle rounded to 2^-25 of a half turn), the rotation adds 3.
FINISH = 2.0 ** -19


def attention(q, k, v, seen, scale, q_rel, p_rel):
    """(out [rows][n_q][d], its bound, lse [rows][n_q], its bound) of one request in
    double; q [rows][n_q][d], k and v [n_kv][keys][d], seen bool [rows][keys].  Queries
    are off by q_rel, weights by p_rel of themselves."""
    r, nq, d = q.shape
    nkv, n = k.shape[0], k.shape[1]
    seen = seen.to(q.device)
    qg = q.view(r, nkv, nq // nkv, d).permute(1, 0, 2, 3)
    k = torch.where(seen.any(0)[None, :, None], k, torch.zeros_like(k))
    v = torch.where(seen.any(0)[None, :, None], v, torch.zeros_like(v))
    out, tol, lses, tol_lse = [], [], [], []
    for g in range(nkv):
        s = torch.einsum("ihd,td->iht", qg[g], k[g]) * scale
        # d products added in 32 bits, each addition off by at most 2^-23 of the sum of
        # magnitudes (truncating adders)
        mag = torch.einsum("ihd,td->iht", qg[g].abs(), k[g].abs()) * scale * (d * 2.0 ** -23 + q_rel)
        s = s.masked_fill(~seen[:, None], -math.inf)
        worst = mag.masked_fill(~seen[:, None], 0).amax(-1, keepdim=True)
        lse = torch.logsumexp(s, -1, keepdim=True)
        p = torch.exp(s - torch.where(lse == -math.inf, torch.zeros_like(lse), lse))
        # a weight is off by twice the scores' error, the exponential's 2^-20 and its rounding (2^-31
        # of the largest where it is small); sums of n terms by n 2^-23
        rel = 2 * worst + 2.0 ** -20 + p_rel + 2 * n * 2.0 ** -23
        out.append(torch.einsum("iht,td->ihd", p, v[g]))
        tol.append(torch.einsum("iht,td->ihd", p, v[g].abs()) * rel +
                   2.0 ** -31 * torch.einsum("it,td->id", seen.double(), v[g].abs())[:, None])
        lses.append(lse[..., 0])
        tol_lse.append((worst + 2.0 ** -20 + n * 2.0 ** -23 + lse.nan_to_num(0, 0, 0).abs() * 2.0 ** -22)[..., 0])
    return torch.cat(out, 1), torch.cat(tol, 1), torch.cat(lses, 1), torch.cat(tol_lse, 1)


def causal(n, r):
    return torch.ones(r, n + r, dtype=torch.bool).tril(n)
