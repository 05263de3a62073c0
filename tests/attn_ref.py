"""Positions, rotation, paged cache and attention in 64 bits, element by element
of their definitions (tr.h), for the tests of paper_2607_13500_amd.attention.
Everything here runs on the CPU."""
import math
from fractions import Fraction

import torch


def kept_positions(idx, K, grid, start):
    cols, r = [], 0
    for k, (T, H, W), s in zip(K, grid, start):
        for n in idx[r:r + k].tolist():
            cols.append((s[0] + n // (H * W), s[1] + n // W % H, s[2] + n % W))
        r += k
    return torch.tensor(cols, dtype=torch.int64).reshape(-1, 3).t()


SCALE = 1 << 150
TURN = round(Fraction("6.28318530717958647692528676655900576839433879875021") * SCALE)


def angles(pos, inv_freq, pair_axis):
    """[tokens, pairs] angles, the fp32 products of positions and frequencies; pos
    int [axes, tokens].  Whole turns are taken out in integers of 2^-150, so that
    large angles keep their bits."""
    out = torch.empty(pos.shape[1], len(inv_freq), dtype=torch.float64)
    for i, (f, a) in enumerate(zip(inv_freq, pair_axis)):
        z = pos[a].float() * torch.tensor(f, dtype=torch.float32)
        ratios = [v.as_integer_ratio() for v in z.double().tolist()]
        out[:, i] = torch.tensor([(n * (SCALE // d) % TURN) / SCALE for n, d in ratios], dtype=torch.float64)
    return out


def pairs(rot_dim, adjacent):
    """Element indices (first, second) of every pair."""
    n = rot_dim // 2
    return [(2 * i, 2 * i + 1) if adjacent else (i, i + n) for i in range(n)]


def turn(x, angle, rot_dim, adjacent):
    """x [tokens, heads, dim] turned by angle [tokens, pairs]."""
    y = x.clone()
    if rot_dim:
        ia, ib = (torch.tensor(v) for v in zip(*pairs(rot_dim, adjacent)))
        c, s = torch.cos(angle)[:, None, :], torch.sin(angle)[:, None, :]
        y[..., ia] = x[..., ia] * c - x[..., ib] * s
        y[..., ib] = x[..., ib] * c + x[..., ia] * s
    return y


def pair_norm(x, rot_dim, adjacent):
    """The length of the pair that each element belongs to (its own, unrotated)."""
    y = x.abs().clone()
    if rot_dim:
        ia, ib = (torch.tensor(v) for v in zip(*pairs(rot_dim, adjacent)))
        n = torch.sqrt(x[..., ia] ** 2 + x[..., ib] ** 2)
        y[..., ia] = n
        y[..., ib] = n
    return y


def norm(x, w, eps):
    r = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    return x * r * (1.0 if w is None else w)


def backward(g, x, w, angle, rot_dim, adjacent, eps, normed):
    """(dx, dw, and the sum of |terms| of dw)."""
    g = turn(g, -angle, rot_dim, adjacent)
    if not normed:
        return g, None, None
    r = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    u = x * r
    gw = g * (1.0 if w is None else w)
    return r * (gw - u * (gw * u).mean(-1, keepdim=True)), (g * u).sum((0, 1)), (g * u).abs().sum((0, 1))


def place(step, b, j, page_size):
    """(page, row) of token j of sequence b, or None outside the table."""
    q_start, kv_len, table = step
    if j < 0 or j // page_size >= table.shape[1]:
        return None
    return int(table[b, j // page_size]), j % page_size


def sequences(step):
    """(b, first packed row, new tokens, length in the cache)."""
    q_start, kv_len, _ = step
    for b in range(kv_len.numel()):
        t0, t1 = int(q_start[b]), int(q_start[b + 1])
        yield b, t0, t1 - t0, int(kv_len[b])


def attend(q, k_cache, v_cache, step, scale, causal, window):
    """(out, lse, sum of weight * |v|, largest |score|) in 64 bits for every
    packed row of a sequence; rows of none stay NaN."""
    T, heads, dim = q.shape
    page_size, kv_heads = k_cache.shape[1], k_cache.shape[2]
    group = heads // kv_heads
    out = torch.full((T, heads, dim), math.nan, dtype=torch.float64)
    lse = torch.full((T, heads), math.nan, dtype=torch.float64)
    mass, most = out.clone(), lse.clone()
    for b, t0, n, kv in sequences(step):
        if n <= 0:
            continue
        at = [place(step, b, j, page_size) for j in range(kv)]
        rows = torch.tensor([g * page_size + r for g, r in at], dtype=torch.long)
        k = k_cache.reshape(-1, kv_heads, dim)[rows].double()
        v = v_cache.reshape(-1, kv_heads, dim)[rows].double()
        for i in range(n):
            p = kv - n + i
            lo, hi = 0, kv
            if causal:
                hi = max(0, min(kv, p + 1))
                lo = max(0, p - window + 1) if window else 0
            for g in range(kv_heads):
                hs = slice(g * group, (g + 1) * group)
                x = q[t0 + i, hs].double()
                if hi <= lo:
                    out[t0 + i, hs], lse[t0 + i, hs], mass[t0 + i, hs], most[t0 + i, hs] = 0.0, -math.inf, 0.0, 0.0
                    continue
                s = scale * (x @ k[lo:hi, g].t())
                z = torch.logsumexp(s, 1)
                w = torch.where(torch.isinf(z)[:, None] & (z < 0)[:, None], torch.zeros_like(s), torch.exp(s - z[:, None]))
                out[t0 + i, hs] = w @ v[lo:hi, g]
                mass[t0 + i, hs] = w @ v[lo:hi, g].abs()
                lse[t0 + i, hs] = z
                most[t0 + i, hs] = s.abs().amax(1)
    return out, lse, mass, most
