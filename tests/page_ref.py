"""The paged 8-bit cache in plain 64-bit arithmetic: what is held of a sequence's rows, attention over it, block tables."""
import math

import numpy as np
import torch

PAGE = 128
LARGEST = 448.0 * 2.0 ** 119             # of a page: the next e4m3 number times a power of two is past bf16's
HALF_BF16, HALF_F32 = 2.0 ** -8, 2.0 ** -24            # half a step, relative to the value


def finite(rows):
    x = rows.double()
    return torch.where(torch.isnan(x), torch.zeros_like(x), x.clamp(-LARGEST, LARGEST))


def e4m3(x):
    """Nearest e4m3 number, ties to even, of values up to 448."""
    step = 2.0 ** (torch.clamp(torch.frexp(x)[1] - 1, min=-6).double() - 3)
    return torch.round(x / step) * step


def held(rows):
    """rows [L, heads, d] of one sequence -> float64 of the same shape."""
    x = finite(rows)
    full = x.shape[0] // PAGE * PAGE
    out = x.clone()
    for first in range(0, full, PAGE):
        for h in range(x.shape[1]):
            block = x[first:first + PAGE, h]
            e = -100
            while float(block.abs().max()) > 448.0 * 2.0 ** e:
                e += 1
            out[first:first + PAGE, h] = e4m3(block / 2.0 ** e) * 2.0 ** e
    return out


def attend(q, k, v, positions, scale, cap=0.0, slopes=None, prefix=0):
    """q [n, H_q, d] at positions, k, v [L, H_kv, d]: outputs, log-sum-exps, and for tolerances sum p |v| and the largest magnitudes of a
    row's scores: of the sum of |q k| and of the finished ones."""
    n, hq, d = q.shape
    length, hkv, _ = k.shape
    g = hq // hkv
    kk, vv = k.repeat_interleave(g, 1).transpose(0, 1), v.repeat_interleave(g, 1).transpose(0, 1)
    qq = q.double().transpose(0, 1)
    s = torch.bmm(qq, kk.transpose(1, 2).contiguous()) * scale
    size = torch.bmm(qq.abs(), kk.abs().transpose(1, 2).contiguous()) * scale
    if cap:
        s = cap * torch.tanh(s / cap)
    keys, pos = torch.arange(length), torch.as_tensor(positions)
    seen = (keys[None] <= pos[:, None]) | (keys < prefix)[None]
    if slopes is not None:
        s = s + slopes.double()[:, None, None] * (keys[None] - pos[:, None])[None]
    s = torch.where(seen[None], s, -math.inf)
    lse = torch.logsumexp(s, 2)
    p = torch.exp(s - lse[:, :, None])
    top = torch.where(seen[None], s.abs() * (p > 1e-9), 0.0).amax(2)
    size = torch.where(seen[None], size, 0.0).amax(2)
    t = lambda x: x.transpose(0, 1).contiguous()
    return t(torch.bmm(p, vv)), t(lse), t(torch.bmm(p, vv.abs())), t(size), t(top)


def tolerances(out, lse, mean_abs, size, top, length, d, out_half, p_half, cap=0.0):
    """Largest errors of (outputs, log-sum-exps).  A score: d products added in fp32, at most (d + 4) half steps of the sum of magnitudes, four more of
    the finished score (scaling to base 2, bias, difference to the maximum), and with a cap four of the cap.  A probability is off
    by that, relatively, and by p_half on its way into the second product; sums over the keys are off by at most a half step per key.
    Probabilities below 2^-126 are zeros in fp32: 2^-126 of the values per key, far below 2^-100 in all (a row whose one
    seen value is 0 has no other part)."""
    ds = HALF_F32 * ((d + 4) * size + 8 * top + 4 * cap + 8)
    sums = HALF_F32 * (length + 16)
    return (2.0 ** -100 + out.abs() * out_half + mean_abs * (2 * ds + 2 * sums + p_half)[..., None],
            ds + sums + HALF_F32 * 4 * lse.abs())


def grow(len0, n_new, free, n_free, table):
    """Lengths, free pages left, table, row_start, slots, positions."""
    table, slots, positions, starts = table.copy(), [], [], [0]
    for b, (c, n) in enumerate(zip(len0, n_new)):
        for blk in range(c // PAGE, (c + n) // PAGE):
            n_free -= 1
            table[b, blk] = free[n_free]
        for p in range(c, c + n):
            slots.append(table[b, p // PAGE] * PAGE + p % PAGE if p // PAGE < (c + n) // PAGE else -1 - (b * PAGE + p % PAGE))
            positions.append(p)
        starts.append(starts[-1] + n)
    return np.array(len0) + np.array(n_new), n_free, table, np.array(starts), np.array(slots, dtype=np.int64), np.array(positions)
