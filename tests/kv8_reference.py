"""Plain 64-bit statements of the 8-bit cache's operations (include/sssd_kv8.h), on the device of their inputs: what its tests compare with."""
import math

import torch

BLOCK = 32
LIMIT = {"e4m3": 448.0, "int8": 127.0}


def frequencies(rotary, base, scaling="none", factor=1.0, low=1.0, high=4.0, original=8192):
    """Radians per position."""
    f = [base ** (-2.0 * i / rotary) for i in range(rotary // 2)]
    if scaling == "linear":
        f = [x / factor for x in f]
    if scaling == "bands":
        w = [min(max((original * x / (2 * math.pi) - low) / (high - low), 0.0), 1.0) for x in f]
        f = [x * (a + (1 - a) / factor) for x, a in zip(f, w)]
    return torch.tensor(f, dtype=torch.float64)


def rotate(x, positions, freq, interleaved=False, magnitude=1.0):
    """x [..., heads, d], positions [...]."""
    r = 2 * len(freq)
    angle = positions.double()[..., None, None] * freq.to(x.device)
    y = x.double().clone()
    a, b = (y[..., 0:r:2].clone(), y[..., 1:r:2].clone()) if interleaved else (y[..., :r // 2].clone(), y[..., r // 2:r].clone())
    u, w = (a * angle.cos() - b * angle.sin()) * magnitude, (b * angle.cos() + a * angle.sin()) * magnitude
    if interleaved:
        y[..., 0:r:2], y[..., 1:r:2] = u, w
    else:
        y[..., :r // 2], y[..., r // 2:r] = u, w
    return y


def scale_of(most, fmt):
    """The smallest power of two s >= 2^-126 with most <= limit * s, 1 for most = 0: found by halving and doubling."""
    if most == 0:
        return 1.0
    s = 1.0
    while most > LIMIT[fmt] * s:
        s *= 2
    while s > 2.0 ** -126 and most <= LIMIT[fmt] * s / 2:
        s /= 2
    return s


def code_steps(y, fmt):
    """Distance of neighbouring codes at |y| (y = value / scale, before rounding)."""
    if fmt == "int8":
        return torch.ones_like(y)
    e = torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))).clamp(max=8)
    return torch.exp2(e - 3)


def rounded(y, fmt):
    """Nearest code, ties to even; infinities to the largest, what is no number to 0."""
    y = torch.nan_to_num(y.double(), nan=0.0, posinf=LIMIT[fmt], neginf=-LIMIT[fmt])
    step = code_steps(y, fmt)
    return torch.round(y / step) * step          # torch.round: half to even


def held(rows, fmt, scale=None):
    """rows [n <= 32][heads][d], live rows of one block: (values that are held, scale per head)."""
    x = rows.double()
    x = torch.where(x.abs() > 2.0 ** 127, torch.copysign(torch.full_like(x, float("inf")), x), x)
    most = torch.where(x.isfinite(), x.abs(), 0.0).amax((0, 2)) if len(x) else torch.zeros(x.shape[1], dtype=torch.float64)
    s = torch.tensor([scale_of(m, fmt) for m in most.tolist()], dtype=torch.float64, device=x.device)
    return rounded(x / s[:, None], fmt) * s[:, None], s


class Cache:
    """One layer of one sequence: K (or V) rows as they are held."""

    def __init__(self, heads, d, fmt, device="cpu"):
        self.x = torch.zeros(0, heads, d, dtype=torch.float64, device=device)
        self.fmt = fmt

    def append(self, length, rows):
        x = torch.cat([self.x[:length], rows.double().to(self.x.device)])
        out = [x[:length // BLOCK * BLOCK]]
        for a in range(length // BLOCK * BLOCK, len(x), BLOCK):
            out.append(held(x[a:a + BLOCK], self.fmt)[0])
        self.x = torch.cat(out)

    def commit(self, length, path):
        """Rows length + path[i] to length + 1 + i; both blocks written anew unless nothing moves."""
        if path != list(range(1, len(path) + 1)):
            x = torch.cat([self.x[:length + 1], self.x[[length + p for p in path]]])
            a = length // BLOCK * BLOCK
            self.x = torch.cat([x[:a]] + [held(x[i:i + BLOCK], self.fmt)[0] for i in range(a, len(x), BLOCK)])
        else:
            self.x = self.x[:length + 1 + len(path)]


def lines(parents, n):
    """For every new row the rows it sees, itself last."""
    out = []
    for j in range(n):
        up = [j]
        while up[-1] > 0:
            up.append(parents[up[-1]] if parents is not None else up[-1] - 1)
        out.append(up[::-1])
    return out


def attend(q, k, v, length, parents=None, window=0, sinks=0):
    """q [n][nq][d]; k, v [length + n][nkv][d] as they are held -> (out, sum of p |v|, largest sum of |q k| / sqrt(d))."""
    n, nq, d = q.shape
    nkv = k.shape[1]
    out, mass, size = (torch.zeros(n, nq, d, dtype=torch.float64, device=q.device) for _ in range(3))
    for j, line in enumerate(lines(parents, n)):
        at = list(range(length)) + [length + i for i in line]
        pos = len(at) - 1
        at = torch.tensor([a for p, a in enumerate(at) if not window or pos - p < window or p < sinks], device=q.device)
        qq = q[j].double().view(nkv, nq // nkv, 1, d)
        kk, vv = k[at].permute(1, 0, 2)[:, None], v[at].permute(1, 0, 2)[:, None]
        prod = qq * kk / math.sqrt(d)
        p = torch.softmax(prod.sum(-1), -1)[..., None]
        out[j] = (p * vv).sum(2).view(nq, d)
        mass[j] = (p * vv.abs()).sum(2).view(nq, d)
        size[j] = prod.abs().sum(-1).amax(-1).view(nq, 1)
    return out, mass, size
