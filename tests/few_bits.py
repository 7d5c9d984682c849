"""Plain statements in 64 bits, on the CPU, of what the calls on few-bit values compute; shared by their tests."""
import math

import numpy as np
import torch

HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}    # of a rounding, relative


def quantize_group(x):
    """lo, step (numbers of x's type, as floats) and codes of 64 values."""
    v = [float(e) for e in x]
    if not all(math.isfinite(e) for e in v) or max(v) - min(v) > 3.4028234663852886e38:
        return math.nan, math.nan, [0] * 64
    lo, span = min(v) + 0.0, max(v) - min(v)                # (a zero of either sign is held as +0)
    if span < 15 * 2.0 ** -126:
        return lo, 0.0, [0] * 64
    step = torch.tensor(span / 15, dtype=torch.float64).to(x.dtype)
    while 15 * float(step) < span:
        step = next_up(step)
    while 15 * float(next_down(step)) >= span:
        step = next_down(step)
    s = float(step)
    return lo, s, [sum(1 for i in range(15) if (e - lo) > (i + 0.5) * s) for e in v]


def next_up(t):
    return (t.view(torch.int16) + 1).view(t.dtype)


def next_down(t):
    return (t.view(torch.int16) - 1).view(t.dtype)


def held_value(x):
    """What a 4-bit cache holds for x, [..., 64 * groups], in fp64. (Vectorised form of quantize_group, which it is tested against.)"""
    v = x.double().unflatten(-1, (-1, 64))
    lo, span = v.amin(-1, keepdim=True), v.amax(-1, keepdim=True) - v.amin(-1, keepdim=True)
    step = (span / 15).to(x.dtype)
    step = torch.where(15 * step.double() < span, next_up(step), step).double()
    step = torch.where(span < 15 * 2.0 ** -126, 0.0, step)
    codes = sum(((v - lo) > (i + 0.5) * step).double() for i in range(15))
    codes = torch.where(step > 0, codes, 0.0)
    out = lo + step * codes
    bad = ~torch.isfinite(span) | (span > 3.4028234663852886e38)
    return torch.where(bad, math.nan, out).flatten(-2)


def cache_bytes(k, v):
    """The bytes of a page and head that hold k and v, [tokens (a multiple of 16), head_dim]."""
    out = bytearray()
    groups = k.shape[1] // 64
    for t0 in range(0, k.shape[0], 16):
        for x in (k, v):
            got = [[quantize_group(x[t0 + t, 64 * j: 64 * j + 64]) for j in range(groups)] for t in range(16)]
            for j in range(groups):
                for t in range(16):
                    c = got[t][j][2]
                    out += bytes(c[i] | c[i + 1] << 4 for i in range(0, 64, 2))
            for t in range(16):
                for j in range(groups):
                    out += torch.tensor(got[t][j][:2], dtype=x.dtype).view(torch.uint8).numpy().tobytes()
    return np.frombuffer(bytes(out), np.uint8)


def attend(q, k, v, scale, length, runs):
    """One sequence: q [runs, heads, dim], k and v [length, kv heads, dim] in fp64. Returns out, lse, and for the tolerance the
    weighted mean of |v| and the largest |scale * q . k| bound of each row."""
    rows, heads, dim = q.shape
    group = heads // max(k.shape[1], 1)
    out, lse = torch.zeros(rows, heads, dim, dtype=torch.float64), torch.full((rows, heads), -math.inf, dtype=torch.float64)
    mean = torch.zeros(rows, heads, dim, dtype=torch.float64)
    for i in range(rows):
        n = length - rows + i + 1
        if n <= 0:
            continue
        s = torch.einsum("nkd,kgd->kgn", k[:n], q[i].double().unflatten(0, (-1, group))) * scale
        lse[i] = torch.logsumexp(s, -1).flatten()
        p = torch.softmax(s, -1)
        out[i] = torch.einsum("kgn,nkd->kgd", p, v[:n]).flatten(0, 1)
        mean[i] = torch.einsum("kgn,nkd->kgd", p, v[:n].abs()).flatten(0, 1)
    return out, lse, mean


def quantize_rows(x):
    v = x.double()
    top = v.abs().amax(-1, keepdim=True)
    fine = torch.isfinite(top)
    some = fine & (top >= 127 * 2.0 ** -126)
    codes = torch.where(some, torch.round(v * 127 / torch.where(some, top, 1.0)), 0.0)
    scale = torch.where(some, top / 127, torch.where(fine, 0.0, math.nan))
    return codes, scale.squeeze(-1)
