"""Rotary positions and a cache held in 8 bits, plainly, on the CPU.  Angles and attention are in double precision; codes and scales are
defined in single precision, so those are computed in it and have to be equal."""
import math

import torch

HIGHEST = {"e4m3": 448.0, "int8": 127.0}
TYPE = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}
EPS = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}  # half a step, relative to the value


# ---------------------------------------------------------------------------------------------------------- rotation
def frequencies(d_rot, theta, scaling="plain", factor=1.0, low=0.0, high=0.0, context=0.0):
    if scaling == "base":
        theta = theta * factor ** (d_rot / (d_rot - 2))
    f = [theta ** (-2.0 * j / d_rot) for j in range(d_rot // 2)]
    if scaling == "linear":
        f = [x / factor for x in f]
    if scaling == "turns":
        t = [min(max((context * x / (2 * math.pi) - low) / (high - low), 0.0), 1.0) for x in f]
        f = [x * (y + (1 - y) / factor) for x, y in zip(f, t)]
    return torch.tensor(f, dtype=torch.float64)


def rotate(x, positions, f, layout, direction, amplitude):
    """x [b][N][heads][d], positions [b][N] -> (result in double, bound of its errors).

    The bound: a turn's fraction, at most a half, is rounded to fp32, which moves the angle by 2 pi 2^-25, and the sine and cosine of that are
    good to 2 steps, 2^-23: together under 2^-21; three roundings of 2^-24 for the amplitude, a product and the sum; the position
    times the frequency in double precision is off by 2^-51 of the angle; the result is rounded once."""
    m = len(f)
    y = x.double()
    idx = torch.arange(m)
    lo, hi = (idx, idx + m) if layout == "half" else (2 * idx, 2 * idx + 1)
    w = (positions.double()[..., None] * f)[:, :, None]
    s = 1.0 if direction == "forward" else -1.0
    a = 1.0 / amplitude if direction == "inverse" else amplitude
    out, reach = y.clone(), torch.zeros_like(y)
    out[..., lo] = a * (y[..., lo] * w.cos() - s * y[..., hi] * w.sin())
    out[..., hi] = a * (y[..., hi] * w.cos() + s * y[..., lo] * w.sin())
    reach[..., lo] = reach[..., hi] = a * (y[..., lo].abs() + y[..., hi].abs()) * (2.0 ** -21 + 3 * 2.0 ** -24 + w.abs() * 2.0 ** -51)
    half = EPS[x.dtype]
    turned = torch.zeros(x.shape[-1], dtype=torch.bool)
    turned[: 2 * m] = True
    return out, torch.where(turned, reach * (1 + half) + half * out.abs(), 0.0)


# -------------------------------------------------------------------------------------------------------------- codes
def encode(x, code):
    """fp32 numbers within the range of the codes -> codes, to nearest, ties to even."""
    return x.round().to(torch.int8) if code == "int8" else x.to(torch.float8_e4m3fn)


def append(new, n, count, codes, scales, c, code):
    """Rows new [N][d] (fp32) of one KV head into codes [L][d], scales [n_c], in place."""
    L, H = codes.shape[0], torch.tensor(HIGHEST[code])
    n, count = min(max(n, 0), L), min(max(count, 0), new.shape[0])
    end = min(n + count, L)
    for j in range(n // c, -(-end // c) if end > n else 0):
        r0, r1 = max(n, j * c), min(end, (j + 1) * c)
        x = new[r0 - n:r1 - n].float()
        top = x.abs().max()
        old = scales[j] if j * c < n else torch.tensor(0.0)
        s = old.clone()
        if not torch.isfinite(x).all():
            s = torch.tensor(math.nan)
        elif old == 0:
            s = torch.clamp(top / H, min=2.0 ** -126) if top > 0 else torch.tensor(0.0)
        else:
            assert not s < 0
            i = 0
            while top > H * s:
                s, i = s * 2, i + 1
            if i:
                codes[j * c:n] = encode(codes[j * c:n].float() * 2.0 ** -i, code)
        scales[j] = s
        codes[r0:r1] = encode(torch.zeros_like(x) if s == 0 or s.isnan() else x / s, code)


def rows(codes, scales, c):
    """What codes [..][L][d] and scales [..][n_c] stand for, in double precision (exactly)."""
    return codes.float().double() * scales.double().repeat_interleave(min(c, codes.shape[-2]), -1)[..., : codes.shape[-2], None]
