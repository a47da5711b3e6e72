"""Plain fp64 forms of rotated appends and of attention with a window (numpy on the CPU, one sequence at a time), for their tests."""
import numpy as np

import verifier_ref as ref


def angles(position, freq):
    """position [rows, axes] whole numbers, freq [axes, pairs] -> angles [rows, pairs] in radians, and how far one worked out in fp64 and then reduced
    to fp32 may be from them: three roundings of the turns in fp64, half a step of fp32 at up to half a turn."""
    p, f = np.asarray(position, np.longdouble), np.asarray(freq, np.longdouble)
    a = (p[:, :, None] * f[None]).sum(1)
    size = (np.abs(p)[:, :, None] * np.abs(f)[None]).sum(1)
    turn = 2 * np.pi
    return a, np.float64(size * (2 + f.shape[0]) * 2.0 ** -53 + turn * 2.0 ** -26)


def turned(x, position, freq, interleaved, gain):
    """x [rows, heads, D] -> turned numbers, and what they may be off by in fp32 before they are rounded: the angle's error, two units of cosine
    and sine in the last place, the gain's rounding, two products and their sum."""
    x = np.asarray(x, np.float64)
    a, ea = angles(position, freq)
    pairs = a.shape[1]
    c, s = gain * np.cos(a).astype(np.float64)[:, None], gain * np.sin(a).astype(np.float64)[:, None]
    first, second = (slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2)) if interleaved else (slice(0, pairs), slice(pairs, 2 * pairs))
    u, v = x[..., first], x[..., second]
    y, tol = x.copy(), np.zeros_like(x)
    y[..., first], y[..., second] = u * c - v * s, u * s + v * c
    tol[..., first] = tol[..., second] = (np.abs(u) + np.abs(v)) * abs(gain) * (ea[:, None] + 5 * 2.0 ** -24)
    return y, tol


def sees(i, slots, base, n, position, mask_row, window, sinks):
    """Which of the slots row i sees.  position: the rows' own (None: a chain), mask_row: truth values over new rows."""
    j = slots - base
    pos = (lambda r: base + r) if position is None else (lambda r: np.clip(np.asarray(position)[r], base, base + r))
    new = (j >= 0) & (j < n)
    at = np.where(j < 0, slots, pos(np.clip(j, 0, max(n - 1, 0))) if n else slots)
    if mask_row is None:
        there = (j < 0) | (new & (j <= i))
    else:
        there = (j < 0) | (new & (j < len(mask_row)) & mask_row[np.clip(j, 0, len(mask_row) - 1)])
    return there & ((pos(i) - at < window) | (at < sinks))


def held_ok(back, exps, y, tol):
    """Whether e4m3 entries (values `back`, exponent bytes `exps` a row) are roundings of numbers that are within tol of y."""
    amax, most = np.abs(y).max(-1), tol.max(-1)
    lo, hi = (ref.quantise_rows(np.maximum(amax + d * most, 0)[..., None])[1] for d in (-1, 1))
    e = exps.astype(np.int64)
    scale = np.ldexp(1.0, e - 127)[..., None]
    # half a step of three bits behind the leading one, or of the least exponent's
    near = np.abs(back - y) <= tol + np.maximum((np.abs(y) + tol) * 2.0 ** -4, scale * 2.0 ** -10)
    return bool(near.all() and ((e >= lo) & (e <= hi)).all())
