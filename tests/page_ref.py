"""Plain float64 reference of page-scaled pools, of attention over K/V rows with and without a
causal mask, and bounds on what the stated roundings can do.  numpy on logical rows; independent
of the kernels."""

from __future__ import annotations

import numpy as np
import torch

PAGE = 16
HALF_BF16 = 2.0 ** -8  # half a bf16 step, relative to the value
F32 = 2.0 ** -24


def f64(t: torch.Tensor) -> np.ndarray:
    return t.detach().cpu().to(torch.float64).numpy()


def exponent(top: np.ndarray) -> np.ndarray:
    """Smallest e with top <= 448 * 2^e, held to [-117, 119]."""
    top = np.minimum(top, 3.5e38)
    m, x = np.frexp(top)
    return np.clip(np.where(top == 0, -117, np.where(m <= 0.875, x - 9, x - 8)), -117, 119)


def codes(y: np.ndarray) -> np.ndarray:
    """e4m3 codes (uint8) of values that float32 holds; torch's cast rounds to nearest even."""
    c = torch.from_numpy(np.clip(y, -448, 448).astype(np.float32)).to(torch.float8_e4m3fn)
    return c.view(torch.uint8).numpy()


def value(code: np.ndarray) -> np.ndarray:
    return torch.from_numpy(np.ascontiguousarray(code)).view(torch.float8_e4m3fn).to(torch.float64).numpy()


class PagePool:
    """A page-scaled pool: codes [pages, 16, heads, dim] and exponents [pages, heads], K and V alike."""

    def __init__(self, pages, heads, dim):
        self.code = [np.zeros((pages, PAGE, heads, dim), np.uint8) for _ in range(2)]
        self.exp = [np.full((pages, heads), -127, np.int64) for _ in range(2)]

    def store(self, pages_of, P, E, k, v):
        """pages_of(r): request r's page ids; k, v [T, heads, dim] float64."""
        at = 0
        for r, (p, e) in enumerate(zip(P, E)):
            ids = pages_of(r)
            for lp in range(p // PAGE, -(-(p + e) // PAGE)) if e else ():
                b, t = max(p - lp * PAGE, 0), min(p + e - lp * PAGE, PAGE)
                for i, rows in enumerate((k, v)):
                    x = np.zeros(self.code[i].shape[1:])
                    if b:
                        x[:b] = self.values(i, ids[lp])[:b]
                    x[b:t] = rows[at + lp * PAGE + b - p:at + lp * PAGE + t - p]
                    with np.errstate(invalid="ignore"):
                        ex = exponent(np.nanmax(np.abs(np.where(np.isnan(x), 0, x)), axis=(0, 2)))
                    self.exp[i][ids[lp]] = ex
                    self.code[i][ids[lp]] = codes(np.ldexp(x, -ex[None, :, None]))
            at += e

    def values(self, i, page):
        return np.ldexp(value(self.code[i][page]), self.exp[i][page][None, :, None])

    def rows(self, ids, first, count):
        """K and V [count, heads, dim] of tokens [first, first + count) of a sequence on pages ids."""
        out = []
        for i in range(2):
            pages = [self.values(i, ids[j]) for j in range(first // PAGE, -(-(first + count) // PAGE))]
            flat = np.concatenate(pages) if pages else np.zeros((0,) + self.code[i].shape[2:])
            out.append(flat[first % PAGE:first % PAGE + count])
        return out


def rotated(x, pos, theta, rd, style, w=None, eps=0.0, inv_freq=None):
    """Heads x [T, heads, dim] float64, normed by w if given, their first rd dims turned by position."""
    if w is not None:
        x = x * w / np.sqrt((x ** 2).mean(-1, keepdims=True) + eps)
    j = np.arange(rd // 2)
    f = theta ** (-2.0 * j / rd) if inv_freq is None else np.asarray(inv_freq, np.float64)
    ang = np.mod(np.asarray(pos, np.float64)[:, None] * f, 2 * np.pi)[:, None, :]
    a, b = (j, j + rd // 2) if style == 0 else (2 * j, 2 * j + 1)
    y = x.copy()
    y[..., a] = x[..., a] * np.cos(ang) - x[..., b] * np.sin(ang)
    y[..., b] = x[..., a] * np.sin(ang) + x[..., b] * np.cos(ang)
    return y


def attend(q, k, v, scale, seen=None, q_err=0.0):
    """q [E, Hq, d] over k, v [n, Hkv, d] (float64): outputs [E, Hq, d], lse [E, Hq], and bounds on
    the errors of both.  seen[i]: keys that row i sees (None: all).

    Counted, at their worst: the weights rounded to bf16 before their product with V, and the
    same rounded weights summed; the output rounded to bf16; queries rounded by q_err (relative)
    before the scores; scores accumulated in float32 (d terms), exponentials, sums and merges in
    float32 (16 steps, and the sum's n adds of positive terms in any order: n / 64 a lane)."""
    E, Hq, d = q.shape
    n, Hkv = k.shape[0], k.shape[1]
    out, lse = np.zeros((E, Hq, d)), np.full((E, Hq), -np.inf)
    tol_o, tol_l = np.zeros((E, Hq, d)), np.zeros((E, Hq))
    g = Hq // Hkv
    for h in range(Hkv if n else 0):
        qh = q[:, h * g:(h + 1) * g].reshape(E * g, d)
        s = (qh @ k[:, h].T) * scale
        mag = (np.abs(qh) @ np.abs(k[:, h]).T) * scale
        if seen is not None:
            hide = np.arange(n)[None, :] >= np.repeat(np.asarray(seen), g)[:, None]
            s, mag = np.where(hide, -np.inf, s), np.where(hide, 0, mag)
        m = s.max(-1, keepdims=True)
        p = np.exp(s - m)
        total = p.sum(-1, keepdims=True)
        o = (p / total) @ v[:, h]
        size = (p / total) @ np.abs(v[:, h])  # of what is added up
        ds = (q_err + (d + 4) * F32) * mag.max(-1, keepdims=True)
        w = np.expm1(2 * ds) + HALF_BF16 + (16 + n / 64) * F32  # a weight's relative error
        out[:, h * g:(h + 1) * g] = o.reshape(E, g, d)
        lse[:, h * g:(h + 1) * g] = (m + np.log(total)).reshape(E, g)
        tol_o[:, h * g:(h + 1) * g] = (w * (size + np.abs(o)) + HALF_BF16 * np.abs(o) * (1 + w) + 1e-38).reshape(E, g, d)
        tol_l[:, h * g:(h + 1) * g] = (w + ds + 8 * F32 * (np.abs(m) + 1)).reshape(E, g)
    return out, lse, tol_o, tol_l


def check(got, want, tol, what):
    got = np.asarray(got, np.float64)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    same_inf = np.isinf(want) & (got == want)
    bad = ~same_inf & ~(np.abs(got - np.where(same_inf, 0, want)) <= tol)
    worst = np.where(same_inf, 0, np.abs(got - np.where(same_inf, 0, want)) / np.maximum(tol, 1e-300))
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, at {np.argwhere(bad)[0]}, {np.nanmax(worst):.2f} times the bound"
    return float(np.nanmax(worst)) if worst.size else 0.0
