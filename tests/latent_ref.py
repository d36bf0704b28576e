"""Plain float64 reference of the latent-cache operators, with bounds on what their stated
roundings can do.  Independent of the kernels: numpy on logical rows, no pages."""

from __future__ import annotations

import numpy as np
import torch

ROPE, GROUP = 64, 64
HALF_BF16 = 2.0 ** -8   # half a bf16 step, relative to the value
F32 = 2.0 ** -24


def f64(t: torch.Tensor) -> np.ndarray:
    return t.detach().cpu().to(torch.float64).numpy()


def scale_exps(c: np.ndarray) -> np.ndarray:
    """Exponents of the 64-value groups of latents [n, lat] (float64): smallest e with
    max|c| <= 448 * 2^e, held to [-117, 119]."""
    top = np.abs(c).reshape(c.shape[0], -1, GROUP).max(-1)
    m, x = np.frexp(top)
    return np.clip(np.where(m <= 0.875, x - 9, x - 8), -117, 119)


def quantised(c: np.ndarray, e: np.ndarray | None = None) -> np.ndarray:
    """Latents [n, lat] as an 8-bit pool holds them (torch's e4m3 cast rounds to nearest even)."""
    e = scale_exps(c) if e is None else e
    by = np.repeat(e, GROUP, axis=1)
    y = np.clip(np.ldexp(c, -by), -448, 448)
    code = torch.from_numpy(y.astype(np.float32)).to(torch.float8_e4m3fn)
    return np.ldexp(code.to(torch.float64).numpy(), by)


def rope_planes(style: int):
    if style == 0:
        return np.arange(ROPE // 2), np.arange(ROPE // 2) + ROPE // 2
    return 2 * np.arange(ROPE // 2), 2 * np.arange(ROPE // 2) + 1


def rotated(x: np.ndarray, pos: np.ndarray, freqs: np.ndarray, style: int) -> np.ndarray:
    """The last dim (64) of x [n, ..., 64] turned by pos[n] * freqs."""
    a, b = rope_planes(style)
    ang = np.mod(pos[:, None].astype(np.float64) * freqs[None, :], 2 * np.pi)
    shape = (len(pos),) + (1,) * (x.ndim - 2) + (ROPE // 2,)
    cos, sin = np.cos(ang).reshape(shape), np.sin(ang).reshape(shape)
    y = x.copy()
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., a] * sin + x[..., b] * cos
    return y


def attend(q: np.ndarray, keys: np.ndarray, values: np.ndarray, prefix: int, scale: float, q_err: float = 0.0,
           k_err: float = 0.0, v_err: float = 0.0):
    """q [E, H, dq], keys [L, dq] or [H, L, dq], values likewise: outputs [E, H, dv], lse
    [E, H], and bounds on their errors before the outputs are rounded.

    What is counted, worst cases throughout: operands rounded by q_err / k_err / v_err
    (relative) before the products; float32 accumulation of a score (dq terms); weights
    rounded to bf16; float32 exponentials, sums and division (16 steps of 2^-24)."""
    e, h, dq = q.shape
    out, lse, tol, ltol = [], [], [], []
    for hh in range(h):
        k = keys if keys.ndim == 2 else keys[hh]
        v = values if values.ndim == 2 else values[hh]
        s = q[:, hh] @ k.T * scale
        size = np.abs(q[:, hh]) @ np.abs(k).T * scale
        seen = np.arange(k.shape[0])[None, :] <= (prefix + np.arange(e))[:, None]
        s = np.where(seen, s, -np.inf)
        top = s.max(-1, keepdims=True)
        w = np.exp(s - top)
        total = w.sum(-1, keepdims=True)
        w = w / total
        s_err = (size * (q_err + k_err + (dq + 8) * F32)) * seen
        # a score also passes through s * scale * log2(e) - m in float32
        s_err = s_err + 4 * F32 * (np.abs(np.where(seen, s, 0)) + np.abs(top))
        worst = (s_err * seen).max(-1, keepdims=True)
        a = w @ np.abs(v)
        out.append(w @ v)
        lse.append((top + np.log(total))[:, 0])
        n = seen.sum(-1, keepdims=True)
        tol.append(a * (np.expm1(2 * worst) + HALF_BF16 + v_err + (n + 16) * F32))
        ltol.append((worst + (n + 16) * F32 + 4 * F32 * np.abs(top + np.log(total)))[:, 0])
    return [np.stack(x, 1) for x in (out, lse, tol, ltol)]


def check_rows(got: torch.Tensor, want: np.ndarray, tol: np.ndarray, rms: float, tag: str = ""):
    """Every value within its bound and half a bf16 step; the whole within `rms` of the
    reference's 2-norm."""
    g = f64(got)
    assert g.shape == want.shape, (g.shape, want.shape)
    assert np.isfinite(g).all(), f"{tag}: non-finite outputs at {np.argwhere(~np.isfinite(g))[:4]}"
    err = np.abs(g - want)
    over = err - (tol + HALF_BF16 * (np.abs(want) + tol) + 2.0 ** -133)
    assert (over <= 0).all(), f"{tag}: {int((over > 0).sum())} of {err.size} values off, worst {err.max():.3e} at {np.unravel_index(over.argmax(), over.shape)}"
    rel = np.linalg.norm(g - want) / max(np.linalg.norm(want), 1e-30)
    assert rel <= rms, f"{tag}: relative error {rel:.2e} of the whole"
