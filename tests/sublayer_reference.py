"""64-bit definitions of the calls for long sequences (e4m3 rows and products,
norms with rotation, windowed attention), in plain loops and products on the CPU."""
import numpy as np
import torch

FP8_MAX, MIN_AMAX = 448.0, 2.0 ** -100
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def half_step(dtype):
    """Largest relative error of one rounding to the type."""
    return torch.finfo(dtype).eps / 2


def blocks(n):
    return -(-n // 128)


def quantize(x):
    """fp32 operations, as the call defines them: (e4m3 [rows, cols], scale [blocks, rows])."""
    x = x.float()
    codes, scales = [], []
    for part in x.split(128, 1):
        a = part.abs().amax(1).clamp_min(MIN_AMAX)  # (a NaN stays)
        inv = torch.full_like(a, FP8_MAX) / a
        codes.append((part * inv[:, None]).to(torch.float8_e4m3fn))
        scales.append(a / torch.full_like(a, FP8_MAX))
    return torch.cat([c.view(torch.uint8) for c in codes], 1).view(torch.float8_e4m3fn), torch.stack(scales)


def gemm_fp8(a, a_scale, w, w_scale, k):
    """(acc, sum of the terms' magnitudes) in 64 bits."""
    n = w.shape[0]
    acc = torch.zeros((a.shape[0], n), dtype=torch.float64)
    mag = torch.zeros_like(acc)
    for b in range(blocks(k)):
        cols = slice(128 * b, min(k, 128 * b + 128))
        pa, pw = a[:, cols].float().double(), w[:, cols].float().double()
        s = a_scale[b].double()[:, None] * w_scale[:, b].double().repeat_interleave(128)[:n]
        acc += s * (pa @ pw.t())
        mag += s.abs() * (pa.abs() @ pw.abs().t())
    return acc, mag


def norm_rope(x, gain, cos, sin, eps, interleaved):
    """x [rows, heads, d] of any type; cos, sin [rows, rot / 2]; 64 bits."""
    y = x.double()
    y = y / torch.sqrt((y * y).mean(2, keepdim=True) + eps)
    if gain is not None:
        y = y * gain.double()
    half = cos.shape[1]
    c, s = cos.double()[:, None], sin.double()[:, None]
    out = y.clone()
    if interleaved:
        a, b = y[..., 0:2 * half:2], y[..., 1:2 * half:2]
        out[..., 0:2 * half:2], out[..., 1:2 * half:2] = a * c - b * s, b * c + a * s
    else:
        a, b = y[..., :half], y[..., half:2 * half]
        out[..., :half], out[..., half:2 * half] = a * c - b * s, b * c + a * s
    return out


def visible(nq, nk, causal, window, sinks):
    """[nq, nk] truth values, from the definition."""
    p = torch.arange(nk - nq, nk)[:, None]
    j = torch.arange(nk)[None]
    near = torch.ones((nq, nk), dtype=torch.bool) if window < 0 else (j - p).abs() <= window
    if causal:
        seen = (j <= p) & (near | (j < sinks))
    else:
        seen = near | (j < sinks) | (p < sinks)
    return seen & (p >= 0)


def attention(q, k, v, scale, causal, window, sinks):
    """One sequence: q [nq, h, d], k, v [nk, hk, d] -> (out, weighted mean of |v|),
    64 bits [nq, h, d]. Hidden keys and values take no part, whatever they hold."""
    nq, h, d = q.shape
    nk, hk, _ = k.shape
    out = torch.zeros((nq, h, d), dtype=torch.float64)
    mean = torch.zeros_like(out)
    if nk == 0:
        return out, mean
    seen = visible(nq, nk, causal, window, sinks)
    for i in range(h):
        kk, vv = k[:, i // (h // hk)].double(), v[:, i // (h // hk)].double()
        used = seen.any(0)
        kk, vv = torch.where(used[:, None], kk, 0.0), torch.where(used[:, None], vv, 0.0)
        x = (q[:, i].double() @ kk.t()) * scale
        x = torch.where(seen, x, -np.inf)
        top = x.max(1, keepdim=True).values
        e = torch.where(seen, torch.exp(x - torch.where(torch.isinf(top), 0.0, top)), 0.0)
        p = e / e.sum(1, keepdim=True).clamp_min(1e-300)
        if torch.isfinite(vv).all():
            out[:, i], mean[:, i] = p @ vv, p @ vv.abs()
        else:  # row by row, the visible values alone
            for r in range(nq):
                s = seen[r]
                out[r, i] = p[r, s] @ vv[s]
                mean[r, i] = p[r, s] @ vv[s].abs()
    return out, mean
