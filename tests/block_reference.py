"""64-bit definitions of the operators of a transformer block (residual sums with norms, rotation on several axes,
attention behind a shared prefix), in plain loops and products on the CPU."""
import torch

NONE, RMS, LAYER = range(3)
HALF, NEIGHBOURS, AXIS = range(3)


def norm(v, kind, gain, bias, eps):
    """(normed rows, 1 / the root) of v [rows, cols], 64 bits."""
    if kind == NONE:
        return v, torch.ones_like(v[:, :1])
    if kind == LAYER:
        v = v - v.mean(1, keepdim=True)
    inv = 1 / torch.sqrt((v * v).mean(1, keepdim=True) + eps)
    y = v * inv
    if gain is not None:
        y = y * gain.double()
    return (y if bias is None else y + bias.double()), inv


def _size(t):
    return 1.0 if t is None else t.double().abs()


def residual_norm(x, y, x_factor=1.0, post=NONE, post_gain=None, post_bias=None, y_scale=None, pre=NONE, pre_gain=None,
                  pre_bias=None, gate=None, shift=None, scale=None, group=None, eps=1e-6):
    """(s, z, error of s, error of z): the definition in 64 bits, and how far fp32 arithmetic may be from it.

    A row's sums run over at most 64 terms one after another and in trees: relative 2^-18 of the terms' magnitudes.
    e: that, with the few roundings of the products beside it, 2^-16. An error D in all values of a row moves its norm by
    at most 2 D / root in a value and by D / root relative in the root."""
    e = 2.0 ** -16
    rows = [None if t is None else t.double()[group] for t in (gate, shift, scale)]
    s = x.double() * x_factor
    ds = e * s.abs()
    if y is not None:
        u, inv = norm(y.double(), post, post_gain, post_bias, eps)
        size = u.abs() if post == NONE else inv * y.double().abs().amax(1, keepdim=True) * _size(post_gain)
        for f in (y_scale, rows[0]):
            if f is not None:
                u, size = u * f.double(), size * f.double().abs()
        s = s + u
        ds = ds + e * (size + u.abs())
    z, inv = norm(s, pre, pre_gain, pre_bias, eps)
    if pre == NONE:
        dz = ds.clone()
    else:
        worst, top = ds.amax(1, keepdim=True), s.abs().amax(1, keepdim=True)
        plain = norm(s, pre, None, None, eps)[0].abs()
        dz = (inv * (2 * worst + e * top) + plain * (e + inv * worst)) * _size(pre_gain) + e * z.abs()
    if rows[2] is not None:
        z, dz = z * (1 + rows[2]), dz * (1 + rows[2].abs()) + e * z.abs() * (1 + rows[2].abs())
    if rows[1] is not None:
        z, dz = z + rows[1], dz + e * rows[1].abs()
    return s, z, ds, dz + e * z.abs()


def channels(axis_of, pairing):
    """The first and the second channel of each pair."""
    n, out = len(axis_of), []
    for j, a in enumerate(axis_of):
        if pairing == NEIGHBOURS:
            out.append((2 * j, 2 * j + 1))
        elif pairing == HALF:
            out.append((j, j + n))
        else:
            s, m = list(axis_of).index(a), list(axis_of).count(a)
            out.append((2 * s + j - s, 2 * s + j - s + m))
    return out


def rope_axes(x, gain, table, positions, axis_of, pairing, normed, eps):
    """x [rows, heads, d]; table [n, rot]; positions [rows, axes]; 64 bits, pair by pair."""
    y = x.double()
    if normed:
        y = y / torch.sqrt((y * y).mean(2, keepdim=True) + eps)
    if gain is not None:
        y = y * gain.double()
    out, half = y.clone(), len(axis_of)
    for j, (a, b) in enumerate(channels(axis_of, pairing)):
        at = table.double()[positions[:, axis_of[j]].long()]
        c, s = at[:, j, None], at[:, half + j, None]
        out[..., a], out[..., b] = y[..., a] * c - y[..., b] * s, y[..., b] * c + y[..., a] * s
    return out


def prefix_attention(q, k, v, prefix_k, prefix_v, scale):
    """One sequence: q [nq, h, d] behind the keys of a prefix [p, hk, d] and its own [nk, hk, d] -> (out, weighted mean
    of |v|), 64 bits [nq, h, d]. Query i sees the prefix and its own keys up to nk - nq + i. Hidden keys and values take
    no part, whatever they hold."""
    nq, h, d = q.shape
    nk, group = k.shape[0], h // k.shape[1]
    out = torch.zeros((nq, h, d), dtype=torch.float64)
    mean = torch.zeros_like(out)
    for i in range(nq):
        seen = max(0, min(nk, nk - nq + i + 1))
        keys, values = torch.cat([prefix_k, k[:seen]]).double(), torch.cat([prefix_v, v[:seen]]).double()
        if keys.shape[0] == 0:
            continue
        for a in range(h):
            x = keys[:, a // group] @ q[i, a].double() * scale
            e = torch.exp(x - x.max())
            p = e / e.sum()
            out[i, a], mean[i, a] = p @ values[:, a // group], p @ values[:, a // group].abs()
    return out, mean


def e4m3_half_step(want):
    """The largest error of one rounding to e4m3 of values within +-448: half a step, of subnormals 2^-10."""
    return torch.maximum(want.abs() * 2.0 ** -4, torch.full_like(want, 2.0 ** -10))
