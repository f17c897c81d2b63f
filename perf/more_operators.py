"""Operators of transformer blocks over image, video and text tokens:

  residual  the sum at a block's end with the norm before the next block: the block's output normed,
            scaled for each channel and gated for each sequence, added to the stream, and the stream
            normed and modulated, as 16-bit rows or as e4m3 rows with scales (elasto_op_residual_norm);
  rope      norms of each query and key head with rotary positions on several axes (time, height,
            width), K and V optionally to their cache rows (elasto_op_qk_norm_rope_axes);
  prefix    attention of sequences that share a long prefix, whose keys are read once for all, each
            with keys of its own behind it (elasto_op_prefix_attention).

`own` chooses between the plain form of each (elementary torch operations in 32 bits) and the
library's call.
"""
import ctypes
import math
import random

import torch

own = False

DEVICE = "cuda"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn}
SIZES = {"bf16": 2, "f16": 2, "f32": 4, "e4m3": 1}
NORMS = {"none": 0, "rms": 1, "layer": 2}
PAIRINGS = {"half": 0, "neighbours": 1, "axis": 2}
FP8_MAX = 448.0
MIN_AMAX = 2.0 ** -100
EPS = 1e-6


def listed():
    return [
        # the fp32 stream of the largest ViT-B batch (256 images of 197 tokens): LayerScale, then the next LayerNorm
        {"name": "residual_256", "kind": "residual", "rows": 50432, "cols": 768, "x": "f32", "y": "bf16", "z": "bf16",
         "post": "none", "pre": "layer", "affine": True, "y_scale": True, "mod": "none", "groups": 1},
        # one image: latency
        {"name": "residual_1", "kind": "residual", "rows": 197, "cols": 768, "x": "f32", "y": "bf16", "z": "bf16",
         "post": "none", "pre": "layer", "affine": True, "y_scale": True, "mod": "none", "groups": 1},
        # four videos whose blocks are gated and modulated by a condition of each
        {"name": "residual_modulated_4", "kind": "residual", "rows": 32760, "cols": 1536, "x": "bf16", "y": "bf16", "z": "bf16",
         "post": "none", "pre": "layer", "affine": False, "y_scale": False, "mod": "bf16", "groups": 4},
        # norms before and after each block, the next products' rows in e4m3; a last block of columns that is not whole
        {"name": "residual_fp8", "kind": "residual", "rows": 8191, "cols": 5000, "x": "bf16", "y": "bf16", "z": "e4m3",
         "post": "rms", "pre": "rms", "affine": True, "y_scale": False, "mod": "none", "groups": 1},
        # a video of 21 x 30 x 52 patches, pairs of neighbouring channels, an uneven share of them for each axis
        {"name": "rope_video", "kind": "rope", "type": "bf16", "frames": 21, "height": 30, "width": 52, "videos": 1, "front": 0, "heads_q": 12,
         "heads_k": 12, "dim": 128, "pairs": "22 21 21", "mixed": False, "pairing": "neighbours", "norm": True, "cache_rows": 0},
        # eight images of 64 x 64 patches behind a class token, half of a head for each axis, no norm
        {"name": "rope_images_8", "kind": "rope", "type": "f16", "frames": 1, "height": 64, "width": 64, "videos": 8, "front": 1, "heads_q": 12,
         "heads_k": 12, "dim": 64, "pairs": "0 16 16", "mixed": False, "pairing": "axis", "norm": False, "cache_rows": 0},
        # one new token of each of 64 sequences, K and V into the cache; three axes within one half-split rotation
        {"name": "rope_decode_64", "kind": "rope", "type": "bf16", "frames": 64, "height": 1, "width": 1, "videos": 1, "front": 0, "heads_q": 32,
         "heads_k": 8, "dim": 128, "pairs": "16 24 24", "mixed": False, "pairing": "half", "norm": True, "cache_rows": 16384},
        # one new token of each of 64 sequences behind a shared document
        {"name": "prefix_decode_64", "kind": "prefix", "type": "bf16", "prefixes": 1, "batch": 64, "queries": 1, "prefix": 8192,
         "keys": 1024, "ragged": 3, "packed": False, "heads": 32, "heads_kv": 8, "dim": 128},
        # many sequences behind a longer one: the prefix's products
        {"name": "prefix_decode_256", "kind": "prefix", "type": "bf16", "prefixes": 1, "batch": 256, "queries": 1, "prefix": 16384,
         "keys": 512, "ragged": 5, "packed": False, "heads": 32, "heads_kv": 8, "dim": 128},
        # four continuations of one image's tokens: latency
        {"name": "prefix_decode_4", "kind": "prefix", "type": "f16", "prefixes": 1, "batch": 4, "queries": 1, "prefix": 2000,
         "keys": 100, "ragged": 7, "packed": False, "heads": 12, "heads_kv": 12, "dim": 64},
        # up to five drafted tokens of each of 32 sequences to be checked at once
        {"name": "prefix_draft_32", "kind": "prefix", "type": "bf16", "prefixes": 1, "batch": 32, "queries": 5, "prefix": 6000,
         "keys": 700, "ragged": 9, "packed": False, "heads": 28, "heads_kv": 4, "dim": 128},
        # eight images of 4097 tokens with eight prompts each, of up to 96 tokens, packed
        {"name": "prefix_images_8", "kind": "prefix", "type": "bf16", "prefixes": 8, "batch": 64, "queries": 96, "prefix": 4097,
         "keys": 96, "ragged": 11, "packed": True, "heads": 32, "heads_kv": 8, "dim": 128},
    ]


def _log_uniform(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_residual(rng):
    cols = _log_uniform(rng, 32, 8192)
    rows = _log_uniform(rng, 1, max(1, min(50000, 28000000 // cols)))
    post, pre = rng.choice(["none", "rms", "layer"]), rng.choice(["rms", "layer", "layer"])
    return {"kind": "residual", "rows": rows, "cols": cols, "x": rng.choice(["f32", "bf16", "f16"]), "y": rng.choice(["bf16", "f16", "f32"]),
            "z": rng.choice(["bf16", "f16", "f32", "e4m3"]), "post": post, "pre": pre, "affine": rng.random() < 0.7,
            "y_scale": rng.random() < 0.5, "mod": rng.choice(["none", "bf16", "f32"]), "groups": rng.randint(1, min(rows, 40))}


def _draw_rope(rng):
    dim = rng.choice([64, 80, 96, 128, 256])
    pairing = rng.choice(["half", "neighbours", "axis"])
    unit = 8 if pairing == "axis" else 1
    units = rng.choice([dim, dim // 32 * 16]) // 2 // unit
    a, b = sorted((rng.randint(0, units), rng.randint(0, units)))
    group, heads_k = rng.choice([1, 2, 4, 8]), _log_uniform(rng, 1, 12)
    most = min(30000, 40000000 // (heads_k * (group + 1) * dim))
    rows = _log_uniform(rng, 1, most)
    h, w = rng.randint(1, 60), rng.randint(1, 60)
    h, w = min(h, rows), max(1, min(w, rows // min(h, rows)))
    frames, front = max(1, rows // (h * w)), rng.choice([0, 1])
    rows = frames * h * w + front
    return {"kind": "rope", "type": rng.choice(["bf16", "f16"]), "frames": frames, "height": h, "width": w, "videos": 1, "front": front,
            "heads_q": heads_k * group, "heads_k": heads_k, "dim": dim,
            "pairs": " ".join(str(n * unit) for n in (a, b - a, units - b)), "mixed": pairing != "axis" and rng.random() < 0.3, "pairing": pairing, "norm": rng.random() < 0.6,
            "cache_rows": rng.choice([0, rows + rng.randrange(0, 999)])}


def _draw_prefix(rng):
    heads_kv, group = rng.choice([1, 2, 3, 4, 8]), rng.choice([1, 2, 3, 4, 7, 8])
    prefixes = rng.choice([1, 1, 1, 2, 5])
    queries = rng.choice([1, 1, 1, rng.randint(2, 8), _log_uniform(rng, 8, 128)])
    batch = _log_uniform(rng, 1, max(1, 256 // (1 + queries // 4)))
    case = {"kind": "prefix", "type": rng.choice(["bf16", "f16"]), "prefixes": min(prefixes, batch), "batch": batch, "queries": queries,
            "prefix": _log_uniform(rng, 16, 16384), "keys": max(queries, _log_uniform(rng, 1, 512)), "ragged": rng.randrange(0, 100),
            "packed": rng.random() < 0.4, "heads": heads_kv * group, "heads_kv": heads_kv, "dim": rng.choice([32, 64, 80, 128, 128])}
    most = 40e9 / (4.0 * case["dim"] * case["heads"] * batch * queries)
    case["prefix"] = max(1, min(case["prefix"], int(most), 40000000 // (case["prefixes"] * heads_kv * case["dim"])))
    return case


def draw(rng):
    kind = rng.choice(["residual", "residual", "rope", "rope", "prefix", "prefix", "prefix"])
    return {"residual": _draw_residual, "rope": _draw_rope, "prefix": _draw_prefix}[kind](rng)


# ---------------------------------------------------------------- inputs

def _generator(seed):
    return torch.Generator(device=DEVICE).manual_seed(int(seed))


def _normal(shape, g, std=1.0):
    return torch.randn(shape, generator=g, device=DEVICE) * std


def _blocks(n):
    return -(-n // 128)


def _spread(total, parts, seed):
    """`total` cut into `parts` lengths that differ (each at least one)."""
    r = random.Random(seed)
    cuts = sorted(r.sample(range(1, total), parts - 1)) if parts > 1 else []
    return [b - a for a, b in zip([0] + cuts, cuts + [total])]


def _starts(lengths):
    out = [0]
    for n in lengths:
        out.append(out[-1] + n)
    return out


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEVICE)


def _prepare_residual(case, s, g):
    rows, cols, groups = case["rows"], case["cols"], case["groups"]
    channels = torch.exp(0.5 * _normal((cols,), g))  # a few channels are much larger, as in trained transformers
    s["x"] = (3 * _normal((rows, cols), g) * channels + 0.5).to(TYPES[case["x"]])
    s["y"] = (_normal((rows, cols), g) * channels.flip(0)).to(TYPES[case["y"]])
    for name in ("post", "pre"):
        affine = case["affine"] and case[name] != "none"
        s[name + "_gain"] = 1 + 0.1 * _normal((cols,), g) if affine else None
        s[name + "_bias"] = 0.1 * _normal((cols,), g) if affine and case[name] == "layer" else None
    s["y_scale"] = 0.3 * _normal((cols,), g) if case["y_scale"] else None
    if case["mod"] != "none":  # columns of one product of the condition, as it writes them
        s["mod"] = _normal((groups, 3 * cols), g, 0.3).to(TYPES[case["mod"]])
        lengths = _spread(rows, groups, rows + groups)
        s["group"] = torch.repeat_interleave(torch.arange(groups, device=DEVICE), torch.tensor(lengths, device=DEVICE)).int()
    s["x_out"] = torch.empty_like(s["x"])
    s["z"] = torch.empty((rows, cols), dtype=TYPES[case["z"]], device=DEVICE)
    if case["z"] == "e4m3":
        s["z_scale"] = torch.empty((_blocks(cols), rows), device=DEVICE)


def _pairs(case):
    """How many pairs of channels each axis turns."""
    return [int(n) for n in case["pairs"].split()]


def _grid(case):
    return case["frames"], case["height"], case["width"]


def _axis_of(case):
    """The axis that turns each pair: runs of pairs, or (mixed) axes taking turns as long as they have pairs left."""
    left, out = _pairs(case), []
    if not case["mixed"]:
        return [a for a, n in enumerate(left) for _ in range(n)]
    while any(left):
        for a in range(len(left)):
            if left[a]:
                out.append(a)
                left[a] -= 1
    return out


def _rope_rows(case):
    t, h, w = _grid(case)
    return case["videos"] * (t * h * w + case["front"])


def _prepare_rope(case, s, g):
    rows, hq, hk, d, rot = _rope_rows(case), case["heads_q"], case["heads_k"], case["dim"], 2 * sum(_pairs(case))
    t = TYPES[case["type"]]
    s["qkv"] = _normal((rows, hq + 2 * hk, d), g).to(t)  # as the QKV product writes it
    s["gain_q"] = 1 + 0.1 * _normal((d,), g) if case["norm"] else None
    s["gain_k"] = 1 + 0.1 * _normal((d,), g) if case["norm"] else None
    s["axis_of"] = axis_of = _axis_of(case)
    # each axis has a ladder of frequencies of its own
    rank, seen = [], [0, 0, 0]
    for a in axis_of:
        rank.append(seen[a] / max(1, _pairs(case)[a]))
        seen[a] += 1
    positions = max(_grid(case)) + case["front"] + 1000
    inv = 10000.0 ** -torch.tensor(rank, dtype=torch.float64, device=DEVICE)
    angle = torch.arange(positions, dtype=torch.float64, device=DEVICE)[:, None] * inv
    s["table"] = torch.cat([angle.cos(), angle.sin()], 1).float().contiguous()
    gt, gh, gw = _grid(case)
    grid = torch.stack(torch.meshgrid(*(torch.arange(n, device=DEVICE) for n in (gt, gh, gw)), indexing="ij")).flatten(1)
    if gt * gh * gw > 1 and gh * gw == 1:  # single tokens of sequences, each at a place of its own
        grid = torch.randint(0, positions, grid.shape, generator=g, device=DEVICE)
    else:
        grid = grid + torch.randint(0, 900, (1,), generator=g, device=DEVICE)
    one = torch.cat([torch.zeros((3, case["front"]), dtype=grid.dtype, device=DEVICE), grid], 1)
    s["pos"] = one.repeat(1, case["videos"]).int().contiguous()  # [axis, row]
    s["q_out"] = torch.empty((rows, hq, d), dtype=t, device=DEVICE)
    out_rows = case["cache_rows"] or rows
    s["k_out"] = torch.zeros((out_rows, hk, d), dtype=t, device=DEVICE)
    s["rot"] = rot
    if case["cache_rows"]:
        s["slots"] = torch.randperm(out_rows, generator=g, device=DEVICE)[:rows].to(torch.int32)
        s["v_out"] = torch.zeros((out_rows, hk, d), dtype=t, device=DEVICE)


def _prefix_lengths(case):
    """(sequences, keys) of each prefix, (queries, own keys with the queries' own) of each sequence."""
    r = random.Random(case["ragged"])
    p, b = case["prefixes"], case["batch"]
    members = _spread(b, p, case["ragged"])
    if not case["ragged"]:
        return members, [case["prefix"]] * p, [case["queries"]] * b, [case["keys"]] * b
    prefix = [case["prefix"]] + [r.randint(max(1, case["prefix"] // 2), case["prefix"]) for _ in range(p - 1)]
    keys = [case["keys"]] + [r.randint(max(1, case["keys"] // 8), case["keys"]) for _ in range(b - 1)]
    if case["packed"]:  # prompts: their keys are the queries' own
        return members, prefix, [min(case["queries"], k) for k in keys], [min(case["queries"], k) for k in keys]
    return members, prefix, [min(k, case["queries"] if i % 3 else max(1, case["queries"] // 2)) for i, k in enumerate(keys)], keys


def _prepare_prefix(case, s, g):
    t, d, h, hk, b = TYPES[case["type"]], case["dim"], case["heads"], case["heads_kv"], case["batch"]
    members, prefix, nq, nk = _prefix_lengths(case)
    s["prefix_k"] = _normal((case["prefixes"], case["prefix"], hk, d), g).to(t)
    s["prefix_v"] = _normal((case["prefixes"], case["prefix"], hk, d), g).to(t)
    s["prefix_len"], s["seq_start"] = _int32(prefix), _int32(_starts(members))
    if case["packed"]:  # q, k and v are columns of one projection's output
        qkv = _normal((sum(nq), h + 2 * hk, d), g).to(t)
        s["q"], s["k"], s["v"] = qkv[:, :h], qkv[:, h:h + hk], qkv[:, h + hk:]
        s["kv_start"] = _int32(_starts(nk))
    else:
        s["q"] = _normal((sum(nq), h, d), g).to(t)
        s["k"] = _normal((b, case["keys"], hk, d), g).to(t)
        s["v"] = _normal((b, case["keys"], hk, d), g).to(t)
        s["kv_len"] = _int32(nk)
    s["q_start"] = _int32(_starts(nq))
    s["out"] = torch.empty((sum(nq), h, d), dtype=t, device=DEVICE)


def prepare(case, seed):
    s = {"case": case}
    {"residual": _prepare_residual, "rope": _prepare_rope, "prefix": _prepare_prefix}[case["kind"]](case, s, _generator(seed))
    if own:
        s["args"] = _own_args(s)
    return s


# ---------------------------------------------------------------- plain forms

def _plain_norm(x, kind, gain, bias):
    if kind == "none":
        return x
    if kind == "layer":
        x = x - x.mean(1, keepdim=True)
    x = x / torch.sqrt((x * x).mean(1, keepdim=True) + EPS)
    if gain is not None:
        x = x * gain
    return x if bias is None else x + bias


def _plain_e4m3(z):
    """z [rows, cols] fp32 -> e4m3 [rows, cols], scales [blocks, rows]."""
    rows, cols = z.shape
    nb = _blocks(cols)
    zb = torch.nn.functional.pad(z, (0, nb * 128 - cols)).view(rows, nb, 128)
    amax = zb.abs().amax(-1).clamp_min(MIN_AMAX)
    q = (zb * (torch.full_like(amax, FP8_MAX) / amax)[..., None]).view(rows, nb * 128)[:, :cols]
    return q.to(torch.float8_e4m3fn), (amax / torch.full_like(amax, FP8_MAX)).t().contiguous()


def _plain_residual(s):
    case, cols = s["case"], s["case"]["cols"]
    u = _plain_norm(s["y"].float(), case["post"], s["post_gain"], s["post_bias"])
    if s["y_scale"] is not None:
        u = u * s["y_scale"]
    if case["mod"] != "none":
        m = s["mod"].float()[s["group"].long()]
        u = u * m[:, :cols]
    x = s["x"].float() + u
    z = _plain_norm(x, case["pre"], s["pre_gain"], s["pre_bias"])
    if case["mod"] != "none":
        z = z * (1 + m[:, 2 * cols:]) + m[:, cols:2 * cols]
    return [x.to(s["x"].dtype)] + (list(_plain_e4m3(z)) if case["z"] == "e4m3" else [z.to(s["z"].dtype)])


def _channels(case):
    """The first and the second channel of each pair."""
    n = sum(_pairs(case))
    j = torch.arange(n, device=DEVICE)
    if case["pairing"] == "neighbours":
        return 2 * j, 2 * j + 1
    if case["pairing"] == "half":
        return j, j + n
    size = torch.tensor(_pairs(case), device=DEVICE)[_int32(_axis_of(case)).long()]
    start = torch.tensor(_starts(_pairs(case))[:-1], device=DEVICE)[_int32(_axis_of(case)).long()]
    return j + start, j + start + size


def _plain_rope(s):
    case = s["case"]
    hq, hk, half = case["heads_q"], case["heads_k"], s["rot"] // 2
    j = torch.arange(half, device=DEVICE)
    at = s["pos"][_int32(s["axis_of"]).long()].t().long()  # [row, pair]
    cos, sin = s["table"][at, j][:, None], s["table"][at, half + j][:, None]
    first, second = _channels(case)

    def one(x, gain):
        x = x.float()
        if case["norm"]:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gain
        a, b = x[..., first], x[..., second]
        y = x.clone()
        y[..., first], y[..., second] = a * cos - b * sin, b * cos + a * sin
        return y.to(s["qkv"].dtype)

    q, k = one(s["qkv"][:, :hq], s["gain_q"]), one(s["qkv"][:, hq:hq + hk], s["gain_k"])
    if not case["cache_rows"]:
        return [q, k]
    s["k_out"][s["slots"].long()] = k
    s["v_out"][s["slots"].long()] = s["qkv"][:, hq + hk:]
    return [q, s["k_out"], s["v_out"]]


def _plain_prefix(s):
    """Scores of a prefix's rows at once, those of the sequences' own keys padded to the longest; one softmax over both."""
    case = s["case"]
    h, hk, d, b = case["heads"], case["heads_kv"], case["dim"], case["batch"]
    scale, group = 1 / math.sqrt(d), h // hk
    q_start, members = s["q_start"].long(), _prefix_lengths(case)[0]
    nq = q_start[1:] - q_start[:-1]
    most = case["queries"]
    i, j = torch.arange(most, device=DEVICE), torch.arange(case["keys"], device=DEVICE)
    rows, is_row = (q_start[:-1, None] + i).clamp_max(s["q"].shape[0] - 1), i < nq[:, None]
    q = s["q"][rows].float().view(b, most, hk, group, d).permute(2, 0, 1, 3, 4).reshape(hk, b, most * group, d)
    if case["packed"]:
        kv_start = s["kv_start"].long()
        nk = kv_start[1:] - kv_start[:-1]
        at = (kv_start[:-1, None] + j).clamp_max(s["k"].shape[0] - 1)
        k, v = s["k"][at].float(), s["v"][at].float()
    else:
        nk, k, v = s["kv_len"].long(), s["k"].float(), s["v"].float()
    k, v = k.permute(2, 0, 3, 1), v.permute(2, 0, 1, 3)
    hidden = (j > (nk - nq)[:, None, None] + i[None, :, None]).repeat_interleave(group, 1)  # [b, most * group, keys]
    x = (q @ k).mul_(scale).masked_fill_(hidden, -math.inf)
    top = x.amax(-1, keepdim=True)
    out = torch.empty_like(q)
    first = 0
    for p, n in enumerate(members):
        part = slice(first, first + n)
        qp = q[:, part].reshape(hk, -1, d)
        px = (qp @ s["prefix_k"][p].float().permute(1, 2, 0)).mul_(scale)
        px.masked_fill_(torch.arange(case["prefix"], device=DEVICE) >= s["prefix_len"][p], -math.inf)
        m = torch.maximum(px.amax(-1, keepdim=True), top[:, part].reshape(hk, -1, 1))
        px.sub_(m).exp_()
        ox = (x[:, part] - m.view(hk, n, -1, 1)).exp_()
        total = px.sum(-1, keepdim=True).view(hk, n, -1, 1) + ox.sum(-1, keepdim=True)
        y = (px @ s["prefix_v"][p].float().permute(1, 0, 2)).view(hk, n, -1, d) + ox @ v[:, part]
        out[:, part] = y / total
        first += n
    out = out.view(hk, b, most, group, d).permute(1, 2, 0, 3, 4).reshape(b, most, h, d)
    return out[is_row].to(s["out"].dtype)


# ---------------------------------------------------------------- the library's calls

def _ptr(t, offset=0):
    return None if t is None else t.data_ptr() + offset * t.element_size()


def _own_args(s):
    """The description of a call, which a program makes once for its buffers."""
    from paper_2609_10018_gb300 import binding
    case = s["case"]
    types = {"f32": binding.F32, "bf16": binding.BF16, "f16": binding.F16, "e4m3": binding.E4M3}
    if case["kind"] == "residual":
        cols, mod, fp8 = case["cols"], s.get("mod"), case["z"] == "e4m3"
        return binding.ResidualNorm(
            rows=case["rows"], cols=cols, eps=EPS, x_factor=1.0,
            x_type=types[case["x"]], x=_ptr(s["x"]), x_row=s["x"].stride(0), x_out=_ptr(s["x_out"]), x_out_row=s["x_out"].stride(0),
            y_type=types[case["y"]], y=_ptr(s["y"]), y_row=s["y"].stride(0),
            post_norm=NORMS[case["post"]], post_gain=_ptr(s["post_gain"]), post_bias=_ptr(s["post_bias"]), y_scale=_ptr(s["y_scale"]),
            pre_norm=NORMS[case["pre"]], pre_gain=_ptr(s["pre_gain"]), pre_bias=_ptr(s["pre_bias"]),
            groups=case["groups"] if mod is not None else 0, group=_ptr(s.get("group")),
            mod_type=types[case["mod"]] if mod is not None else 0, mod_row=mod.stride(0) if mod is not None else 0,
            gate=_ptr(mod), shift=_ptr(mod, cols) if mod is not None else None, scale=_ptr(mod, 2 * cols) if mod is not None else None,
            z_type=types[case["z"]], z=_ptr(s["z"]), z_row=s["z"].stride(0),
            z_scale=_ptr(s["z_scale"]) if fp8 else None, z_scale_row=s["z_scale"].stride(0) if fp8 else 0)
    if case["kind"] == "rope":
        hq, hk, d, cached = case["heads_q"], case["heads_k"], case["dim"], case["cache_rows"] > 0
        qkv, row = s["qkv"], s["qkv"].stride(0)
        return binding.QkNormRopeAxes(
            dtype=types[case["type"]], rows=qkv.shape[0], heads_q=hq, heads_k=hk, head_dim=d, rot_dim=s["rot"],
            pairing=PAIRINGS[case["pairing"]], norm=int(case["norm"]), eps=EPS,
            q=_ptr(qkv), q_row=row, q_head=d, k=_ptr(qkv, hq * d), k_row=row, k_head=d,
            v=_ptr(qkv, (hq + hk) * d) if cached else None, v_row=row, v_head=d,
            q_out=_ptr(s["q_out"]), q_out_row=hq * d, q_out_head=d, k_out=_ptr(s["k_out"]), k_out_row=hk * d, k_out_head=d,
            v_out=_ptr(s["v_out"]) if cached else None, v_out_row=hk * d, v_out_head=d,
            q_gain=_ptr(s["gain_q"]), k_gain=_ptr(s["gain_k"]), cos_sin=_ptr(s["table"]), n_positions=s["table"].shape[0],
            axes=3, axis_of=(ctypes.c_uint8 * len(s["axis_of"]))(*s["axis_of"]),
            positions=_ptr(s["pos"]), positions_row=1, positions_axis=s["pos"].stride(0),
            slots=_ptr(s["slots"]) if cached else None, n_slots=case["cache_rows"])
    packed, q, k, v, out = case["packed"], s["q"], s["k"], s["v"], s["out"]
    pk, pv = s["prefix_k"], s["prefix_v"]
    args = binding.PrefixAttention(
        dtype=types[case["type"]], batch=case["batch"], heads=case["heads"], heads_kv=case["heads_kv"], head_dim=case["dim"],
        scale=1 / math.sqrt(case["dim"]), max_queries=case["queries"], q_rows=q.shape[0], q_start=_ptr(s["q_start"]),
        q=_ptr(q), q_row=q.stride(0), q_head=q.stride(1), out=_ptr(out), out_row=out.stride(0), out_head=out.stride(1),
        prefixes=case["prefixes"], seq_start=_ptr(s["seq_start"]), max_prefix=case["prefix"], prefix_rows=pk.shape[1],
        prefix_len=_ptr(s["prefix_len"]), prefix_k=_ptr(pk), prefix_k_batch=pk.stride(0), prefix_k_row=pk.stride(1), prefix_k_head=pk.stride(2),
        prefix_v=_ptr(pv), prefix_v_batch=pv.stride(0), prefix_v_row=pv.stride(1), prefix_v_head=pv.stride(2),
        max_keys=case["keys"], kv_rows=k.shape[0] if packed else case["keys"],
        kv_start=_ptr(s.get("kv_start")), kv_len=_ptr(s.get("kv_len")),
        k=_ptr(k), k_batch=0 if packed else k.stride(0), k_row=k.stride(-3), k_head=k.stride(-2),
        v=_ptr(v), v_batch=0 if packed else v.stride(0), v_row=v.stride(-3), v_head=v.stride(-2))
    s["workspace"] = torch.empty(max(16, binding.elasto_op_prefix_attention_workspace(args)), dtype=torch.uint8, device=DEVICE)
    args.workspace, args.workspace_bytes = s["workspace"].data_ptr(), s["workspace"].numel()
    return args


def _own_run(s):
    from paper_2609_10018_gb300 import binding
    stream, case = torch.cuda.current_stream().cuda_stream, s["case"]
    if case["kind"] == "residual":
        binding.elasto_op_residual_norm(stream, s["args"])
        return [s["x_out"], s["z"]] + ([s["z_scale"]] if case["z"] == "e4m3" else [])
    if case["kind"] == "rope":
        binding.elasto_op_qk_norm_rope_axes(stream, s["args"])
        return [s["q_out"], s["k_out"]] + ([s["v_out"]] if case["cache_rows"] else [])
    binding.elasto_op_prefix_attention(stream, s["args"])
    return s["out"]


def run(state):
    if own:
        return _own_run(state)
    return {"residual": _plain_residual, "rope": _plain_rope, "prefix": _plain_prefix}[state["case"]["kind"]](state)


# ---------------------------------------------------------------- work

def work(case):
    if case["kind"] == "residual":
        n, cols = case["rows"] * case["cols"], case["cols"]
        size = 2 * SIZES[case["x"]] + SIZES[case["y"]] + SIZES[case["z"]]
        vectors = (2 if case["affine"] else 0) + case["y_scale"]
        mod = (3 * SIZES[case["mod"]] * case["groups"] * cols + 4 * case["rows"]) if case["mod"] != "none" else 0
        scales = 4 * _blocks(cols) * case["rows"] if case["z"] == "e4m3" else 0
        return {"bytes": n * size + 4 * cols * vectors + mod + scales, "flops": 16 * n}
    if case["kind"] == "rope":
        rows, rot = _rope_rows(case), 2 * sum(_pairs(case))
        values = rows * (case["heads_q"] + case["heads_k"]) * case["dim"]
        copied = 2 * rows * case["heads_k"] * case["dim"] if case["cache_rows"] else 0
        table = 4 * rot * min(rows, max(_grid(case)) + case["front"])
        return {"bytes": 4 * values + 2 * copied + table + 12 * rows, "flops": 8 * values}
    members, prefix, nq, nk = _prefix_lengths(case)
    h, hk, d = case["heads"], case["heads_kv"], case["dim"]
    pairs, first = 0, 0
    for n, p in zip(members, prefix):
        for b in range(first, first + n):
            pairs += nq[b] * (p + nk[b] - nq[b]) + nq[b] * (nq[b] + 1) // 2
        first += n
    return {"bytes": 2 * d * (2 * h * sum(nq) + 2 * hk * (sum(prefix) + sum(nk))), "flops": 4 * d * h * pairs}


# ---------------------------------------------------------------- 64 bits

def _exact_norm(x, kind, gain, bias):
    """By the mean and the mean square, or the variance about the mean."""
    if kind == "none":
        return x
    if kind == "layer":
        var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
        y = (x - mean) / (var + EPS).sqrt()
    else:
        y = x / (x.square().sum(1, keepdim=True) / x.shape[1] + EPS).sqrt()
    y = y if gain is None else y * gain.double()
    return y if bias is None else y + bias.double()


def _exact_residual(case, s):
    """Some thousand rows at a time."""
    cols, outs = case["cols"], []
    for lo in range(0, case["rows"], 8192):
        rows = slice(lo, lo + 8192)
        u = _exact_norm(s["y"][rows].double(), case["post"], s["post_gain"], s["post_bias"])
        if s["y_scale"] is not None:
            u *= s["y_scale"].double()
        if case["mod"] != "none":
            gate, shift, scale = s["mod"].double().split(cols, 1)
            which = s["group"][rows].long()
            u *= gate[which]
        x = s["x"][rows].double() + u
        z = _exact_norm(x, case["pre"], s["pre_gain"], s["pre_bias"])
        if case["mod"] != "none":
            z = torch.addcmul(shift[which] + z, scale[which], z)
        if case["z"] == "e4m3":
            codes, scales = [], []
            for part in z.split(128, 1):
                a = part.abs().max(1).values.clamp_min(MIN_AMAX)
                codes.append((part * (FP8_MAX / a)[:, None]).to(torch.float8_e4m3fn).double())
                scales.append(a / FP8_MAX)
            outs.append([x, torch.cat(codes, 1), torch.stack(scales, 1)])
        else:
            outs.append([x, z])
    out = [torch.cat(part) for part in zip(*outs)]
    return out[:2] + [o.t() for o in out[2:]]


def _exact_rope(case, s):
    """The rotation as a product with e^(i angle), pair by pair, channels put in pairs and back by one permutation."""
    hq, hk, half = case["heads_q"], case["heads_k"], s["rot"] // 2
    pairs, placed, done = [], [], 0
    if case["pairing"] == "axis":
        for n in _pairs(case):
            pairs += [(done + i, done + n + i) for i in range(n)]
            done += 2 * n
    else:
        pairs = [(2 * i, 2 * i + 1) if case["pairing"] == "neighbours" else (i, half + i) for i in range(half)]
    placed = torch.tensor([c for p in pairs for c in p], dtype=torch.long, device=DEVICE)
    table = s["table"].double()
    turn = torch.stack([torch.complex(table[:, j], table[:, half + j])[s["pos"][a].long()] for j, a in enumerate(s["axis_of"])], 1)
    x = s["qkv"].double()
    outs = []
    for part, gain in ((x[:, :hq], s["gain_q"]), (x[:, hq:hq + hk], s["gain_k"])):
        if case["norm"]:
            part = part / (part.square().mean(2, keepdim=True) + EPS).sqrt() * gain.double()
        z = torch.view_as_complex(part[..., placed].unflatten(-1, (-1, 2)).contiguous()) * turn[:, None]
        outs.append(part.clone().index_copy_(2, placed, torch.view_as_real(z).flatten(-2)))
    if not case["cache_rows"]:
        return outs
    k, v = s["k_out"].double(), s["v_out"].double()
    k[s["slots"].long()], v[s["slots"].long()] = outs[1], x[:, hq + hk:]
    return [outs[0], k, v]


def _exact_prefix(case, s):
    """Sequence by sequence: its prefix's keys and its own in one row, a softmax for each head."""
    members, prefix, nq, nk = _prefix_lengths(case)
    group = case["heads"] // case["heads_kv"]
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEVICE)
    b = row = own_row = 0
    for p, n in enumerate(members):
        pk, pv = s["prefix_k"][p, :prefix[p]].double(), s["prefix_v"][p, :prefix[p]].double()
        for b in range(b, b + n):
            where = (slice(own_row, own_row + nk[b]),) if case["packed"] else (b, slice(0, nk[b]))
            k, v = torch.cat([pk, s["k"][where].double()]), torch.cat([pv, s["v"][where].double()])
            q = s["q"][row:row + nq[b]].double().unflatten(1, (-1, group))
            x = torch.einsum("ihgd,jhd->hgij", q, k) / math.sqrt(case["dim"])
            last = prefix[p] + nk[b] - nq[b] + torch.arange(nq[b], device=DEVICE)[:, None]
            x.masked_fill_(torch.arange(k.shape[0], device=DEVICE) > last, -math.inf)
            out[row:row + nq[b]] = torch.einsum("hgij,jhd->ihgd", torch.softmax(x, -1), v).flatten(1, 2)
            row, own_row = row + nq[b], own_row + nk[b]
        b += 1
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return {"residual": _exact_residual, "rope": _exact_rope, "prefix": _exact_prefix}[case["kind"]](case, s)
