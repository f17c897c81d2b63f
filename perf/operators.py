"""The operators of one attention sublayer over long token sequences with 8-bit weights:

  quantize   rows -> e4m3 values with an fp32 scale for each block of 128 (elasto_op_quantize_fp8);
  gemm       matrix product of such rows with block-scaled e4m3 weights (elasto_op_gemm_fp8);
  rope       RMS norm of each query and key head with the position rotation, K and V
             optionally written to their cache rows (elasto_op_qk_norm_rope);
  attention  attention with a sliding window and a few first tokens that stay visible
             (elasto_op_window_attention): whole sequences, chunks behind a cache, single tokens.

`own` chooses between the plain form of each (elementary torch operations in 32 bits) and the
library's call.
"""
import math
import random

import numpy as np
import torch

own = False

DEVICE = "cuda"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
FP8_MAX = 448.0
MIN_AMAX = 2.0 ** -100


def listed():
    return [
        # the normalised tokens of the largest ViT-B batch (256 images of 197 tokens) before a projection
        {"name": "quantize_256", "kind": "quantize", "type": "bf16", "rows": 50432, "cols": 768},
        # one image's fp32 stream: latency
        {"name": "quantize_1", "kind": "quantize", "type": "f32", "rows": 197, "cols": 768},
        # QKV projection of the largest ViT-B batch
        {"name": "gemm_qkv_256", "kind": "gemm", "epilogue": "bias", "M": 50432, "N": 2304, "K": 768},
        # a wide projection with a long reduction, where the arithmetic sets the pace
        {"name": "gemm_wide", "kind": "gemm", "epilogue": "bias", "M": 8192, "N": 8192, "K": 4096},
        # MLP up-projection + GELU of the 50 % mode at a middling batch (32 x 197 tokens)
        {"name": "gemm_gelu_32", "kind": "gemm", "epilogue": "gelu", "M": 6304, "N": 1536, "K": 768},
        # a projection of eight single tokens: the weights' bytes and latency
        {"name": "gemm_tokens_8", "kind": "gemm", "epilogue": "f32", "M": 8, "N": 4096, "K": 4096},
        # queries and keys of eight 1024 x 1024 images (4096 patches and the class token), ViT-B heads
        {"name": "rope_images_8", "kind": "rope", "type": "bf16", "rows": 32776, "heads_q": 12, "heads_k": 12,
         "dim": 64, "rot": 64, "interleaved": False, "cache_rows": 0, "positions": 4097},
        # one new token of each of 64 sequences, K and V into the cache
        {"name": "rope_decode_64", "kind": "rope", "type": "bf16", "rows": 64, "heads_q": 32, "heads_k": 8,
         "dim": 128, "rot": 128, "interleaved": False, "cache_rows": 16384, "positions": 131072},
        # 1024 x 1024 images: a band of patches around each, the class token sees and is seen by all
        {"name": "attention_images_4", "kind": "attention", "type": "bf16", "causal": False, "packed": True, "batch": 4,
         "queries": 4097, "keys": 4097, "ragged": 0, "heads": 12, "heads_kv": 12, "dim": 64, "window": 256, "sinks": 1},
        # token streams of different lengths, causal, queries sharing key heads
        {"name": "attention_prefill", "kind": "attention", "type": "bf16", "causal": True, "packed": True, "batch": 3,
         "queries": 8192, "keys": 8192, "ragged": 5, "heads": 32, "heads_kv": 8, "dim": 128, "window": 1024, "sinks": 4},
        # one new token of each of 64 sequences against caches of up to 8192
        {"name": "attention_decode_64", "kind": "attention", "type": "bf16", "causal": True, "packed": False, "batch": 64,
         "queries": 1, "keys": 8192, "ragged": 7, "heads": 32, "heads_kv": 8, "dim": 128, "window": 4095, "sinks": 4},
        # one token of one sequence: latency
        {"name": "attention_decode_1", "kind": "attention", "type": "f16", "causal": True, "packed": False, "batch": 1,
         "queries": 1, "keys": 2000, "ragged": 0, "heads": 12, "heads_kv": 12, "dim": 64, "window": 1023, "sinks": 4},
    ]


def _log_uniform(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["quantize", "gemm", "gemm", "rope", "attention", "attention", "attention"])
    if kind == "quantize":
        return {"kind": kind, "type": rng.choice(["bf16", "f16", "f32"]), "rows": _log_uniform(rng, 1, 50000),
                "cols": _log_uniform(rng, 64, 8192)}
    if kind == "gemm":
        m, n, k = _log_uniform(rng, 1, 50000), _log_uniform(rng, 64, 8192), _log_uniform(rng, 128, 8192)
        m = max(1, min(m, 8192 * 8192 * 4096 // (n * k)))
        return {"kind": kind, "epilogue": rng.choice(["bias", "gelu", "f32"]), "M": m, "N": n, "K": k}
    if kind == "rope":
        dim = rng.choice([64, 80, 96, 128, 256])
        group, heads_k = rng.choice([1, 2, 4, 8]), _log_uniform(rng, 1, 12)
        rows = _log_uniform(rng, 1, 200000 * 64 * 32 // (heads_k * (group + 1) * dim) // 4)
        return {"kind": kind, "type": rng.choice(["bf16", "f16"]), "rows": rows, "heads_q": heads_k * group,
                "heads_k": heads_k, "dim": dim, "rot": rng.choice([dim, dim // 32 * 16]),
                "interleaved": rng.random() < 0.5, "cache_rows": rng.choice([0, rows + rng.randrange(0, 999)]),
                "positions": _log_uniform(rng, 64, 100000)}
    form = rng.choice(["images", "prefill", "chunk", "decode"])
    heads_kv, group = rng.choice([1, 2, 3, 4, 8]), rng.choice([1, 2, 3, 4, 7, 8])
    case = {"kind": kind, "type": rng.choice(["bf16", "f16"]), "causal": form != "images",
            "packed": form in ("images", "prefill"), "batch": _log_uniform(rng, 1, 64 if form == "decode" else 8),
            "queries": 1, "keys": _log_uniform(rng, 16, 8192), "ragged": rng.randrange(0, 100),
            "heads": heads_kv * group, "heads_kv": heads_kv, "dim": rng.choice([32, 64, 80, 128, 128]),
            "window": rng.choice([-1, _log_uniform(rng, 16, 4096)]), "sinks": rng.choice([0, 1, 4, 16])}
    if case["packed"]:
        case["keys"] = case["queries"] = max(16, min(case["keys"], int(math.sqrt(2.5e9 / case["batch"] / case["heads"]))))
    elif form == "chunk":
        case["queries"] = min(case["keys"], _log_uniform(rng, 2, 512))
    return case


# ---------------------------------------------------------------- inputs

def _generator(seed):
    return torch.Generator(device=DEVICE).manual_seed(int(seed))


def _normal(shape, g, std=1.0):
    return torch.randn(shape, generator=g, device=DEVICE) * std


def _activations(rows, cols, g):
    """Normalised tokens: a few channels are much larger than the rest, as in trained transformers."""
    x = _normal((rows, cols), g)
    return x * torch.exp(0.5 * _normal((cols,), g))


def _blocks(n):
    return -(-n // 128)


def _quantize(x):
    """x [rows, cols] fp32 -> e4m3 [rows, cols], scales [blocks, rows]."""
    rows, cols = x.shape
    nb = _blocks(cols)
    xb = torch.nn.functional.pad(x, (0, nb * 128 - cols)).view(rows, nb, 128)
    amax = xb.abs().amax(-1).clamp_min(MIN_AMAX)
    # (the numerator on the device: dividing a Python number by a tensor takes a reciprocal first)
    q = (xb * (torch.full_like(amax, FP8_MAX) / amax)[..., None]).view(rows, nb * 128)[:, :cols]
    return q.to(torch.float8_e4m3fn), (amax / torch.full_like(amax, FP8_MAX)).t().contiguous()


def _padded_codes(q):
    """Rows on 16-byte boundaries, as the product reads them."""
    rows, cols = q.shape
    out = torch.zeros((rows, -(-cols // 16) * 16), dtype=torch.uint8, device=DEVICE)
    out[:, :cols] = q.view(torch.uint8)
    return out.view(torch.float8_e4m3fn)


def _block_weights(n, k, g):
    """N(0, 0.02) weights in e4m3 with one scale for each 128 x 128 block."""
    w = _normal((n, k), g, 0.02)
    wb = torch.nn.functional.pad(w, (0, _blocks(k) * 128 - k, 0, _blocks(n) * 128 - n)).view(_blocks(n), 128, _blocks(k), 128)
    scale = wb.abs().amax((1, 3)).clamp_min(MIN_AMAX) / FP8_MAX
    q = (wb / scale[:, None, :, None]).clamp(-FP8_MAX, FP8_MAX).view(_blocks(n) * 128, _blocks(k) * 128)[:n, :k]
    return q.to(torch.float8_e4m3fn), scale.contiguous()


def _lengths(case):
    """(queries, keys) of each sequence: all full, or spread over the range by the case's number."""
    b, nq, nk = case["batch"], case["queries"], case["keys"]
    if not case["ragged"]:
        return [nq] * b, [nk] * b
    r = random.Random(case["ragged"])
    lo = max(1, nk // 4)
    keys = [nk] + [r.randint(lo, nk) for _ in range(b - 1)]
    if case["packed"]:
        return list(keys), keys
    return [min(nq, k) if i % 2 == 0 else max(1, min(nq, k) // 2) for i, k in enumerate(keys)], keys


def _starts(lengths):
    return [0] + np.cumsum(lengths).tolist()


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEVICE)


def prepare(case, seed):
    g = _generator(seed)
    s = {"case": case}
    kind = case["kind"]
    if kind == "quantize":
        s["x"] = _activations(case["rows"], case["cols"], g).to(TYPES[case["type"]])
        s["q"] = torch.empty((case["rows"], case["cols"]), dtype=torch.float8_e4m3fn, device=DEVICE)
        s["scale"] = torch.empty((_blocks(case["cols"]), case["rows"]), device=DEVICE)
    elif kind == "gemm":
        m, n, k = case["M"], case["N"], case["K"]
        a, s["a_scale"] = _quantize(_activations(m, k, g))
        w, s["w_scale"] = _block_weights(n, k, g)
        s["a"], s["w"] = _padded_codes(a), _padded_codes(w)
        s["bias"] = _normal((n,), g, 0.05)
        s["out"] = torch.empty((m, n), dtype=torch.float32 if case["epilogue"] == "f32" else torch.bfloat16, device=DEVICE)
    elif kind == "rope":
        rows, hq, hk, d, rot = case["rows"], case["heads_q"], case["heads_k"], case["dim"], case["rot"]
        t = TYPES[case["type"]]
        s["qkv"] = _normal((rows, hq + 2 * hk, d), g).to(t)  # as the QKV product writes it
        s["gain_q"], s["gain_k"] = 1 + 0.1 * _normal((d,), g), 1 + 0.1 * _normal((d,), g)
        inv = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=DEVICE) / max(rot, 1))
        angle = torch.arange(case["positions"], dtype=torch.float64, device=DEVICE)[:, None] * inv
        s["table"] = torch.cat([angle.cos(), angle.sin()], 1).float().contiguous()
        s["pos"] = torch.randint(0, case["positions"], (rows,), generator=g, device=DEVICE, dtype=torch.int32)
        s["q_out"] = torch.empty((rows, hq, d), dtype=t, device=DEVICE)
        out_rows = case["cache_rows"] or rows
        s["k_out"] = torch.zeros((out_rows, hk, d), dtype=t, device=DEVICE)
        if case["cache_rows"]:
            s["slots"] = torch.randperm(out_rows, generator=g, device=DEVICE)[:rows].to(torch.int32)
            s["v_out"] = torch.zeros((out_rows, hk, d), dtype=t, device=DEVICE)
    else:
        t, d, h, hk = TYPES[case["type"]], case["dim"], case["heads"], case["heads_kv"]
        nq, nk = _lengths(case)
        if case["packed"]:  # q, k and v are columns of one projection's output
            qkv = _normal((sum(nq), h + 2 * hk, d), g).to(t)
            s["q"], s["k"], s["v"] = qkv[:, :h], qkv[:, h:h + hk], qkv[:, h + hk:]
            s["kv_start"] = _int32(_starts(nk))
        else:
            s["q"] = _normal((sum(nq), h, d), g).to(t)
            s["k"] = _normal((case["batch"], case["keys"], hk, d), g).to(t)
            s["v"] = _normal((case["batch"], case["keys"], hk, d), g).to(t)
            s["kv_len"] = _int32(nk)
        s["q_start"] = _int32(_starts(nq))
        s["out"] = torch.empty((sum(nq), h, d), dtype=t, device=DEVICE)
    return s


# ---------------------------------------------------------------- plain forms

def _dequantized(q, k, scale_rows):
    """fp32 values of e4m3 rows: scale_rows [rows, blocks]."""
    return q[:, :k].float() * scale_rows.repeat_interleave(128, 1)[:, :k]


def _plain_gemm(s):
    case = s["case"]
    n, k = case["N"], case["K"]
    y = _dequantized(s["a"], k, s["a_scale"].t()) @ _dequantized(s["w"], k, s["w_scale"].repeat_interleave(128, 0)[:n]).t()
    y = y + s["bias"]
    if case["epilogue"] == "gelu":
        y = 0.5 * y * (1 + torch.erf(y * math.sqrt(0.5)))
    return y.to(s["out"].dtype)


def _rotated(x, cos, sin, rot, interleaved):
    """x [rows, heads, d]; cos, sin [rows, 1, rot / 2]."""
    r, rest = x[..., :rot], x[..., rot:]
    if interleaved:
        a, b = r[..., 0::2], r[..., 1::2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = r[..., :rot // 2], r[..., rot // 2:]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, rest], -1)


def _plain_rope(s):
    case = s["case"]
    hq, hk, rot = case["heads_q"], case["heads_k"], case["rot"]
    cs = s["table"][s["pos"].long()][:, None]
    cos, sin = cs[..., :rot // 2], cs[..., rot // 2:]

    def one(x, gain):
        x = x.float()
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * gain
        return _rotated(x, cos, sin, rot, case["interleaved"]).to(s["qkv"].dtype)

    q, k = one(s["qkv"][:, :hq], s["gain_q"]), one(s["qkv"][:, hq:hq + hk], s["gain_k"])
    if not case["cache_rows"]:
        return [q, k]
    s["k_out"][s["slots"].long()] = k
    s["v_out"][s["slots"].long()] = s["qkv"][:, hq + hk:]
    return [q, s["k_out"], s["v_out"]]


def _padded_rows(start, count, most, last):
    """[batch, most] row numbers of packed sequences (clamped), and which of them are rows of the sequence."""
    i = torch.arange(most, device=DEVICE)
    return (start[:, None] + i).clamp_max(last), i < count[:, None]


def _plain_attention(s):
    case = s["case"]
    h, hk, d, b = case["heads"], case["heads_kv"], case["dim"], case["batch"]
    w, sinks = case["window"], case["sinks"]
    q_start = s["q_start"].long()
    nq = q_start[1:] - q_start[:-1]
    rows, is_row = _padded_rows(q_start[:-1], nq, case["queries"], s["q"].shape[0] - 1)
    q = s["q"][rows].float().view(b, -1, hk, h // hk, d).permute(0, 2, 3, 1, 4).reshape(b, hk, -1, d)
    if case["packed"]:
        kv_start = s["kv_start"].long()
        nk = kv_start[1:] - kv_start[:-1]
        at, _ = _padded_rows(kv_start[:-1], nk, case["keys"], s["k"].shape[0] - 1)
        k, v = s["k"][at].float(), s["v"][at].float()
    else:
        nk, k, v = s["kv_len"].long(), s["k"].float(), s["v"].float()
    k, v = k.permute(0, 2, 3, 1), v.permute(0, 2, 1, 3)
    p = (nk - nq)[:, None, None] + torch.arange(case["queries"], device=DEVICE)[None, :, None]
    j = torch.arange(case["keys"], device=DEVICE)
    near = torch.ones_like(p + j, dtype=torch.bool) if w < 0 else p - j <= w
    if case["causal"]:
        seen = (near | (j < sinks)) & (j <= p)
    else:
        seen = (near & ((w < 0) | (j - p <= w))) | (j < sinks) | (p < sinks)
    seen = seen & (j < nk[:, None, None]) & (p >= 0)
    x = (q @ k).mul_(1 / math.sqrt(d)).view(b, h, -1, case["keys"])
    x = x.masked_fill_(~seen[:, None], -math.inf)
    top = x.amax(-1, keepdim=True).clamp_min(-3e38)
    x = x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    y = (x.view(b, hk, -1, case["keys"]) @ v).view(b, h, -1, d) / total.clamp_min(1e-30)
    return y.transpose(1, 2)[is_row].to(s["out"].dtype)


# ---------------------------------------------------------------- the library's calls

def _own_run(s):
    from paper_2609_10018_gb300 import binding
    case = s["case"]
    kind = case["kind"]
    stream = torch.cuda.current_stream().cuda_stream
    if kind == "quantize":
        x, q, scale = s["x"], s["q"], s["scale"]
        dtype = {"bf16": binding.BF16, "f16": binding.F16, "f32": binding.F32}[case["type"]]
        binding.elasto_op_quantize_fp8(stream, x.data_ptr(), dtype, x.stride(0), q.data_ptr(), q.stride(0), scale.data_ptr(),
                                       scale.stride(0), case["rows"], case["cols"])
        return [q, scale]
    if kind == "gemm":
        epilogue = {"bias": binding.EPI_BIAS_BF16, "gelu": binding.EPI_BIAS_GELU_BF16, "f32": binding.EPI_BIAS_F32}
        a, w, out = s["a"], s["w"], s["out"]
        binding.elasto_op_gemm_fp8(stream, a.data_ptr(), a.stride(0), s["a_scale"].data_ptr(), s["a_scale"].stride(0),
                                   w.data_ptr(), w.stride(0), s["w_scale"].data_ptr(), s["bias"].data_ptr(), out.data_ptr(),
                                   out.stride(0), case["M"], case["N"], case["K"], epilogue[case["epilogue"]])
        return out
    dtype = binding.BF16 if case["type"] == "bf16" else binding.F16
    if kind == "rope":
        hq, hk, d = case["heads_q"], case["heads_k"], case["dim"]
        qkv, cached = s["qkv"], case["cache_rows"] > 0
        row, at = qkv.stride(0), qkv.data_ptr()
        binding.elasto_op_qk_norm_rope(stream, binding.QkNormRope(
            dtype=dtype, rows=case["rows"], heads_q=hq, heads_k=hk, head_dim=d, rot_dim=case["rot"],
            interleaved=int(case["interleaved"]), eps=1e-6,
            q=at, q_row=row, q_head=d, k=at + 2 * hq * d, k_row=row, k_head=d,
            v=at + 2 * (hq + hk) * d if cached else None, v_row=row, v_head=d,
            q_out=s["q_out"].data_ptr(), q_out_row=hq * d, q_out_head=d,
            k_out=s["k_out"].data_ptr(), k_out_row=hk * d, k_out_head=d,
            v_out=s["v_out"].data_ptr() if cached else None, v_out_row=hk * d, v_out_head=d,
            q_gain=s["gain_q"].data_ptr(), k_gain=s["gain_k"].data_ptr(), cos_sin=s["table"].data_ptr(),
            positions=s["pos"].data_ptr(), n_positions=case["positions"],
            slots=s["slots"].data_ptr() if cached else None, n_slots=case["cache_rows"]))
        return [s["q_out"], s["k_out"]] + ([s["v_out"]] if cached else [])
    q, k, v, out, packed = s["q"], s["k"], s["v"], s["out"], case["packed"]
    binding.elasto_op_window_attention(stream, binding.WindowAttention(
        dtype=dtype, batch=case["batch"], heads=case["heads"], heads_kv=case["heads_kv"], head_dim=case["dim"],
        causal=int(case["causal"]), window=case["window"], sinks=case["sinks"], scale=1 / math.sqrt(case["dim"]),
        max_queries=case["queries"], q_rows=q.shape[0], q_start=s["q_start"].data_ptr(),
        q=q.data_ptr(), q_row=q.stride(0), q_head=q.stride(1),
        out=out.data_ptr(), out_row=out.stride(0), out_head=out.stride(1),
        max_keys=case["keys"], kv_rows=k.shape[0] if packed else case["keys"],
        kv_start=s["kv_start"].data_ptr() if packed else None, kv_len=None if packed else s["kv_len"].data_ptr(),
        k=k.data_ptr(), k_batch=0 if packed else k.stride(0), k_row=k.stride(-3), k_head=k.stride(-2),
        v=v.data_ptr(), v_batch=0 if packed else v.stride(0), v_row=v.stride(-3), v_head=v.stride(-2)))
    return out


def run(state):
    if own:
        return _own_run(state)
    kind = state["case"]["kind"]
    if kind == "quantize":
        return list(_quantize(state["x"].float()))
    return {"gemm": _plain_gemm, "rope": _plain_rope, "attention": _plain_attention}[kind](state)


# ---------------------------------------------------------------- work

def _visible(case, nq, nk):
    """(pairs of a query and a key it sees, keys that some query sees) of one sequence."""
    w, sinks = case["window"], case["sinks"]
    p = np.arange(max(0, nk - nq), nk, dtype=np.int64)
    far = nk if w < 0 else w
    low = np.maximum(0, p - far)
    high = p if case["causal"] else np.minimum(nk - 1, p + far)
    first = np.minimum(np.minimum(sinks, low), p + 1 if case["causal"] else nk)  # sinks below the band
    count = high - low + 1 + first
    if not case["causal"]:
        count = count + np.clip(np.minimum(sinks, nk) - (high + 1), 0, None)  # sinks above the band
        count = np.where(p < sinks, nk, count)
        if sinks > 0 and p[0] < sinks:
            return int(count.sum()), nk
    return int(count.sum()), int(high.max() - low.min() + 1 + min(sinks, low.min()))


def work(case):
    kind = case["kind"]
    if kind == "quantize":
        rows, cols = case["rows"], case["cols"]
        size = 4 if case["type"] == "f32" else 2
        return {"bytes": rows * cols * (size + 1) + 4 * rows * _blocks(cols), "flops": 3 * rows * cols}
    if kind == "gemm":
        m, n, k = case["M"], case["N"], case["K"]
        scales = 4 * _blocks(k) * (m + _blocks(n))
        return {"bytes": m * k + n * k + scales + 4 * n + (4 if case["epilogue"] == "f32" else 2) * m * n,
                "flops": 2 * m * n * k}
    if kind == "rope":
        values = case["rows"] * (case["heads_q"] + case["heads_k"]) * case["dim"]
        copied = 2 * case["rows"] * case["heads_k"] * case["dim"] if case["cache_rows"] else 0
        tables = 4 * case["rot"] * min(case["rows"], case["positions"]) + 8 * case["rows"]
        return {"bytes": 4 * values + 2 * copied + tables, "flops": 8 * values}
    nq, nk = _lengths(case)
    seen = [_visible(case, a, b) for a, b in zip(nq, nk)]
    d = case["dim"]
    return {"bytes": 2 * d * (2 * sum(nq) * case["heads"] + 2 * sum(k for _, k in seen) * case["heads_kv"]),
            "flops": 4 * d * case["heads"] * sum(p for p, _ in seen)}


# ---------------------------------------------------------------- 64 bits

def _exact_quantize(case, s):
    """The block maxima and scales in 64 bits, values rounded to e4m3 once."""
    x = s["x"].double()
    codes, scales = [], []
    for part in x.split(128, 1):
        a = part.abs().max(1).values.clamp_min(MIN_AMAX)
        codes.append((part * (FP8_MAX / a)[:, None]).to(torch.float8_e4m3fn).double())
        scales.append(a / FP8_MAX)
    return [torch.cat(codes, 1), torch.stack(scales)]


def _exact_gemm(case, s):
    n, k = case["N"], case["K"]
    out = s["bias"].double().expand(case["M"], n).clone()
    for b in range(_blocks(k)):
        cols = slice(128 * b, min(k, 128 * b + 128))
        part = s["a"][:, cols].double() @ s["w"][:, cols].double().t()
        row = s["w_scale"][:, b].double()[torch.arange(n, device=DEVICE) // 128]
        out += part * s["a_scale"][b].double()[:, None] * row
    return torch.nn.functional.gelu(out) if case["epilogue"] == "gelu" else out


def _exact_rope(case, s):
    """The rotation as a product with e^(i angle) of complex pairs."""
    hq, hk, rot = case["heads_q"], case["heads_k"], case["rot"]
    t = s["table"].double()[s["pos"].long()]
    turn = torch.complex(t[:, :rot // 2], t[:, rot // 2:])[:, None]
    x = s["qkv"].double()
    outs = []
    for part, gain in ((x[:, :hq], s["gain_q"]), (x[:, hq:hq + hk], s["gain_k"])):
        y = part / torch.sqrt(part.square().mean(2, keepdim=True) + 1e-6) * gain.double()
        r = y[..., :rot].clone()
        z = torch.view_as_complex(r.unflatten(-1, (-1, 2)).contiguous()) if case["interleaved"] else torch.complex(
            r[..., :rot // 2].contiguous(), r[..., rot // 2:].contiguous())
        z = z * turn
        r = torch.view_as_real(z).flatten(-2) if case["interleaved"] else torch.cat([z.real, z.imag], -1)
        outs.append(torch.cat([r, y[..., rot:]], -1))
    if not case["cache_rows"]:
        return outs
    k, v = s["k_out"].double(), s["v_out"].double()
    k[s["slots"].long()], v[s["slots"].long()] = outs[1], x[:, hq + hk:]
    return [outs[0], k, v]


def _exact_attention(case, s):
    """Sequence by sequence, head by head, 1024 queries at a time."""
    nq, nk = _lengths(case)
    w, sinks, group = case["window"], case["sinks"], case["heads"] // case["heads_kv"]
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEVICE)
    first_q, first_k = 0, 0
    for b in range(case["batch"]):
        k = s["k"][first_k:first_k + nk[b]] if case["packed"] else s["k"][b, :nk[b]]
        v = s["v"][first_k:first_k + nk[b]] if case["packed"] else s["v"][b, :nk[b]]
        j = torch.arange(nk[b], device=DEVICE)
        for lo in range(0, nq[b], 1024):
            hi = min(nq[b], lo + 1024)
            p = nk[b] - nq[b] + torch.arange(lo, hi, device=DEVICE)[:, None]
            far = (j - p).abs() > w if w >= 0 else torch.zeros_like(j - p, dtype=torch.bool)
            hidden = far & (j >= sinks)
            hidden = hidden | (j > p) if case["causal"] else hidden & (p >= sinks)
            for head in range(case["heads"]):
                q = s["q"][first_q + lo:first_q + hi, head].double()
                x = (q @ k[:, head // group].double().t()) / math.sqrt(case["dim"])
                prob = torch.softmax(x.masked_fill(hidden, -math.inf), -1)
                out[first_q + lo:first_q + hi, head] = prob @ v[:, head // group].double()
        first_q, first_k = first_q + nq[b], first_k + nk[b]
    return out


def exact(case, seed):
    s = prepare(case, seed)
    f = {"quantize": _exact_quantize, "gemm": _exact_gemm, "rope": _exact_rope, "attention": _exact_attention}
    return f[case["kind"]](case, s)
