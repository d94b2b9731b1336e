"""What a transformer layer computes beside its matrix products, as cases that can be timed and checked.

A case is a dict of plain values; ``kind`` names the calls that a pass makes:

  norm_fwd   fmt_layernorm_fwd: dropout of a sublayer's result, addition to the residual stream, layer norm
  norm_bwd   fmt_layernorm_bwd: the gradients of the same (input, residual, weight and bias)
  dropout    fmt_dropout: forward; the backward pass is the same call on the gradient
  attn_fwd   fmt_attention_fwd: attention with a sliding window and a few first tokens that stay visible
  attn_step  fmt_attention_fwd and fmt_attention_bwd: output and gradients
  attn_token fmt_attention_fwd with one query token per sequence over a cache of keys and values

``own`` chooses who computes: the framework's kernels, or the plain form in elementary torch operations in
32 bits.  Both take what :func:`prepare` gives.

``format`` is the 1/e/m format that the operands are rounded to ("1/8/23/d" is fp32: nothing is rounded);
``codes`` says that tensors are held as the format's own 16-bit codes (those of 1/5/10 and 1/8/7 are IEEE
half and bfloat16) instead of fp32.  Results of 1/5/10 and 1/8/7 codes are such codes again; all
others are unrounded fp32.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

FORMATS = {"1/5/10/d": (5, 10, True), "1/6/9/d": (6, 9, True), "1/8/7/n": (8, 7, False), "1/8/23/d": (8, 23, True)}
HALF = {"1/5/10/d": torch.float16, "1/8/7/n": torch.bfloat16}
EPS = 1e-5
SITE = 3


def listed():
    return [
        # the last norm of a small encoder (hidden size 128) on one sequence of 128 tokens: a call of a few microseconds
        {"name": "norm_fwd_small", "kind": "norm_fwd", "rows": 128, "cols": 128, "format": "1/6/9/d", "codes": False,
         "residual": True, "p": 0.1},
        # dropout, residual and norm behind a sublayer of the encoder step, 4096 tokens, bfloat16 activations
        {"name": "norm_fwd_encoder", "kind": "norm_fwd", "rows": 4096, "cols": 1024, "format": "1/8/7/n", "codes": True,
         "residual": True, "p": 0.1},
        # its backward pass
        {"name": "norm_bwd_encoder", "kind": "norm_bwd", "rows": 4096, "cols": 1024, "format": "1/8/7/n", "codes": True,
         "p": 0.1},
        # backward of a norm alone over a large batch, hidden size 768, an odd number of rows, values in 1/6/9 held in fp32
        {"name": "norm_bwd_large", "kind": "norm_bwd", "rows": 50001, "cols": 768, "format": "1/6/9/d", "codes": False, "p": 0.0},
        # the hidden layer of the 784-1024-1024-10 perceptron at batch 256
        {"name": "dropout_small", "kind": "dropout", "rows": 256, "cols": 1024, "format": "1/6/9/d", "codes": False, "p": 0.5},
        # a feed-forward layer's inner activations with an odd row length, binary16 codes
        {"name": "dropout_large", "kind": "dropout", "rows": 30011, "cols": 4097, "format": "1/5/10/d", "codes": True, "p": 0.1},
        # an encoder's attention over padded sequences: 32 sequences of up to 128 tokens, 12 heads of 64, every token sees every other
        {"name": "attn_encoder", "kind": "attn_fwd", "batch": 32, "q_len": 128, "k_len": 128, "heads": 12, "kv_heads": 12,
         "dim": 64, "causal": False, "window": 0, "sinks": 0, "ragged": True, "format": "1/6/9/d", "codes": False},
        # a training step's attention: 4096 tokens in 4 sequences, 16 heads of 64, the last 256 tokens and the first 4
        {"name": "attn_step_window", "kind": "attn_step", "batch": 4, "q_len": 1024, "k_len": 1024, "heads": 16, "kv_heads": 16,
         "dim": 64, "causal": True, "window": 256, "sinks": 4, "ragged": False, "format": "1/8/7/n", "codes": True},
        # odd lengths and head size, heads that share keys and values, padding, values in 1/6/9 held in fp32
        {"name": "attn_step_ragged", "kind": "attn_step", "batch": 3, "q_len": 777, "k_len": 777, "heads": 6, "kv_heads": 2,
         "dim": 40, "causal": True, "window": 0, "sinks": 0, "ragged": True, "format": "1/6/9/d", "codes": False},
        # reading a long document: 16384 tokens, the last 2048 and the first 16, binary16, heads of 128 that share keys and values
        {"name": "attn_long", "kind": "attn_fwd", "batch": 1, "q_len": 16384, "k_len": 16384, "heads": 8, "kv_heads": 2,
         "dim": 128, "causal": True, "window": 2048, "sinks": 16, "ragged": False, "format": "1/5/10/d", "codes": True},
        # serving: one new token for each of 48 sequences over a cache of up to 8191 tokens in 1/6/9 codes
        {"name": "attn_token", "kind": "attn_token", "batch": 48, "q_len": 1, "k_len": 8191, "heads": 16, "kv_heads": 4,
         "dim": 64, "causal": True, "window": 4096, "sinks": 4, "ragged": True, "format": "1/6/9/d", "codes": True},
        # serving one sequence: a single token over a long bfloat16 cache, where latency counts
        {"name": "attn_token_one", "kind": "attn_token", "batch": 1, "q_len": 1, "k_len": 32768, "heads": 8, "kv_heads": 8,
         "dim": 128, "causal": True, "window": 0, "sinks": 0, "ragged": False, "format": "1/8/7/n", "codes": True},
    ]


def draw(rng):
    def size(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(("norm_fwd", "norm_bwd", "dropout", "attn_fwd", "attn_step", "attn_token"))
    if kind in ("norm_fwd", "norm_bwd", "dropout"):
        format, codes = rng.choice((("1/8/7/n", True), ("1/5/10/d", True), ("1/6/9/d", False), ("1/8/23/d", False)))
        cols = size(1, 16384)
        case = {"kind": kind, "rows": size(1, min(100000, 100000000 // cols)), "cols": cols, "format": format, "codes": codes,
                "p": rng.choice((0.0, 0.1, 0.25, 0.5)) if kind != "dropout" else rng.choice((0.05, 0.1, 0.3, 0.5))}
        if kind == "norm_fwd":
            case["residual"] = rng.random() < 0.7
        return case
    format, codes = rng.choice((("1/8/7/n", True), ("1/5/10/d", True), ("1/6/9/d", False), ("1/6/9/d", True)))
    kv_heads = rng.choice((1, 2, 3, 4, 8))
    heads = kv_heads * rng.choice((1, 1, 2, 3, 4))
    most = 200_000_000 if kind == "attn_step" else 400_000_000      # pairs of a query and a key
    if kind == "attn_token":
        k_len, q_len = size(1, 32768), 1
        batch = size(1, max(1, min(64, 4_000_000 // (heads * k_len))))
    else:
        k_len = size(1, 8192 if kind == "attn_fwd" else 4096)
        q_len = k_len if kind == "attn_step" or rng.random() < 0.7 else size(1, k_len)
        batch = size(1, max(1, min(32, most // (heads * q_len * k_len))))
        while batch * heads * q_len * k_len > most:
            k_len = max(1, k_len // 2)
            q_len = min(q_len, k_len)
    return {"kind": kind, "batch": batch, "q_len": q_len, "k_len": k_len, "heads": heads, "kv_heads": kv_heads,
            "dim": rng.choice((16, 40, 64, 64, 80, 128, 128)), "causal": kind == "attn_token" or rng.random() < 0.7,
            "window": rng.choice((0, 0, size(1, k_len))), "sinks": rng.choice((0, 1, 4, 33)), "ragged": rng.random() < 0.4,
            "format": format, "codes": codes}


# ---------------------------------------------------------------------------------------------- formats

def _rounded(x, format):
    """fp32 to the nearest value of the format, ties to even, as fp32."""
    if format == "1/8/23/d":
        return x
    if format in HALF:
        r = x.to(HALF[format]).float()
        return torch.where(r.abs() < 2.0 ** -126, r * 0.0, r) if format == "1/8/7/n" else r
    q = (((x.view(torch.int32) >> 23) & 255) - 127).clamp_(min=-30) - 9          # 1/6/9: the step is 2^q
    step = ((q + 127) << 23).view(torch.float32)
    r = torch.round(x / step) * step
    return torch.where(r.abs() >= 2.0 ** 32, torch.copysign(torch.full_like(r, math.inf), r), torch.where(x.isnan(), x, r))


def _stored(x, case):
    """fp32 as a user's program holds it: rounded codes, or fp32."""
    if not case["codes"]:
        return x
    r = _rounded(x, case["format"])
    if case["format"] in HALF:
        return r.to(HALF[case["format"]])
    a = r.abs()
    small = (a * 2.0 ** 39).to(torch.int32)                                      # a multiple of the smallest denormal
    code = torch.where(a < 2.0 ** -30, small, (a.view(torch.int32) >> 14) - (96 << 9))
    code = torch.where(a == math.inf, 63 << 9, code)
    return (code | (torch.signbit(r).to(torch.int32) << 15)).to(torch.int16)


def _values(t, case):
    """What a stored tensor stands for, rounded to the format, in fp32."""
    if t is None:
        return None
    if not case["codes"]:
        return _rounded(t, case["format"])
    if case["format"] in HALF:
        return _rounded(t.float(), case["format"])
    c = t.to(torch.int32)
    body = c & 0x7FFF
    a = torch.where(body < 512, body * 2.0 ** -39, ((body << 14) + (96 << 23)).view(torch.float32))
    a = torch.where(body >= 63 << 9, torch.where(body == 63 << 9, math.inf, math.nan), a)
    return torch.where((c & 0x8000) != 0, -a, a)


def _result(x, case):
    return x.to(HALF[case["format"]]) if case["codes"] and case["format"] in HALF else x


# ---------------------------------------------------------------------------------------------- inputs

def _lens(case):
    """Lengths of the sequences: all of it, or, ragged, different ones of which the third is empty."""
    n, b = case["k_len"], np.arange(case["batch"], dtype=np.int64)
    if not case["ragged"]:
        return np.full(case["batch"], n, dtype=np.int64)
    return np.where(b == 2, 0, n - (b * 7919) % (n // 2 + 1))


def _positions(case):
    """Where each sequence's first query stands: a new token is the last of its sequence."""
    return _lens(case) - 1 if case["kind"] == "attn_token" else np.full(case["batch"], case["k_len"] - case["q_len"], dtype=np.int64)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    def gradient(*shape):                                   # scaled activation gradients: magnitudes over many binades
        return torch.exp2(normal(*shape) * 4.0 - 14.0) * torch.sign(normal(*shape))

    state = {"case": case}
    if case["kind"] in ("norm_fwd", "norm_bwd", "dropout"):
        rows, cols = case["rows"], case["cols"]
        state["rng"] = torch.tensor([int(seed) * 2654435761 % (1 << 62), 17], dtype=torch.int64, device="cuda")
        state["gamma"], state["beta"] = 1.0 + 0.2 * normal(cols), 0.1 * normal(cols)
        if case["kind"] == "norm_bwd":
            state["dy"] = _stored(gradient(rows, cols), case)
            state["z"] = _stored(0.3 + 2.0 * normal(rows, cols), case)
            z = _values(state["z"], case)
            state["mean"] = z.mean(1)
            state["rstd"] = torch.rsqrt((z - state["mean"][:, None]).square().mean(1) + EPS)
        else:
            state["x"] = _stored(normal(rows, cols), case)
            state["residual"] = _stored(0.3 + 2.0 * normal(rows, cols), case) if case.get("residual") else None
        return state
    b, n, h, hk, d = case["batch"], case["k_len"], case["heads"], case["kv_heads"], case["dim"]
    lens = torch.from_numpy(_lens(case)).to(device="cuda", dtype=torch.int32)
    state["k_lens"] = lens if case["ragged"] else None
    state["q_pos"] = torch.from_numpy(_positions(case)).to(device="cuda", dtype=torch.int32) if case["kind"] == "attn_token" else None
    if case["q_len"] == n and case["kind"] != "attn_token":      # the three parts of one projection's result
        whole = normal(b, n, h + 2 * hk, d)
    else:                                                        # queries on their own, keys and values in a cache with room to grow
        whole = normal(b, n + 5, 2 * hk, d)
        state["q"] = _stored(1.5 * normal(b, case["q_len"], h, d), case)
    past = torch.arange(whole.shape[1], device="cuda")[None, :] >= lens[:, None]
    whole = torch.where(past[:, :, None, None], math.nan, whole) if "q" in state else whole       # what a cache holds past its end is nobody's
    whole = _stored(whole, case) if "q" not in state else _stored(torch.nan_to_num(whole, nan=3e38), case)
    if "q" not in state:
        state["q"] = whole[:, :, :h]
    state["k"], state["v"] = whole[:, :n, -2 * hk:-hk], whole[:, :n, -hk:]
    if case["kind"] == "attn_step":
        state["do"] = _stored(gradient(b, case["q_len"], h, d), case) if _halves(case) else gradient(b, case["q_len"], h, d)
    return state


def _halves(case):
    return case["codes"] and case["format"] in HALF


# ---------------------------------------------------------------------------------------------- the operators

def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(state):
    import paper_2103_15940_amd as fmt
    case = state["case"]
    f = FORMATS[case["format"]]
    result = "code16" if _halves(case) else "f32"
    if case["kind"] == "norm_fwd":
        y, z, mean, rstd = fmt.fmt_layernorm_fwd(state["x"], state["gamma"], state["beta"], f, residual=state["residual"], p=case["p"],
                                                 rng=state["rng"], site=SITE, eps=EPS, result=result)
        return {"y": y, "z": z, "mean": mean, "rstd": rstd}
    if case["kind"] == "norm_bwd":
        dz, dx, dgamma, dbeta = fmt.fmt_layernorm_bwd(state["dy"], state["z"], state["mean"], state["rstd"], state["gamma"], f,
                                                      p=case["p"], rng=state["rng"], site=SITE, result=result)
        return {"dz": dz, "dx": dx if case["p"] else None, "dgamma": dgamma, "dbeta": dbeta}
    if case["kind"] == "dropout":
        return fmt.fmt_dropout(state["x"], case["p"], state["rng"], f, site=SITE, result=result)
    how = {"causal": case["causal"], "window": case["window"], "sinks": case["sinks"], "k_lens": state["k_lens"],
           "q_pos": state["q_pos"], "result": result}
    o, lse = fmt.fmt_attention_fwd(state["q"], state["k"], state["v"], f, **how)
    if case["kind"] != "attn_step":
        return {"o": o, "lse": lse}
    dq, dk, dv = fmt.fmt_attention_bwd(state["do"], state["q"], state["k"], state["v"], o, lse, f, **how)
    return {"o": o, "lse": lse, "dq": dq, "dk": dk, "dv": dv}


def _kept(rng, rows, cols, p):
    """Which elements a dropout keeps, and by what they are multiplied.  Block n of eight consecutive elements of a row takes the 128
    bits that Philox-4x32 (ten rounds) makes of the counter (n, n / 2^32, step, site) and the key `seed`, 16 bits each, low half first;
    an element is kept where its 16 bits are at least 65536 p."""
    mask = 0xFFFFFFFF
    blocks = (cols + 7) // 8
    n = torch.arange(rows * blocks, dtype=torch.int64, device=rng.device)
    c0, c1 = n & mask, n >> 32
    c2, c3 = (rng[1] & mask) + torch.zeros_like(n), torch.full_like(n, SITE)
    k0, k1 = rng[0] & mask, (rng[0] >> 32) & mask
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((b >> 32) & mask) ^ c1 ^ k0, b & mask, ((a >> 32) & mask) ^ c3 ^ k1, a & mask
        k0, k1 = (k0 + 0x9E3779B9) & mask, (k1 + 0xBB67AE85) & mask
    words = torch.stack((c0, c1, c2, c3), 1)
    bits = torch.stack((words & 0xFFFF, words >> 16), 2).reshape(rows, blocks * 8)[:, :cols]
    least = int(round(p * 65536))
    return bits >= least, float(np.float32(65536.0 / (65536 - least)))


def _run_plain(state):
    case = state["case"]
    if case["kind"] == "dropout":
        x = _values(state["x"], case)
        keep, scale = _kept(state["rng"], *x.shape, case["p"])
        return _result(torch.where(keep, x * scale, 0.0), case)
    if case["kind"] == "norm_fwd":
        z = _values(state["x"], case)
        if case["p"]:
            keep, scale = _kept(state["rng"], *z.shape, case["p"])
            z = torch.where(keep, z * scale, 0.0)
        if case["residual"]:
            z = _values(state["residual"], case) + z
        z = _rounded(z, case["format"])
        mean = z.mean(1)
        c = z - mean[:, None]
        rstd = torch.rsqrt(c.square().mean(1) + EPS)
        y = c * rstd[:, None] * _rounded(state["gamma"], case["format"]) + _rounded(state["beta"], case["format"])
        return {"y": _result(y, case), "z": _as_stored(z, case) if case["p"] or case["residual"] else None, "mean": mean, "rstd": rstd}
    if case["kind"] == "norm_bwd":
        dy, z = _values(state["dy"], case), _values(state["z"], case)
        xhat = (z - state["mean"][:, None]) * state["rstd"][:, None]
        g = dy * _rounded(state["gamma"], case["format"])
        dz = (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True)) * state["rstd"][:, None]
        dx = None
        if case["p"]:
            keep, scale = _kept(state["rng"], *z.shape, case["p"])
            dx = _result(torch.where(keep, dz * scale, 0.0), case)
        return {"dz": _result(dz, case), "dx": dx, "dgamma": (dy * xhat).sum(0), "dbeta": dy.sum(0)}
    return _attention_plain(state)


def _as_stored(z, case):
    return z.to(HALF[case["format"]]) if _halves(case) else z


def _attention_plain(state):
    case = state["case"]
    seen = _visible(case, state["q"].device)
    group, scale = case["heads"] // case["kv_heads"], case["dim"] ** -0.5
    q = _values(state["q"], case).transpose(1, 2)
    k, v = (_values(state[t], case).transpose(1, 2).repeat_interleave(group, 1).contiguous() for t in ("k", "v"))
    if state["k_lens"] is not None:
        past = (torch.arange(case["k_len"], device=q.device)[None, :] >= state["k_lens"][:, None])[:, None, :, None]
        k, v = k.masked_fill(past, 0.0), v.masked_fill(past, 0.0)
    s = (q @ k.transpose(2, 3) * scale).masked_fill(~seen, -math.inf)
    top = s.amax(3, keepdim=True)
    p = torch.exp(s - torch.where(top == -math.inf, 0.0, top))
    del s
    total = p.sum(3, keepdim=True)
    p /= torch.where(total == 0, 1.0, total)
    o = p @ v
    out = {"o": _result(o.transpose(1, 2), case), "lse": (top + torch.log(total)).squeeze(3)}
    if case["kind"] != "attn_step":
        return out
    do = (_values(state["do"], case) if _halves(case) else _rounded(state["do"], case["format"])).transpose(1, 2)
    dv = p.transpose(2, 3) @ do
    ds = p * (do @ v.transpose(2, 3) - (do * o).sum(3, keepdim=True)) * scale
    dq, dk = ds @ k, ds.transpose(2, 3) @ q
    shared = (case["batch"], case["kv_heads"], group, case["k_len"], case["dim"])
    dk, dv = dk.reshape(shared).sum(2), dv.reshape(shared).sum(2)
    out.update({name: _result(t.transpose(1, 2), case) for name, t in (("dq", dq), ("dk", dk), ("dv", dv))})
    return out


def _visible(case, device):
    """Which keys each query sees: [batch, 1, q_len, k_len]."""
    lens, first = (torch.from_numpy(a).to(device)[:, None, None, None] for a in (_lens(case), _positions(case)))
    i = first + torch.arange(case["q_len"], device=device)[:, None]
    j = torch.arange(case["k_len"], device=device)
    seen = (j < lens) & (i == i)
    if case["causal"]:
        seen = seen & (j <= i)
    if case["window"]:
        near = (j > i - case["window"]) & (j < i + case["window"])
        seen = seen & (near | (j < case["sinks"]))
    return seen


# ---------------------------------------------------------------------------------------------- what a pass cannot do without

def _pairs(case):
    """Pairs of a query and a key that it sees, and keys that some query sees, of one head over the batch."""
    total = keys = 0
    for length, first in zip(_lens(case), _positions(case)):
        i = first + np.arange(case["q_len"], dtype=np.int64)
        end = np.minimum(length, i + 1) if case["causal"] else np.full_like(i, length)
        start, sinks = np.zeros_like(i), np.zeros_like(i)
        if case["window"]:
            start = np.maximum(0, i - case["window"] + 1)
            end = np.minimum(end, i + case["window"])
            last = np.minimum(length, i + 1) if case["causal"] else np.full_like(i, length)
            sinks = np.maximum(0, np.minimum(np.minimum(start, case["sinks"]), last))
        total += int((np.maximum(0, end - start) + sinks).sum())
        covered = max(0, int(end.max()) - int(start.min())) if len(i) else 0
        keys += min(int(length), covered + int(sinks.max(initial=0)))
    return total, keys


def work(case):
    size = 2 if case["codes"] else 4
    result = size if not case["codes"] or _halves(case) else 4
    if case["kind"] in ("norm_fwd", "norm_bwd", "dropout"):
        rows, cols = case["rows"], case["cols"]
        n = rows * cols
        if case["kind"] == "dropout":
            return {"bytes": n * (size + result), "flops": n}
        if case["kind"] == "norm_fwd":
            z = result * n if case["residual"] or case["p"] else 0
            return {"bytes": n * (size * (2 if case["residual"] else 1) + result) + z + 8 * rows + 8 * cols, "flops": 8 * n}
        return {"bytes": n * (2 * size + result * (2 if case["p"] else 1)) + 8 * rows + 12 * cols, "flops": 14 * n}
    b, h, hk, d = case["batch"], case["heads"], case["kv_heads"], case["dim"]
    pairs, keys = _pairs(case)
    queries = b * case["q_len"] * h
    nbytes = queries * (d * (size + result) + 4) + keys * hk * d * 2 * size
    flops = 4 * d * h * pairs
    if case["kind"] == "attn_step":
        nbytes += queries * d * 2 * result + keys * hk * d * 2 * result      # dO and dQ, dK and dV
        flops += 10 * d * h * pairs
    return {"bytes": nbytes, "flops": flops}


# ---------------------------------------------------------------------------------------------- in 64 bits, from the definitions

def exact(case, seed):
    state = prepare(case, seed)
    e, m, denorm = FORMATS[case["format"]]
    bias = (1 << (e - 1)) - 1

    def value(t):
        """A stored tensor's values in 64 bits: the nearest of k * 2^(max(E, Emin) - m), ties to the even k."""
        if t.dtype == torch.int16:
            c = t.to(torch.int64)
            field, mantissa = (c >> m) & ((1 << e) - 1), (c & ((1 << m) - 1)).double()
            a = torch.where(field == 0, mantissa, mantissa + 2.0 ** m) * power(field.clamp(min=1) - bias - m)
            a = torch.where(field == (1 << e) - 1, torch.where(mantissa == 0, math.inf, math.nan), a)
            return a * torch.where(c < 0, -1.0, 1.0)
        return nearest(t.double())

    def power(n):
        """2^n, exactly, by its bits."""
        return ((n.to(torch.int64) + 1023) << 52).view(torch.float64)

    def nearest(x):
        if (e, m) == (8, 23):
            return x.float().double()
        exponent = ((x.view(torch.int64) >> 52) & 2047) - 1023
        step = power(exponent.clamp(min=1 - bias, max=200) - m)
        r = torch.round(x / step) * step
        r = torch.where(r.abs() >= 2.0 ** (bias + 1), torch.sign(r) * math.inf, r)
        r = torch.where(x.isfinite(), r, x)
        return r if denorm else torch.where(r.abs() < 2.0 ** (1 - bias), 0.0, r)

    def keeps(rows, cols, p):
        blocks = -(-cols // 8)
        seed64, step = (int(v) for v in state["rng"].tolist())
        low = np.uint64(0xFFFFFFFF)
        key = [seed64 & 0xFFFFFFFF, (seed64 >> 32) & 0xFFFFFFFF]
        bits = np.empty((rows * blocks, 8), dtype=np.int32)
        for at in range(0, rows * blocks, 1 << 16):          # as many as a processor's cache holds
            n = np.arange(at, min(at + (1 << 16), rows * blocks), dtype=np.uint64)
            c = [n & low, n >> np.uint64(32), np.full(n.shape, step & 0xFFFFFFFF, np.uint64), np.full(n.shape, SITE, np.uint64)]
            for turn in range(10):
                left, right = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
                k0, k1 = (np.uint64((v + turn * w) & 0xFFFFFFFF) for v, w in zip(key, (0x9E3779B9, 0xBB67AE85)))
                c = [(right >> np.uint64(32)) ^ c[1] ^ k0, right & low, (left >> np.uint64(32)) ^ c[3] ^ k1, left & low]
            for w in range(4):
                bits[at:at + n.size, 2 * w], bits[at:at + n.size, 2 * w + 1] = c[w] & np.uint64(0xFFFF), c[w] >> np.uint64(16)
        least = int(round(p * 65536))
        factor = 65536.0 / (65536 - least)
        return torch.from_numpy((bits.reshape(rows, blocks * 8)[:, :cols] >= least)).cuda(), float(np.float32(factor))

    if case["kind"] in ("norm_fwd", "norm_bwd", "dropout"):
        rows, cols = case["rows"], case["cols"]
        keep, factor = keeps(rows, cols, case["p"]) if case["p"] else (None, 1.0)
        if case["kind"] == "dropout":
            return torch.where(keep, value(state["x"]) * factor, 0.0)
        weight, bias_vector = nearest(state["gamma"].double()), nearest(state["beta"].double())
        if case["kind"] == "norm_fwd":
            z = value(state["x"])
            if keep is not None:
                z = torch.where(keep, z * factor, 0.0)
            if case["residual"]:
                z = z + value(state["residual"])
            z = nearest(z)
            var, mean = torch.var_mean(z, dim=1, correction=0)
            rstd = 1.0 / torch.sqrt(var + EPS)
            y = weight * ((z - mean.unsqueeze(1)) / torch.sqrt(var + EPS).unsqueeze(1)) + bias_vector
            return {"y": y, "z": z if case["p"] or case["residual"] else None, "mean": mean, "rstd": rstd}
        dy, z = value(state["dy"]), value(state["z"])
        mean, rstd = state["mean"].double(), state["rstd"].double()
        xhat = torch.addcmul(torch.zeros_like(z), z - mean.unsqueeze(1), rstd.unsqueeze(1))
        t = dy * weight
        along = (t * xhat).sum(1) / cols
        dz = rstd.unsqueeze(1) * (t - t.sum(1).div(cols).unsqueeze(1) - xhat * along.unsqueeze(1))
        dx = torch.where(keep, dz * factor, 0.0) if keep is not None else None
        return {"dz": dz, "dx": dx, "dgamma": torch.linalg.vecdot(dy, xhat, dim=0), "dbeta": dy.sum(0)}

    b, nq, h, d = state["q"].shape
    nk, group = case["k_len"], h // case["kv_heads"]
    step = case["kind"] == "attn_step"
    o = torch.zeros(b, nq, h, d, dtype=torch.float64, device="cuda")
    lse = torch.full((b, h, nq), -math.inf, dtype=torch.float64, device="cuda")
    dq, dk, dv = torch.zeros_like(o), *(torch.zeros(b, nk, case["kv_heads"], d, dtype=torch.float64, device="cuda") for _ in range(2))
    for i in range(b):
        length, first = int(_lens(case)[i]), int(_positions(case)[i])
        if length == 0:
            continue
        at, key = first + torch.arange(nq, device="cuda").unsqueeze(1), torch.arange(length, device="cuda").unsqueeze(0)
        hidden = key > at if case["causal"] else torch.zeros(nq, length, dtype=torch.bool, device="cuda")
        if case["window"]:
            hidden = hidden | (((at - key).abs() >= case["window"]) & (key >= case["sinks"]))
        for j in range(h):
            q, k, v = value(state["q"][i, :, j]), value(state["k"][i, :length, j // group]), value(state["v"][i, :length, j // group])
            s = torch.mm(q, k.t().contiguous()) / math.sqrt(d)
            s[hidden] = -math.inf
            lse[i, j] = torch.logsumexp(s, 1)
            p = torch.exp(s - lse[i, j].nan_to_num(neginf=0.0).unsqueeze(1))
            o[i, :, j] = torch.mm(p, v)
            if step:
                do = value(state["do"][i, :, j])
                dv[i, :length, j // group] += torch.mm(p.t().contiguous(), do)
                dp = torch.mm(do, v.t().contiguous())
                ds = p * (dp - (p * dp).sum(1, keepdim=True)) / math.sqrt(d)
                dq[i, :, j] = torch.mm(ds, k)
                dk[i, :length, j // group] += torch.mm(ds.t().contiguous(), q)
    return {"o": o, "lse": lse, "dq": dq, "dk": dk, "dv": dv} if step else {"o": o, "lse": lse}
