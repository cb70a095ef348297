"""The gated feed-forward block of both roles in 8 bits and its activation checkpoints, as cases that can be timed and
compared.

Every case is one pass as a user of the library makes it.  With `own` set, `run` calls the public binding
(paper_2607_22614_amd.dr); otherwise it computes the same with elementary torch operations in 32 bits.

    op         calls               stands for
    gated      dr_qgated           a rollout rank's gate and up projections, activation and product, on staged weights
    save       dr_qgated_save      the same in training: the block's inner activations and its checkpoint in 8 bits
    backward   dr_gated_backward   the gradients of gate and up, both ways, from the 8-bit checkpoint, and the inner
                                   activations again for the down projection's gradient
    transpose  dr_qtranspose       an 8-bit activation checkpoint, turned for the gradient of the weights it met

With x [M, K] and the fused weights w [2F, K], gate and up are the halves of x w^T and h = act(gate) * up, where
act(g) = g / (1 + exp(-z)), z = k1 g + k3 g^3: silu has k1 = 1 and k3 = 0, the tanh form of gelu k1 = 2 sqrt(2/pi)
and k3 = 0.044715 k1.

An 8-bit matrix holds e4m3 codes in rows padded with zeros to a multiple of 128 columns, and one power of two
(e8m0 code) for each block of 1 x 128 (activations, gradients) or 128 x 128 (weights) elements: the smallest one by
which the block's largest finite magnitude is at most 448.  The scales lie as [column blocks / 4][row blocks][4].
Results in bf16 and in 8 bits take the library's fast sums, results in fp32 its exact ones.
"""
import math

import torch

own = False  # set by the caller: the framework's kernels instead of the plain forms

DEVICE = "cuda"
BLOCK = 128
ACTS = {"silu": (1.0, 0.0), "gelu": (2.0 * math.sqrt(2.0 / math.pi), 0.08943 * math.sqrt(2.0 / math.pi))}
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------ the cases
# Shapes: the repository's decoders (tiny: hidden 256, ffn 688; 0.5B: 896, 4864; 8B: 4096, 14336 on 4 ranks; 32B:
# 5120, 27648 on 8 ranks) and ragged ones of the same ranges.
def _gated(name, m, f, k, act, dtype, out):
    return {"name": name, "op": "gated", "m": m, "f": f, "k": k, "act": act, "dtype": dtype, "out": out}


def _save(name, m, f, k, act):
    return {"name": name, "op": "save", "m": m, "f": f, "k": k, "act": act}


def _backward(name, m, f, act, dtype, again):
    return {"name": name, "op": "backward", "m": m, "f": f, "act": act, "dtype": dtype, "again": again}


def _transpose(name, rows, cols):
    return {"name": name, "op": "transpose", "rows": rows, "cols": cols}


def listed():
    return [
        # decoding one token: the 8B feed-forward of one rank, all latency and weight bytes
        _gated("gated_one_token_8b", 1, 3584, 4096, "silu", "bf16", "bf16"),
        # decoding a small batch: the 32B feed-forward of one rank
        _gated("gated_16_tokens_32b", 16, 3456, 5120, "silu", "bf16", "bf16"),
        # a decoding batch that is no multiple of anything on the 0.5B model
        _gated("gated_61_tokens_half_b", 61, 4864, 896, "silu", "bf16", "bf16"),
        # a short prompt through one of two ranks of the tiny decoder, kept in fp32: 344 columns are 2.7 blocks
        _gated("gated_ragged_tiny", 333, 344, 256, "gelu", "f32", "f32"),
        # a long prompt through the 32B feed-forward of one rank
        _gated("gated_prompt_32b", 8192, 3456, 5120, "silu", "bf16", "bf16"),
        # the tiny decoder in training, a short batch
        _save("save_tiny", 200, 688, 256, "gelu"),
        # an 8B layer in training, 8192 tokens
        _save("save_8b", 8192, 14336, 4096, "silu"),
        # the gradients of the tiny decoder's short batch
        _backward("backward_tiny", 200, 688, "gelu", "bf16", True),
        # an odd number of columns, so that up's begin inside gate's last block; the inner activations were kept
        _backward("backward_odd", 1001, 1377, "silu", "f32", False),
        # the gradients of an 8B layer, 8192 tokens
        _backward("backward_8b", 8192, 14336, "silu", "bf16", True),
        # the input of the tiny decoder's down projection on one of two ranks
        _transpose("transpose_ragged", 333, 344),
        # the input of an 8B layer, 8192 tokens
        _transpose("transpose_8b", 8192, 4096),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    op, act = rng.choice(["gated", "gated", "gated", "save", "save", "backward", "backward", "transpose"]), rng.choice(["silu", "gelu"])
    if op == "gated":
        m, f, k = _log(rng, 1, 8192), _log(rng, 48, 27648), 8 * _log(rng, 12, 3456)
        dtype = rng.choice(["bf16", "bf16", "f32"])
        c = _gated("", min(m, max(1, (1 << 37) // (f * k))), f, k, act, dtype, rng.choice(["bf16", dtype]))
    elif op == "save":
        m, f, k = _log(rng, 16, 8192), _log(rng, 48, 14336), 8 * _log(rng, 12, 1024)
        c = _save("", min(m, max(16, (1 << 38) // (f * k))), f, k, act)
    elif op == "backward":
        m, f = _log(rng, 1, 16384), _log(rng, 48, 14336)
        c = _backward("", min(m, (1 << 26) // f), f, act, rng.choice(["bf16", "f32"]), rng.random() < 0.5)
    else:
        rows, cols = _log(rng, 1, 16384), _log(rng, 64, 16384)
        c = _transpose("", min(rows, (1 << 25) // cols), cols)
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs
def _up(n, to):
    return -(-n // to) * to


def _normal(gen, shape, scale):
    return torch.randn(shape, generator=gen, device=DEVICE, dtype=torch.float32) * scale


def _activations(gen, rows, cols, scale=1.0):
    """Normal values with rows of different size and a few columns that stand out, as activations have them."""
    x = _normal(gen, (rows, cols), scale)
    x *= torch.exp2(torch.randn((rows, 1), generator=gen, device=DEVICE))
    x[:, torch.randint(cols, (max(1, cols // 256),), generator=gen, device=DEVICE)] *= 24.0
    return x


def _inputs(c, seed):
    """What a program has from the steps before, 8-bit matrices as (codes, scales)."""
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    if c["op"] == "transpose":
        return {"src": quantize_plain(_activations(gen, c["rows"], c["cols"]), 1)}
    if c["op"] == "backward":
        s = {"dh": _activations(gen, c["m"], c["f"], 1e-4).to(TYPES[c["dtype"]])}
        for name in ("gate", "up"):
            s[name] = quantize_plain(_activations(gen, c["m"], c["f"]), 1)
        return s
    x = _activations(gen, c["m"], c["k"])
    weights = _normal(gen, (2 * c["f"], c["k"]), c["k"] ** -0.5)
    return {"x": x.to(TYPES[c["dtype"]]) if c["op"] == "gated" else quantize_plain(x, 1), "w": quantize_plain(weights, 128)}


def prepare(case, seed):
    """The inputs, and the buffers that the outputs go to; a linear layer's weights are in 8 bits, laid out once as a
    program that keeps them does."""
    s = dict(_inputs(case, seed), case=case)
    if case["op"] == "gated":
        s["h"] = torch.empty((case["m"], case["f"]), dtype=TYPES[case["out"]], device=DEVICE)
    if own:
        _handles(s, case)
    return s


def _handles(s, case):
    """The 8-bit matrices, workspaces and options that a program keeps beside its tensors."""
    from paper_2607_22614_amd import dr

    def matrix(pair, rows, cols, block_rows=1):
        return dr.QMatrix(*(t.view(torch.uint8) for t in pair), rows, cols, block_rows)

    s["dr"] = dr
    if case["op"] == "transpose":
        rows, cols = case["rows"], case["cols"]
        s["src"], s["qt"] = matrix(s["src"], rows, cols), dr.QMatrix.empty(cols, rows, 1)
        return
    m, f = case["m"], case["f"]
    s["act"] = dr.DR_ACT_SILU if case["act"] == "silu" else dr.DR_ACT_GELU_TANH
    if case["op"] == "backward":
        s["gate"], s["up"] = matrix(s["gate"], m, f), matrix(s["up"], m, f)
        s["d"], s["dt"] = dr.QMatrix.empty(m, 2 * f, 1), dr.QMatrix.empty(2 * f, m, 1)
        s["ht"] = dr.QMatrix.empty(f, m, 1) if case["again"] else None
        return
    k = case["k"]
    s["w"] = matrix(s["w"], 2 * f, k, 128)
    if case["op"] == "gated":
        need = dr.dr_qgated_workspace(m, s["w"])
    else:
        s["x"] = matrix(s["x"], m, k)
        s["h"], s["gate"], s["up"] = (dr.QMatrix.empty(m, f, 1) for _ in range(3))
        need = dr.dr_qgated_save_workspace(m, s["w"])
    s["workspace"] = torch.empty((need,), dtype=torch.uint8, device=DEVICE)


# ------------------------------------------------------------------ the plain forms
def _power_of_two(code):
    """2^(code - 127) of e8m0 codes, from its bits: a library's exp2 need not be exact."""
    code = code.to(torch.int32)
    return torch.where(code == 0, 0x400000, code << 23).view(torch.float32)


def quantize_plain(x, block_rows):
    """(e4m3 codes [rows, padded columns], e8m0 scales [column blocks / 4, row blocks, 4])."""
    rows, cols = x.shape
    p = torch.zeros((_up(rows, block_rows), _up(cols, BLOCK)), dtype=torch.float32, device=x.device)
    p[:rows, :cols] = x
    b = p.view(-1, block_rows, p.shape[1] // BLOCK, BLOCK)
    amax = torch.where(torch.isfinite(b), b.abs(), 0.0).amax(dim=(1, 3))
    # biased exponent of the smallest power of two that takes amax to 448 = 1.75 * 2^8 or below
    code = (((amax.view(torch.int32) + 0x1FFFFF) >> 23) - 8).clamp(min=0)
    code = torch.where(amax == 0, 127, code)
    inverse = _power_of_two(254 - code)
    q = (b * inverse[:, None, :, None]).to(torch.float8_e4m3fn).view(b.shape[0] * block_rows, -1)[:rows]
    scales = torch.full((_up(b.shape[2], 4), b.shape[0]), 127, dtype=torch.uint8, device=x.device)
    scales[:b.shape[2]] = code.t().to(torch.uint8)
    scales = scales.view(-1, 4, b.shape[0]).permute(0, 2, 1).contiguous()
    return [q.contiguous(), scales.view(torch.float8_e8m0fnu)]


def _values(pair, cols, block_rows):
    """What codes and scales stand for, in 32 bits: [rows, cols]."""
    q, scales = pair
    rows, padded = q.shape
    per = _power_of_two(scales.view(torch.uint8).permute(0, 2, 1).reshape(-1, scales.shape[1]).t())
    per = per[:, :padded // BLOCK].repeat_interleave(block_rows, dim=0)[:rows].repeat_interleave(BLOCK, dim=1)
    return (q.to(torch.float32) * per)[:, :cols]


def _sigmoid(g, act):
    k1, k3 = ACTS[act]
    return 1.0 / (1.0 + torch.exp(-(k1 * g + k3 * g * g * g)))


def _halves(x, s, case):
    y = x @ _values(s["w"], case["k"], 128).t()
    return y[:, :case["f"]], y[:, case["f"]:]


def _plain_gated(s, case):
    gate, up = _halves(_values(quantize_plain(s["x"], 1), case["k"], 1), s, case)
    s["h"].copy_(gate * _sigmoid(gate, case["act"]) * up)
    return s["h"]


def _plain_save(s, case):
    gate, up = _halves(_values(s["x"], case["k"], 1), s, case)
    return {"h": quantize_plain(gate * _sigmoid(gate, case["act"]) * up, 1), "gate": quantize_plain(gate, 1), "up": quantize_plain(up, 1)}


def _plain_backward(s, case):
    gate, up, dh = _values(s["gate"], case["f"], 1), _values(s["up"], case["f"], 1), s["dh"].to(torch.float32)
    k1, k3 = ACTS[case["act"]]
    sig = _sigmoid(gate, case["act"])
    dgate = dh * up * (sig + gate * sig * (1.0 - sig) * (k1 + 3.0 * k3 * gate * gate))
    d = torch.cat([dgate, dh * gate * sig], dim=1)
    out = {"d": quantize_plain(d, 1), "dt": quantize_plain(d.t(), 1)}
    return dict(out, ht=quantize_plain((gate * sig * up).t(), 1)) if case["again"] else out


def _plain_transpose(s, case):
    return quantize_plain(_values(s["src"], case["cols"], 1).t(), 1)


# ------------------------------------------------------------------ the framework's calls
def _codes(q):
    return [q.data.view(torch.float8_e4m3fn), q.scales.view(torch.float8_e8m0fnu)]


def _own_gated(s, case):
    s["dr"].dr_qgated(s["x"], s["w"], s["h"], act=s["act"], fast=case["out"] == "bf16", workspace=s["workspace"])
    return s["h"]


def _own_save(s, case):
    s["dr"].dr_qgated_save(s["x"], s["w"], s["h"], s["gate"], s["up"], act=s["act"], fast=True, workspace=s["workspace"])
    return {name: _codes(s[name]) for name in ("h", "gate", "up")}


def _own_backward(s, case):
    s["dr"].dr_gated_backward(s["dh"], s["gate"], s["up"], s["d"], s["dt"], s["ht"], act=s["act"])
    return {name: _codes(s[name]) for name in ("d", "dt", "ht") if s[name] is not None}


def _own_transpose(s, case):
    s["dr"].dr_qtranspose(s["src"], s["qt"])
    return _codes(s["qt"])


_RUN = {False: {"gated": _plain_gated, "save": _plain_save, "backward": _plain_backward, "transpose": _plain_transpose},
        True: {"gated": _own_gated, "save": _own_save, "backward": _own_backward, "transpose": _own_transpose}}


def run(state):
    return _RUN[own][state["case"]["op"]](state, state["case"])


# ------------------------------------------------------------------ what a pass cannot do without
def _matrix_bytes(rows, cols, block_rows=1):
    return rows * cols + _up(rows, block_rows) // block_rows * (_up(cols, BLOCK) // BLOCK)


def work(case):
    if case["op"] == "transpose":
        rows, cols = case["rows"], case["cols"]
        return {"bytes": _matrix_bytes(rows, cols) + _matrix_bytes(cols, rows), "flops": rows * cols}
    m, f = case["m"], case["f"]
    if case["op"] == "backward":
        moved = m * f * TYPES[case["dtype"]].itemsize + 2 * _matrix_bytes(m, f) + _matrix_bytes(m, 2 * f) + _matrix_bytes(2 * f, m)
        return {"bytes": moved + (_matrix_bytes(f, m) if case["again"] else 0), "flops": 20 * m * f}
    k = case["k"]
    weights = _matrix_bytes(2 * f, k, 128)
    if case["op"] == "gated":
        moved = m * k * TYPES[case["dtype"]].itemsize + weights + m * f * TYPES[case["out"]].itemsize
    else:
        moved = _matrix_bytes(m, k) + weights + 3 * _matrix_bytes(m, f)
    return {"bytes": moved, "flops": 4 * m * f * k + 8 * m * f}


# ------------------------------------------------------------------ the definition in 64 bits
def _two_to_the(e):
    """2^e in 64 bits, from its bits."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _meant(pair, cols, block_rows):
    """The numbers of an 8-bit matrix, in 64 bits."""
    codes, scales = pair
    words, lines, _ = scales.shape
    per = _two_to_the(scales.view(torch.uint8).to(torch.int64) - 127)
    row = torch.arange(codes.shape[0], device=codes.device) // block_rows
    col = torch.arange(cols, device=codes.device) // BLOCK
    return codes[:, :cols].to(torch.float64) * per[(col // 4)[None, :], row[:, None], (col % 4)[None, :]]


def _round_e4m3(v):
    """v to 4 significant bits (steps of 2^-9 below 2^-6), ties to even."""
    _, e = torch.frexp(v)
    step = _two_to_the(e.clamp(min=-5) - 4)
    return torch.round(v / step) * step


def _exact_quantize(x):
    """[codes' values, scales] of blocks of 1 x 128, from the definition."""
    p = torch.nn.functional.pad(x, (0, -x.shape[1] % BLOCK)).unflatten(1, (-1, BLOCK))
    amax = p.abs().amax(dim=2)
    mantissa, e = torch.frexp(amax / 448.0)
    e = torch.where(mantissa == 0.5, e - 1, e).clamp(min=-127)
    scale = torch.where(amax == 0, 1.0, _two_to_the(e))
    laid = torch.nn.functional.pad(scale, (0, -scale.shape[1] % 4), value=1.0).unflatten(1, (-1, 4)).transpose(0, 1)
    return [_round_e4m3(p / scale[:, :, None]).flatten(1), laid.contiguous()]


def _exact_act(g, act):
    """(act(g), its derivative)."""
    if act == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1.0 + g * (1.0 - s))
    c = math.sqrt(2.0 / math.pi)
    t = torch.tanh(c * (g + 0.044715 * g ** 3))
    return 0.5 * g * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * g * (1.0 - t * t) * c * (1.0 + 0.134145 * g * g)


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "transpose":
        return _exact_quantize(_meant(s["src"], case["cols"], 1).t().contiguous())
    if case["op"] == "backward":
        gate, up, dh = _meant(s["gate"], case["f"], 1), _meant(s["up"], case["f"], 1), s["dh"].to(torch.float64)
        a, slope = _exact_act(gate, case["act"])
        d = torch.cat([dh * up * slope, dh * a], dim=1)
        out = {"d": _exact_quantize(d), "dt": _exact_quantize(d.t().contiguous())}
        return dict(out, ht=_exact_quantize((a * up).t().contiguous())) if case["again"] else out
    if case["op"] == "gated":
        codes, laid = _exact_quantize(s["x"].to(torch.float64))
        per = laid.transpose(0, 1).flatten(1)[:, :codes.shape[1] // BLOCK].repeat_interleave(BLOCK, dim=1)
        x = (codes * per)[:, :case["k"]]
    else:
        x = _meant(s["x"], case["k"], 1)
    y = torch.matmul(x, _meant(s["w"], case["k"], 128).t())
    gate, up = y[:, :case["f"]], y[:, case["f"]:]
    h = _exact_act(gate, case["act"])[0] * up
    return h if case["op"] == "gated" else {name: _exact_quantize(v) for name, v in (("h", h), ("gate", gate), ("up", up))}
