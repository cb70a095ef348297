"""The 8-bit linear layers of both roles and the clipping of the gradients they give, as cases that can be
timed and compared.

Every case is one pass as a user of the library makes it.  With `own` set, `run` calls the public binding
(paper_2607_22614_amd.dr); otherwise it computes the same with elementary torch operations in 32 bits.

    op         calls                                     stands for
    quantize   dr_quantize                               weights or activations to 8 bits, a scale for each block
    linear     dr_qlinear                                a rollout rank's linear layer on its staged weights
    train      dr_quantize, dr_qmatmul (3 products)      a training rank's linear layer, forward and backward
    clip       dr_grad_clip                              global gradient norm and clipping over many tensors

An 8-bit matrix holds e4m3 codes in rows padded with zeros to a multiple of 128 columns, and one power of two
(e8m0 code) for each block of 1 x 128 or 128 x 128 elements: the smallest one by which the block's largest finite
magnitude is at most 448.  The scales lie as [column blocks / 4][row blocks][4].  A product sums over the 128
columns of a block pair and over the blocks; results in bf16 take the library's fast sums, gradients of
weights in fp32 its exact ones.  Clipping multiplies by min(1, max_norm / (norm + 1e-6)).
"""
import torch

own = False  # set by the caller: the framework's kernels instead of the plain forms

DEVICE = "cuda"
BLOCK = 128


# ------------------------------------------------------------------ the cases
# Shapes: the repository's decoders (tiny: hidden 256, ffn 688; 0.5B: 896, 4864; 8B: 4096, 14336 on 4 ranks; 32B:
# 5120, 27648 on 8 ranks) and ragged ones of the same ranges.
def _quantize(name, rows, cols, dtype, block_rows, both):
    return {"name": name, "op": "quantize", "rows": rows, "cols": cols, "dtype": dtype, "block_rows": block_rows,
            "both": both}


def _linear(name, m, n, k):
    return {"name": name, "op": "linear", "m": m, "n": n, "k": k}


def _train(name, m, n, k, accumulate):
    return {"name": name, "op": "train", "m": m, "n": n, "k": k, "accumulate": accumulate}


def _clip(name, layers, hidden, kv, ffn, vocab, cut, dtype, sigma):
    return {"name": name, "op": "clip", "layers": layers, "hidden": hidden, "kv": kv, "ffn": ffn, "vocab": vocab,
            "cut": cut, "dtype": dtype, "sigma": sigma}


def listed():
    return [
        # activations of a short odd batch of the tiny decoder's feed-forward: 344 columns are 2.7 blocks
        _quantize("quantize_ragged", 333, 344, "bf16", 1, False),
        # the fused gate/up weights of one 8B rollout rank after staging, square blocks
        _quantize("quantize_weights_8b", 7168, 4096, "bf16", 128, False),
        # the gradient of an 8B layer's output in training: along its rows and, for the weights' gradient, its columns
        _quantize("quantize_both_ways_8b", 8192, 4096, "bf16", 1, True),
        # decoding one token: the 8B down projection of one rank, all latency and weight bytes
        _linear("linear_one_token_8b", 1, 4096, 3584),
        # decoding a small batch: the 32B gate/up projection of one rank
        _linear("linear_16_tokens_32b", 16, 6912, 5120),
        # a decoding batch that is no multiple of anything on the 0.5B model's output matrix (all 151936 words)
        _linear("linear_61_tokens_vocab", 61, 151936, 896),
        # a prompt of ordinary length through the 0.5B gate/up projection
        _linear("linear_prompt_half_b", 777, 9728, 896),
        # a long prompt through the 32B gate/up projection of one rank
        _linear("linear_prompt_32b", 8192, 6912, 5120),
        # the tiny decoder's feed-forward in training, gradients accumulated over micro-batches
        _train("train_tiny", 200, 688, 256, True),
        # an 8B gate projection in training, a batch of 8192 tokens
        _train("train_8b", 8192, 14336, 4096, False),
        # the gradients of the tiny decoder, tensor by tensor, to its flat fp32 buffer
        _clip("clip_tiny_tensors", 2, 256, 256, 688, 2048, 0, "mixed", 0.02),
        # the gradients of the 0.5B decoder in its 8 flat shards
        _clip("clip_half_b_shards", 24, 896, 128, 4864, 151936, 8, "f32", 1e-3),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    op = rng.choice(["quantize", "linear", "linear", "linear", "train", "train", "clip"])
    if op == "quantize":
        rows, cols = _log(rng, 1, 16384), _log(rng, 64, 16384)
        c = _quantize("", min(rows, (1 << 27) // cols), cols, rng.choice(["bf16", "f32"]), rng.choice([1, 128]),
                      rng.random() < 0.5)
    elif op == "linear":
        m, n, k = _log(rng, 1, 8192), _log(rng, 96, 151936), 8 * _log(rng, 12, 3456)
        c = _linear("", min(m, max(1, (1 << 38) // (n * k))), n, k)
    elif op == "train":
        m, n, k = _log(rng, 16, 8192), 4 * _log(rng, 24, 6912), 4 * _log(rng, 24, 2048)
        c = _train("", min(m, max(16, (1 << 38) // (n * k))), n, k, rng.random() < 0.5)
    else:
        hidden, layers = _log(rng, 64, 2048), _log(rng, 1, 24)
        c = _clip("", layers, hidden, max(1, hidden // 4), int(2.7 * hidden), 8 * hidden, rng.choice([0, 0, 1, 5, 8]),
                  rng.choice(["f32", "bf16", "mixed"]), rng.choice([1e-5, 1e-3, 0.02]))
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


def _tensors(c):
    """Elements of each gradient, in model order; cut: of each flat shard."""
    h, kv, f = c["hidden"], c["kv"], c["ffn"]
    layer = [h, h * h, kv * h, kv * h, h * h, h, f * h, f * h, h * f]
    sizes = [c["vocab"] * h] + layer * c["layers"] + [h, c["vocab"] * h]
    if c["cut"]:
        per = _up(sum(sizes), 256 * c["cut"]) // c["cut"]
        return [per] * c["cut"]
    return sizes


def _grad_types(c):
    kinds = {"f32": [torch.float32], "bf16": [torch.bfloat16], "mixed": [torch.float32, torch.bfloat16]}[c["dtype"]]
    return [kinds[i % len(kinds)] for i in range(len(_tensors(c)))]


def _inputs(c, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    if c["op"] == "quantize":
        src = _activations(gen, c["rows"], c["cols"])
        return {"src": src.to(torch.bfloat16 if c["dtype"] == "bf16" else torch.float32)}
    if c["op"] == "clip":
        return {"grads": [_normal(gen, (n,), c["sigma"]).to(t) for n, t in zip(_tensors(c), _grad_types(c))]}
    s = {"x": _activations(gen, c["m"], c["k"]).to(torch.bfloat16),
         "weight": _normal(gen, (c["n"], c["k"]), 0.02).to(torch.bfloat16)}
    if c["op"] == "train":
        s["dy"] = _activations(gen, c["m"], c["n"], 1e-4).to(torch.bfloat16)
        s["dw"] = _normal(gen, (c["n"], c["k"]), 1e-3) if c["accumulate"] else torch.zeros((c["n"], c["k"]), device=DEVICE)
    return s


def _out(shape, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device=DEVICE)


def prepare(case, seed):
    """The inputs; for a linear layer the weights in 8 bits, laid out once as a program that keeps them does; and
    the buffers that the outputs go to."""
    s = dict(_inputs(case, seed), case=case)
    if case["op"] in ("linear", "train"):
        m, n, k = case["m"], case["n"], case["k"]
        weight = s.pop("weight")
        s["w"] = quantize_plain(weight, 128)
        s["y"] = _out((m, n))
        if case["op"] == "train":
            s["wt"] = quantize_plain(weight.t(), 128)  # square blocks: the same codes, transposed
            s["dx"] = _out((m, k))
    elif case["op"] == "clip":
        sizes = _tensors(case)
        s["flat"] = _out((sum(sizes),), torch.float32)
        s["outs"] = list(torch.split(s["flat"], sizes))
        s["norm"] = _out((1,), torch.float32)
    if own:
        _handles(s, case)
    return s


def _handles(s, case):
    """The 8-bit buffers, workspaces and lists that a program keeps beside its tensors."""
    from paper_2607_22614_amd import dr

    s["dr"] = dr
    if case["op"] == "quantize":
        rows, cols, br = case["rows"], case["cols"], case["block_rows"]
        s["q"] = dr.QMatrix.empty(rows, cols, br)
        s["qt"] = dr.QMatrix.empty(cols, rows, br) if case["both"] else None
    elif case["op"] == "clip":
        s["list"] = dr.GradList(s["grads"], s["outs"])
        s["workspace"] = _out((dr.dr_grad_workspace(),), torch.uint8)
    else:
        m, n, k = case["m"], case["n"], case["k"]
        s["w"] = dr.QMatrix(*(t.view(torch.uint8) for t in s["w"]), n, k, 128)
        if case["op"] == "linear":
            s["workspace"] = _out((dr.dr_qlinear_workspace(m, s["w"]),), torch.uint8)
        else:
            s["wt"] = dr.QMatrix(*(t.view(torch.uint8) for t in s["wt"]), k, n, 128)
            s["xq"], s["xt"] = dr.QMatrix.empty(m, k, 1), dr.QMatrix.empty(k, m, 1)
            s["dyq"], s["dyt"] = dr.QMatrix.empty(m, n, 1), dr.QMatrix.empty(n, m, 1)
            need = max(dr.dr_qmatmul_workspace(*p) for p in ((m, n, k), (m, k, n), (n, k, m)))
            s["workspace"] = _out((need,), torch.uint8)


# ------------------------------------------------------------------ the plain forms
def _blocks(x, block_rows):
    """x in 32 bits, padded with zeros to whole blocks: [row blocks, block_rows, column blocks, 128]."""
    rows, cols = x.shape
    p = torch.zeros((_up(rows, block_rows), _up(cols, BLOCK)), dtype=torch.float32, device=x.device)
    p[:rows, :cols] = x
    return p.view(-1, block_rows, p.shape[1] // BLOCK, BLOCK)


def _power_of_two(code):
    """2^(code - 127) of e8m0 codes, from its bits: a library's exp2 need not be exact."""
    code = code.to(torch.int32)
    return torch.where(code == 0, 0x400000, code << 23).view(torch.float32)


def quantize_plain(x, block_rows):
    """(e4m3 codes [rows, padded columns], e8m0 scales [column blocks / 4, row blocks, 4])."""
    b = _blocks(x, block_rows)
    amax = torch.where(torch.isfinite(b), b.abs(), 0.0).amax(dim=(1, 3))
    # biased exponent of the smallest power of two that takes amax to 448 = 1.75 * 2^8 or below
    code = (((amax.view(torch.int32) + 0x1FFFFF) >> 23) - 8).clamp(min=0)
    code = torch.where(amax == 0, 127, code)
    inverse = _power_of_two(254 - code)
    q = (b * inverse[:, None, :, None]).to(torch.float8_e4m3fn).view(b.shape[0] * block_rows, -1)[:x.shape[0]]
    scales = torch.full((_up(b.shape[2], 4), b.shape[0]), 127, dtype=torch.uint8, device=x.device)
    scales[:b.shape[2]] = code.t().to(torch.uint8)
    scales = scales.view(-1, 4, b.shape[0]).permute(0, 2, 1).contiguous()
    return q.contiguous(), scales.view(torch.float8_e8m0fnu)


def _values(q, scales, cols, block_rows):
    """What codes and scales stand for, in 32 bits: [rows, cols]."""
    rows, padded = q.shape
    per = _power_of_two(scales.view(torch.uint8).permute(0, 2, 1).reshape(-1, scales.shape[1]).t())
    per = per[:, :padded // BLOCK].repeat_interleave(block_rows, dim=0)[:rows].repeat_interleave(BLOCK, dim=1)
    return (q.to(torch.float32) * per)[:, :cols]


def _plain_quantize(s, case):
    out = list(quantize_plain(s["src"], case["block_rows"]))
    return out + list(quantize_plain(s["src"].t(), case["block_rows"])) if case["both"] else out


def _plain_linear(s, case):
    x = _values(*quantize_plain(s["x"], 1), case["k"], 1)
    s["y"].copy_(x @ _values(*s["w"], case["k"], 128).t())
    return s["y"]


def _plain_train(s, case):
    m, n, k = case["m"], case["n"], case["k"]
    x, xt = _values(*quantize_plain(s["x"], 1), k, 1), _values(*quantize_plain(s["x"].t(), 1), m, 1)
    dy, dyt = _values(*quantize_plain(s["dy"], 1), n, 1), _values(*quantize_plain(s["dy"].t(), 1), m, 1)
    s["y"].copy_(x @ _values(*s["w"], k, 128).t())
    s["dx"].copy_(dy @ _values(*s["wt"], n, 128).t())
    dw = dyt @ xt.t()
    s["dw"].copy_(s["dw"] + dw if case["accumulate"] else dw)
    return {"y": s["y"], "dx": s["dx"], "dw": s["dw"]}


def _plain_clip(s, case):
    squares = torch.stack([g.to(torch.float32).square().sum() for g in s["grads"]])
    s["norm"][0] = squares.sum().sqrt()
    factor = (1.0 / (s["norm"] + 1e-6)).clamp(max=1.0)
    for g, o in zip(s["grads"], s["outs"]):
        o.copy_(g.to(torch.float32) * factor)
    return {"norm": s["norm"], "flat": s["flat"]}


# ------------------------------------------------------------------ the framework's calls
def _codes(q):
    return [q.data.view(torch.float8_e4m3fn), q.scales.view(torch.float8_e8m0fnu)]


def _own_quantize(s, case):
    s["dr"].dr_quantize(s["src"], s["q"], s["qt"])
    return _codes(s["q"]) + (_codes(s["qt"]) if case["both"] else [])


def _own_linear(s, case):
    s["dr"].dr_qlinear(s["x"], s["w"], s["y"], fast=True, workspace=s["workspace"])
    return s["y"]


def _own_train(s, case):
    dr, ws = s["dr"], s["workspace"]
    dr.dr_quantize(s["x"], s["xq"], s["xt"])
    dr.dr_qmatmul(s["xq"], s["w"], s["y"], fast=True, workspace=ws)
    dr.dr_quantize(s["dy"], s["dyq"], s["dyt"])
    dr.dr_qmatmul(s["dyq"], s["wt"], s["dx"], fast=True, workspace=ws)
    dr.dr_qmatmul(s["dyt"], s["xt"], s["dw"], accumulate=case["accumulate"], workspace=ws)
    return {"y": s["y"], "dx": s["dx"], "dw": s["dw"]}


def _own_clip(s, case):
    s["dr"].dr_grad_clip(s["list"], 1.0, s["norm"], s["workspace"])
    return {"norm": s["norm"], "flat": s["flat"]}


_RUN = {False: {"quantize": _plain_quantize, "linear": _plain_linear, "train": _plain_train, "clip": _plain_clip},
        True: {"quantize": _own_quantize, "linear": _own_linear, "train": _own_train, "clip": _own_clip}}


def run(state):
    return _RUN[own][state["case"]["op"]](state, state["case"])


# ------------------------------------------------------------------ what a pass cannot do without
def _matrix_bytes(rows, cols, block_rows):
    return rows * cols + _up(rows, block_rows) // block_rows * (_up(cols, BLOCK) // BLOCK)


def work(case):
    if case["op"] == "quantize":
        rows, cols, br = case["rows"], case["cols"], case["block_rows"]
        out = _matrix_bytes(rows, cols, br) + (_matrix_bytes(cols, rows, br) if case["both"] else 0)
        return {"bytes": rows * cols * (2 if case["dtype"] == "bf16" else 4) + out, "flops": 2 * rows * cols}
    if case["op"] == "clip":
        read = sum(n * t.itemsize for n, t in zip(_tensors(case), _grad_types(case)))
        total = sum(_tensors(case))
        return {"bytes": read + 4 * total, "flops": 3 * total}
    m, n, k = case["m"], case["n"], case["k"]
    if case["op"] == "linear":
        return {"bytes": 2 * m * k + _matrix_bytes(n, k, 128) + 2 * m * n, "flops": 2 * m * n * k}
    moved = 2 * m * k + 2 * m * n + 2 * _matrix_bytes(n, k, 128)        # x, dy and the weights both ways
    moved += 2 * m * n + 2 * m * k + (8 if case["accumulate"] else 4) * n * k  # y, dx, dw
    return {"bytes": moved, "flops": 6 * m * n * k}


# ------------------------------------------------------------------ the definition in 64 bits
def _two_to_the(e):
    """2^e in 64 bits, from its bits."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _round_e4m3(v):
    """v to 4 significant bits (steps of 2^-9 below 2^-6), ties to even."""
    _, e = torch.frexp(v)
    step = _two_to_the(e.clamp(min=-5) - 4)
    return torch.round(v / step) * step


def _exact_codes(x, block_rows):
    """Codes' values [rows, padded columns], scales [row blocks, column blocks], from the definition."""
    rows, cols = x.shape
    p = torch.nn.functional.pad(x.to(torch.float64), (0, -cols % BLOCK, 0, -rows % block_rows))
    amax = p.abs().unflatten(1, (-1, BLOCK)).unflatten(0, (-1, block_rows)).amax(dim=(1, 3))
    mantissa, e = torch.frexp(amax / 448.0)
    e = torch.where(mantissa == 0.5, e - 1, e).clamp(min=-127)
    scale = torch.where(amax == 0, 1.0, _two_to_the(e))
    full = scale.repeat_interleave(block_rows, 0).repeat_interleave(BLOCK, 1)
    return _round_e4m3(p / full)[:rows], scale, full[:rows]


def _exact_values(x, block_rows):
    codes, _, full = _exact_codes(x, block_rows)
    return (codes * full)[:, :x.shape[1]]


def _exact_quantize(x, block_rows):
    codes, scale, _ = _exact_codes(x, block_rows)
    kb = scale.shape[1]
    laid = torch.nn.functional.pad(scale, (0, -kb % 4), value=1.0).unflatten(1, (-1, 4)).transpose(0, 1)
    return [codes, laid.contiguous()]


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "quantize":
        out = _exact_quantize(s["src"], case["block_rows"])
        return out + (_exact_quantize(s["src"].t(), case["block_rows"]) if case["both"] else [])
    if case["op"] == "clip":
        norm = torch.sqrt(sum((g.to(torch.float64) ** 2).sum() for g in s["grads"]))
        factor = torch.clamp(1.0 / (norm + 1e-6), max=1.0)
        return {"norm": norm.reshape(1), "flat": torch.cat([g.to(torch.float64) * factor for g in s["grads"]])}
    w = _exact_values(s["weight"], 128)
    y = torch.matmul(_exact_values(s["x"], 1), w.t())
    if case["op"] == "linear":
        return y
    dx = torch.matmul(_exact_values(s["dy"], 1), w)
    dw = torch.matmul(_exact_values(s["dy"].t(), 1), _exact_values(s["x"].t(), 1).t())
    return {"y": y, "dx": dx, "dw": s["dw"].to(torch.float64) + dw if case["accumulate"] else dw}
