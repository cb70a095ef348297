"""Both roles of a GPU with 8-bit linear layers: rollout on staged weights, training, and the switch in between.

    python examples/eight_bit_roles.py [--workload tiny|0.5b|8b] [--layers 1] [--tokens 200] [--steps 3]

The decoder's flat fp32 training shards are staged to the rollout ranks' bf16 weights (dr_stage_all); every rank's last down
projection and output matrix become 8-bit matrices (dr_quantize), and a prompt and then a single token run through
them (dr_qlinear).  The training role runs the same two layers forward and backward in 8 bits over two micro-batches
(dr_quantize along rows and columns, three dr_qmatmul a layer, the weights' gradients added up in a flat fp32
buffer of the training layout), clips the shards of that buffer to a global norm (dr_grad_clip) and takes a gradient step;
then the weights are staged again.  The targets stay the same, so that the losses of both roles fall together.

    down:  h = r + a Wd^T        (r, the residual, and a, the activations, are random inputs)
    head:  logits = h Wl^T       loss = mean cross entropy of the targets
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2607_22614_amd import datagen, dr, workloads  # noqa: E402

MICRO_BATCHES = 2


class TrainedLinear:
    """y = x W^T in 8 bits, forward and backward, over views of the flat weights and of the flat gradients."""

    def __init__(self, weight, grad, tokens: int):
        n, k = weight.shape
        self.weight, self.grad = weight, grad
        self.w, self.wt = dr.QMatrix.empty(n, k, 128), dr.QMatrix.empty(k, n, 128)
        self.xq, self.xt = dr.QMatrix.empty(tokens, k), dr.QMatrix.empty(k, tokens)
        self.dyq, self.dyt = dr.QMatrix.empty(tokens, n), dr.QMatrix.empty(n, tokens)
        need = max(dr.dr_qmatmul_workspace(*s) for s in ((tokens, n, k), (tokens, k, n), (n, k, tokens)))
        self.workspace = torch.empty(need, dtype=torch.uint8, device=weight.device)

    def take_weights(self):
        """Once a step: square blocks give W and its transpose the same codes."""
        dr.dr_quantize(self.weight, self.w, self.wt)

    def forward(self, x, y):
        dr.dr_quantize(x, self.xq, self.xt)
        dr.dr_qmatmul(self.xq, self.w, y, fast=True, workspace=self.workspace)
        return y

    def backward(self, dy, dx, first: bool):
        """dx = dy W; dy^T x into the gradient's place, or on top of the micro-batches before."""
        dr.dr_quantize(dy, self.dyq, self.dyt)
        if dx is not None:
            dr.dr_qmatmul(self.dyq, self.wt, dx, fast=True, workspace=self.workspace)
        dr.dr_qmatmul(self.dyt, self.xt, self.grad, accumulate=not first, workspace=self.workspace)
        return dx


class RolloutRank:
    """A tensor-parallel rank's down projection (a slice of its columns) and output matrix (a slice of the words)."""

    def __init__(self, stream, tensors, name_down: str):
        self.views = [stream[t["byte_offset"]:t["byte_offset"] + 2 * t["rows"] * t["cols"]].view(torch.bfloat16)
                      .view(t["rows"], t["cols"]) for t in (tensors[name_down], tensors["lm_head"])]
        self.down, self.head = (dr.QMatrix.empty(*v.shape, 128) for v in self.views)

    def take_weights(self):
        for view, q in zip(self.views, (self.down, self.head)):
            dr.dr_quantize(view, q)


def linear(x, w, dtype):
    out = torch.empty((x.shape[0], w.rows), dtype=dtype, device=x.device)
    workspace = torch.empty(dr.dr_qlinear_workspace(x.shape[0], w), dtype=torch.uint8, device=x.device)
    dr.dr_qlinear(x, w, out, fast=True, workspace=workspace)
    return out


def rollout(ranks, a, residual):
    """Logits; the sum over the ranks and the joining of the words are collectives where the ranks are GPUs."""
    per = a.shape[1] // len(ranks)
    h = residual.float()
    for i, rank in enumerate(ranks):
        h = h + linear(a[:, i * per:(i + 1) * per], rank.down, torch.float32)
    h = h.to(torch.bfloat16)
    return torch.cat([linear(h, rank.head, torch.bfloat16) for rank in ranks], dim=1)


def cross_entropy(logits, targets):
    return torch.nn.functional.cross_entropy(logits.float(), targets).item()


def run(workload="tiny", layers=1, tokens=200, steps=3, lr=1.0, max_norm=1.0, seed=0, device="cuda"):
    """Losses of the training role and of the rollout role (before each step, and after the last one for the rollout),
    the gradients' norms before and the clipped gradients of the last step."""
    wl = workloads.BY_NAME[workload]
    model = (layers,) + wl.model[1:]
    hidden, ffn, vocab = model[1], model[5], model[6]
    w = wl.train_shards
    flat = datagen.make_flat_torch(model, w, seed, device)
    grads = torch.zeros_like(flat)
    shards, grad_shards = flat.chunk(w), grads.chunk(w)

    at, place = 0, {}
    for name, numel, _ in datagen.tensor_list(model):
        place[name] = slice(at, at + numel)
        at += numel
    name_down = f"layers.{layers - 1}.down"
    micro = tokens // MICRO_BATCHES
    down = TrainedLinear(flat[place[name_down]].view(hidden, ffn), grads[place[name_down]].view(hidden, ffn), micro)
    head = TrainedLinear(flat[place["lm_head"]].view(vocab, hidden), grads[place["lm_head"]].view(vocab, hidden), micro)
    clip = dr.GradList(grad_shards)
    norm = torch.empty(1, device=device)
    clip_workspace = torch.empty(dr.dr_grad_workspace(), dtype=torch.uint8, device=device)

    plan = dr.dr_plan_create(model, w, wl.tp, wl.chunk_bytes)
    info = dr.dr_plan_get_info(plan)
    stream = torch.empty(info["rollout_bytes"], dtype=torch.uint8, device=device)
    checksums = torch.empty((info["num_chunks"], 2), dtype=torch.int64, device=device)
    ranks = []
    for r in range(wl.tp):
        described = [dr.dr_plan_tensor(plan, r, i) for i in range(3 + 6 * layers)]
        ranks.append(RolloutRank(stream, {t["name"]: t for t in described}, name_down))

    gen = torch.Generator(device=device).manual_seed(seed)
    count = micro * MICRO_BATCHES
    a = torch.randn((count, ffn), generator=gen, device=device).to(torch.bfloat16)
    residual = torch.randn((count, hidden), generator=gen, device=device).to(torch.bfloat16)
    targets = torch.randint(vocab, (count,), generator=gen, device=device)

    out = {"train_loss": [], "rollout_loss": [], "norm": [], "token_matches": []}
    projected = torch.empty((micro, hidden), dtype=torch.bfloat16, device=device)
    logits = torch.empty((micro, vocab), dtype=torch.bfloat16, device=device)
    dh = torch.empty((micro, hidden), dtype=torch.bfloat16, device=device)
    for step in range(steps + 1):
        dr.dr_stage_all(plan, shards, stream, checksums)
        for rank in ranks:
            rank.take_weights()
        prompt = rollout(ranks, a, residual)
        token = rollout(ranks, a[-1:], residual[-1:])
        out["rollout_loss"].append(cross_entropy(prompt, targets))
        out["token_matches"].append((token.float() - prompt[-1:].float()).abs().max().item())
        if step == steps:
            break

        down.take_weights()
        head.take_weights()
        loss = 0.0
        for i in range(MICRO_BATCHES):
            rows = slice(i * micro, (i + 1) * micro)
            h = residual[rows] + down.forward(a[rows], projected)
            head.forward(h, logits)
            loss += cross_entropy(logits, targets[rows]) / MICRO_BATCHES
            dlogits = torch.softmax(logits.float(), dim=1)
            dlogits[torch.arange(micro, device=device), targets[rows]] -= 1.0
            head.backward((dlogits / count).to(torch.bfloat16), dh, first=i == 0)
            down.backward(dh, None, first=i == 0)
        dr.dr_grad_clip(clip, max_norm, norm, clip_workspace)
        torch._foreach_add_(list(shards), list(grad_shards), alpha=-lr)
        out["train_loss"].append(loss)
        out["norm"].append(norm.item())
    out["clipped"] = list(grad_shards)
    torch.cuda.synchronize()
    plan.close()
    return out


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--workload", choices=sorted(workloads.BY_NAME), default="tiny")
    p.add_argument("--layers", type=int, default=1)
    p.add_argument("--tokens", type=int, default=200)
    p.add_argument("--steps", type=int, default=3)
    args = p.parse_args()
    out = run(args.workload, args.layers, args.tokens, args.steps)
    for i, loss in enumerate(out["rollout_loss"]):
        line = f"step {i}: rollout loss {loss:.4f}"
        if i < args.steps:
            line += f", training loss {out['train_loss'][i]:.4f}, gradient norm {out['norm'][i]:.4f}"
        print(line, flush=True)


if __name__ == "__main__":
    main()
