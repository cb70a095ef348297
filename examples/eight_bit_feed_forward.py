"""A decoder layer's gated feed-forward block in 8 bits: training with 8-bit activation checkpoints, rollout on the staged weights.

    python examples/eight_bit_feed_forward.py [--workload tiny|0.5b|8b] [--tokens 200] [--steps 3] [--act silu|gelu]

    block:  y = h Wd^T,  h = act(x Wg^T) * (x Wu^T)        loss = half the mean square of y - target

gate and up lie one behind the other in the flat training layout, so that the training role sees them as one matrix of
2F rows, as the rollout ranks do after staging.  Between its forward and its backward pass the training role keeps x, gate
and up in 8 bits and nothing else of the block (TrainedBlock.saved); the backward pass takes x^T from x and h^T from gate
and up.  The weights' gradients add up in a flat fp32 buffer of the training layout.  Then the weights are staged again and
every rollout rank runs the block on its slice, for a prompt and for a single token.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2607_22614_amd import datagen, dr, workloads  # noqa: E402

ACTS = {"silu": dr.DR_ACT_SILU, "gelu": dr.DR_ACT_GELU_TANH}


class TrainedBlock:
    """Forward and backward over views of the flat weights and of the flat gradients, for `tokens` rows."""

    def __init__(self, gate_up, down, grad_gate_up, grad_down, tokens: int, act: int):
        f2, hidden = gate_up.shape
        f, m = f2 // 2, tokens
        self.weights, self.grads, self.act = (gate_up, down), (grad_gate_up, grad_down), act
        empty = dr.QMatrix.empty
        self.w, self.wt = empty(f2, hidden, 128), empty(hidden, f2, 128)
        self.wd, self.wdt = empty(hidden, f, 128), empty(f, hidden, 128)
        self.saved = {"x": empty(m, hidden), "gate": empty(m, f), "up": empty(m, f)}
        # used within one pass; a program with many layers keeps one of each for all of them
        self.h, self.ht, self.xt = empty(m, f), empty(f, m), empty(hidden, m)
        self.dy, self.dyt, self.d, self.dt = empty(m, hidden), empty(hidden, m), empty(m, f2), empty(f2, m)
        self.dh = torch.empty((m, f), dtype=torch.bfloat16, device=gate_up.device)
        products = ((m, hidden, f), (m, f, hidden), (m, hidden, f2), (f2, hidden, m), (hidden, f, m))
        need = max([dr.dr_qmatmul_workspace(*p) for p in products] + [dr.dr_qgated_save_workspace(m, self.w)])
        self.workspace = torch.empty(need, dtype=torch.uint8, device=gate_up.device)

    def take_weights(self):
        """Once a step: square blocks give a matrix and its transpose the same codes."""
        dr.dr_quantize(self.weights[0], self.w, self.wt)
        dr.dr_quantize(self.weights[1], self.wd, self.wdt)

    def forward(self, x, y):
        s = self.saved
        dr.dr_quantize(x, s["x"])
        dr.dr_qgated_save(s["x"], self.w, self.h, s["gate"], s["up"], act=self.act, fast=True, workspace=self.workspace)
        dr.dr_qmatmul(self.h, self.wd, y, fast=True, workspace=self.workspace)
        return y

    def backward(self, dy, dx, first: bool):
        """dx, and the weights' gradients in their places, or on top of the micro-batches before."""
        s, ws = self.saved, self.workspace
        dr.dr_quantize(dy, self.dy, self.dyt)
        dr.dr_qmatmul(self.dy, self.wdt, self.dh, fast=True, workspace=ws)
        dr.dr_gated_backward(self.dh, s["gate"], s["up"], self.d, self.dt, self.ht, act=self.act)
        dr.dr_qtranspose(s["x"], self.xt)
        dr.dr_qmatmul(self.d, self.wt, dx, fast=True, workspace=ws)
        dr.dr_qmatmul(self.dt, self.xt, self.grads[0], accumulate=not first, workspace=ws)
        dr.dr_qmatmul(self.dyt, self.ht, self.grads[1], accumulate=not first, workspace=ws)
        return dx


class RolloutRank:
    """A tensor-parallel rank's slice of the block: gate's and up's rows, and the down projection's columns."""

    def __init__(self, stream, tensors, layer: int):
        self.views = [stream[t["byte_offset"]:t["byte_offset"] + 2 * t["rows"] * t["cols"]].view(torch.bfloat16)
                      .view(t["rows"], t["cols"]) for t in (tensors[f"layers.{layer}.gate_up"], tensors[f"layers.{layer}.down"])]
        self.w, self.wd = (dr.QMatrix.empty(*v.shape, 128) for v in self.views)

    def take_weights(self):
        for view, q in zip(self.views, (self.w, self.wd)):
            dr.dr_quantize(view, q)

    def forward(self, x, act: int):
        """The rank's share of y; the sum over the ranks is a collective where the ranks are GPUs."""
        m = x.shape[0]
        need = max(dr.dr_qgated_workspace(m, self.w), dr.dr_qlinear_workspace(m, self.wd))
        workspace = torch.empty(need, dtype=torch.uint8, device=x.device)
        h = torch.empty((m, self.w.rows // 2), dtype=torch.bfloat16, device=x.device)
        y = torch.empty((m, self.wd.rows), dtype=torch.float32, device=x.device)
        dr.dr_qgated(x, self.w, h, act=act, fast=True, workspace=workspace)
        dr.dr_qlinear(h, self.wd, y, fast=True, workspace=workspace)
        return y


def run(workload="tiny", tokens=200, steps=3, lr=100.0, act="silu", seed=0, device="cuda"):
    """Losses, the rollout's outputs for the prompt and for its last token alone, and the block of the last step (weights before
    the update, inputs, gradients)."""
    wl = workloads.BY_NAME[workload]
    model = (1,) + wl.model[1:]
    hidden, ffn = model[1], model[5]
    flat = datagen.make_flat_torch(model, wl.train_shards, seed, device)
    grads = torch.zeros_like(flat)
    at, place = 0, {}
    for name, numel, _ in datagen.tensor_list(model):
        place[name] = slice(at, at + numel)
        at += numel

    def fused(buffer):
        assert place["layers.0.gate"].stop == place["layers.0.up"].start
        return buffer[place["layers.0.gate"].start:place["layers.0.up"].stop].view(2 * ffn, hidden)

    def down(buffer):
        return buffer[place["layers.0.down"]].view(hidden, ffn)

    block = TrainedBlock(fused(flat), down(flat), fused(grads), down(grads), tokens, ACTS[act])
    plan = dr.dr_plan_create(model, wl.train_shards, wl.tp, wl.chunk_bytes)
    info = dr.dr_plan_get_info(plan)
    stream = torch.empty(info["rollout_bytes"], dtype=torch.uint8, device=device)
    checksums = torch.empty((info["num_chunks"], 2), dtype=torch.int64, device=device)
    ranks = []
    for r in range(wl.tp):
        described = [dr.dr_plan_tensor(plan, r, i) for i in range(9)]
        ranks.append(RolloutRank(stream, {t["name"]: t for t in described}, 0))

    gen = torch.Generator(device=device).manual_seed(seed)
    x = torch.randn((tokens, hidden), generator=gen, device=device).to(torch.bfloat16)
    target = torch.randn((tokens, hidden), generator=gen, device=device)
    y, dx = (torch.empty((tokens, hidden), dtype=torch.bfloat16, device=device) for _ in range(2))
    out = {"loss": [], "x": x, "act": act}
    for _ in range(steps):
        block.take_weights()
        block.forward(x, y)
        error = y.float() - target
        out["loss"].append(0.5 * error.square().mean().item())
        out["dy"] = (error / error.numel() * 1024.0).to(torch.bfloat16)  # scaled, so that bf16 and 8 bits stay far from their ends
        block.backward(out["dy"], dx, first=True)
        out["weights"] = (fused(flat).clone(), down(flat).clone())
        torch._foreach_add_(list(block.weights), list(block.grads), alpha=-lr / 1024.0)
    out.update(dx=dx, gate_up_grad=block.grads[0], down_grad=block.grads[1])

    dr.dr_stage_all(plan, flat.chunk(wl.train_shards), stream, checksums)
    for rank in ranks:
        rank.take_weights()
    block.take_weights()
    out["trained_y"] = block.forward(x, y).float()
    out["prompt_y"] = sum(rank.forward(x, ACTS[act]) for rank in ranks)
    out["token_y"] = sum(rank.forward(x[-1:], ACTS[act]) for rank in ranks)
    torch.cuda.synchronize()
    plan.close()
    return out


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--workload", choices=sorted(workloads.BY_NAME), default="tiny")
    p.add_argument("--tokens", type=int, default=200)
    p.add_argument("--steps", type=int, default=3)
    p.add_argument("--act", choices=sorted(ACTS), default="silu")
    args = p.parse_args()
    out = run(args.workload, args.tokens, args.steps, act=args.act)
    for i, loss in enumerate(out["loss"]):
        print(f"step {i}: loss {loss:.5f}", flush=True)
    difference = (out["prompt_y"] - out["trained_y"]).norm() / out["trained_y"].norm()
    print(f"rollout against training: {difference.item():.4f} of the output's norm", flush=True)


if __name__ == "__main__":
    main()
