"""Prunes one MoE layer and wins back what that cost by distilling from the unpruned layer.

    python examples/recover_pruned_layer.py

A toy language model: embeddings, one MoE layer with its residual, and a head.  The unpruned model scores the calibration tokens once and
keeps each token's best alternatives (moe_token_logprobs); the layer is pruned to the experts with the smallest reconstruction loss
(moe_expert_outputs, prune_enumerate); then the kept experts are trained on the distillation loss against the kept alternatives
(moe_distill_topk), its gradient carried through the head into each expert's block on the rows routed to it (expert_ffn_forward,
expert_ffn_backward).  Likelihoods of held-out tokens are reported before and after.
"""
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import torch

import paper_2402_14800_amd as moep
from paper_2402_14800_amd import workloads as wl

DEV = "cuda:0"


class Layer:
    """The layer's weights; the experts' in fp32 as well, which is where they are updated."""

    def __init__(self, E, k, H, F, T, seed):
        layer = wl.make_layer(wl.LayerConfig("toy", seed, "bf16", E=E, k=k, H=H, F=F, T=T, rs=(E // 2,), rms_norm=True))
        self.x = layer["x"].to(DEV)
        self.Wgate, self.W1, self.W3, self.W2 = (layer[n].to(DEV).contiguous() for n in ("Wgate", "W1", "W3", "W2"))
        self.master = [w.float() for w in (self.W1, self.W3, self.W2)]

    def update(self, e, grads, rate):
        for w, m, g in zip((self.W1, self.W3, self.W2), self.master, grads):
            m[e] -= rate * g.float()
            w[e] = m[e].to(w.dtype)


def routed(layer, x, kept):
    """Rows and weights (Eq. 1) of every kept expert, from the routing of the pruned layer itself."""
    _, _, logits, top2 = moep.moe_forward_pruned_skip(x, layer.Wgate, layer.W1, layer.W3, layer.W2, kept, 0.0)
    w = torch.softmax(logits.gather(1, top2.long()), dim=1)
    for e in range(layer.Wgate.shape[0]):
        if (kept >> e) & 1:
            row, slot = (top2 == e).nonzero(as_tuple=True)
            yield e, row, w[row, slot][:, None]


def recover(E=8, r=4, H=256, F=512, V=4003, T=2048, K=32, steps=30, rate=0.1, temperature=1.0, seed=3):
    layer = Layer(E, 2, H, F, 256, seed)
    g = torch.Generator(device=DEV).manual_seed(seed)
    head = (4.0 * torch.randn((V, H), generator=g, device=DEV) / H ** 0.5).to(torch.bfloat16)
    # tokens of 256 kinds in contexts that differ: what is learnt on some of them holds for others
    kind = torch.randint(0, 256, (2 * T,), generator=g, device=DEV)
    rows = layer.x.float()[kind] + 0.3 * torch.randn((2 * T, H), generator=g, device=DEV)
    rows = (rows / rows.square().mean(1, keepdim=True).sqrt()).to(torch.bfloat16)
    x, held_out = rows[:T].contiguous(), rows[T:].contiguous()

    # the unpruned model: what it says, kept as each token's best alternatives
    def say(rows, kept):
        out = moep.moe_forward_pruned_skip(rows, layer.Wgate, layer.W1, layer.W3, layer.W2, kept, 0.0)[0]
        return (rows.float() + 2.0 * out.float()).to(torch.bfloat16) @ head.T

    everyone = (1 << E) - 1
    none = torch.full((T,), -1, dtype=torch.int64, device=DEV)
    _, _, top_lp, top_ids = moep.moe_token_logprobs(say(x, everyone), none, K)
    _, _, _, answers = moep.moe_token_logprobs(say(held_out, everyone), none, 1)
    answers = answers[:, 0].long().contiguous()

    # the pruned layer
    logits, Y = moep.moe_expert_outputs(x, layer.Wgate, layer.W1, layer.W3, layer.W2)
    _, _, mask, _ = moep.prune_enumerate(logits, Y, 2, r)
    kept = int(mask.item()) & 0xFFFFFFFF

    def score():
        logprob, _, _, best = moep.moe_token_logprobs(say(held_out, kept), answers, 1)
        return float(logprob.mean()), float((best[:, 0] == answers).float().mean())

    before, losses = score(), []
    weights = torch.full((T,), 1.0 / T, device=DEV)
    for _ in range(steps):
        out, passes = torch.zeros((T, H), device=DEV), []
        for e, row, w in routed(layer, x, kept):
            rows = x[row]
            y, gate_up = moep.expert_ffn_forward(rows, layer.W1[e], layer.W3[e], layer.W2[e], save=True)
            out.index_add_(0, row, w * y.float())
            passes.append((e, row, w, rows, gate_up))
        student = (x.float() + 2.0 * out).to(torch.bfloat16) @ head.T
        loss, _, grad = moep.moe_distill_topk(student, top_ids, top_lp, temperature, weights=weights, gradient=True, out=student)
        losses.append(float(loss.mean()))
        dout = 2.0 * (grad @ head).float()
        for e, row, w, rows, gate_up in passes:
            dy = (w * dout[row]).to(torch.bfloat16)
            grads = moep.expert_ffn_backward(dy, rows, layer.W1[e], layer.W3[e], layer.W2[e], gate_up, input_gradient=False)
            layer.update(e, grads[1:], rate)
    return {"kept": kept, "losses": losses, "before": before, "after": score()}


if __name__ == "__main__":
    result = recover()
    print(f"kept experts {result['kept']:#x}; distillation loss {result['losses'][0]:.4f} -> {result['losses'][-1]:.4f}")
    for when in ("before", "after"):
        logprob, same = result[when]
        print(f"{when:>6}: log probability of the unpruned model's answers {logprob:.4f}, the same answer for {100 * same:.1f} %")
