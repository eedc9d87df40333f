"""Trains a pruned MoE layer on its own answers and on preferred ones.

    python examples/align_pruned_layer.py

A toy language model as in recover_pruned_layer.py: rows, one MoE layer with its residual, and a head.  The layer is pruned
(moe_expert_outputs, prune_enumerate) and then trained as a whole: every token's row goes to the experts that it is routed to, all of an
expert's side by side (moe_dispatch_rows), each expert's block runs on its own (expert_ffn_forward), and the outputs come back weighted
(moe_combine_rows).  Two losses take turns: the clipped policy loss of tokens sampled from the layer itself, with the unpruned
layer's log probabilities as rewards and a KL term to the pruned one as it was (moe_policy_loss), and the preference loss of pairs of answers
(moe_preference_loss).  Their gradients go back the same way, into the experts, the router and the rows (moe_combine_rows_backward,
expert_ffn_backward, moe_dispatch_rows_backward).
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
    """A layer's weights, and what a forward pass leaves for the backward one."""

    def __init__(self, E, k, H, F, dtype, seed, kept=None, beta=0.0):
        layer = wl.make_layer(wl.LayerConfig("toy", seed, dtype, E=E, k=k, H=H, F=F, T=64, rs=(E // 2,), rms_norm=True))
        self.k, self.kept, self.beta = k, (1 << E) - 1 if kept is None else kept, beta
        self.Wgate, self.W1, self.W3, self.W2 = (layer[n].to(DEV).contiguous() for n in ("Wgate", "W1", "W3", "W2"))

    def weights(self):
        return self.Wgate, self.W1, self.W3, self.W2

    def forward(self, x):
        E = self.Wgate.shape[0]
        # (the routing alone is wanted here: the layer's output that comes with it is thrown away, a forward pass in all)
        _, used, logits, experts = moep.moe_forward_skip_topk(x, *self.weights(), self.k, self.beta, self.kept)
        there = torch.arange(self.k, device=x.device) < used[:, None]
        weights = torch.softmax(logits.gather(1, experts.long()).masked_fill(~there, -torch.inf), 1).contiguous()
        rows, slot_of, offsets = moep.moe_dispatch_rows(x, experts, E, used=used)
        y, ends, gate_up = torch.empty_like(rows), offsets.tolist(), {}
        for e in range(E):
            mine = slice(ends[e], ends[e + 1])
            if ends[e] < ends[e + 1]:
                y[mine], gate_up[e] = moep.expert_ffn_forward(rows[mine], self.W1[e], self.W3[e], self.W2[e], save=True)
        self.saved = x, experts, weights, slot_of, rows, y, ends, gate_up
        return moep.moe_combine_rows(y, slot_of, weights)

    def backward(self, dout):
        """The gradients of x, Wgate, W1, W3 and W2 from that of the last forward pass's output."""
        x, experts, weights, slot_of, rows, y, ends, gate_up = self.saved
        grads = [torch.zeros_like(w) for w in self.weights()]
        dy, dw = moep.moe_combine_rows_backward(dout, y, slot_of, weights, dy=y)
        for e, kept in gate_up.items():
            mine = slice(ends[e], ends[e + 1])
            drows, *of_weights = moep.expert_ffn_backward(dy[mine], rows[mine], self.W1[e], self.W3[e], self.W2[e], kept)
            dy[mine] = drows
            for g, d in zip(grads[1:], of_weights):
                g[e] = d
        dx = moep.moe_dispatch_rows_backward(dy, slot_of)
        # the routing weights are a softmax over the token's own experts
        of_slots = weights * (dw - (weights * dw).sum(1, keepdim=True))
        of_logits = torch.zeros((x.shape[0], self.Wgate.shape[0]), device=x.device).scatter_add_(1, experts.long(), of_slots)
        grads[0] = (of_logits.T @ x.float()).to(x.dtype)
        return ((dx.float() + of_logits @ self.Wgate.float()).to(x.dtype), *grads)


def say(layer, x, head):
    """Logits of the toy model: the rows, the layer's output on top, and the head."""
    return (x.float() + 2.0 * layer.forward(x).float()).to(x.dtype) @ head.T


def learn(layer, dlogits, head, rate):
    """One step down the gradient, `rate` of every weight's own size, from the gradient of the logits; the gradient of the rows."""
    dx, *grads = layer.backward((2.0 * (dlogits @ head).float()).to(head.dtype))
    for w, g in zip(layer.weights(), grads):
        m, d = w.float(), g.float()
        w.copy_(m - rate * m.norm() / d.norm().clamp(min=1e-30) * d)
    return dx


def align(E=8, r=4, k=2, H=256, F=512, V=4003, P=8, length=64, steps=6, rate=0.001, dtype="bf16", seed=5):
    full = Layer(E, k, H, F, dtype, seed)
    g = torch.Generator(device=DEV).manual_seed(seed)
    dt = full.Wgate.dtype
    head = (4.0 * torch.randn((V, H), generator=g, device=DEV) / H ** 0.5).to(dt)
    # 2 P answers of up to `length` tokens, the first P of them preferred; a few rows of padding behind
    lengths = torch.randint(length // 2, length + 1, (2 * P,), generator=g, device=DEV)
    offsets = torch.cat([torch.zeros(1, dtype=torch.int64, device=DEV), lengths.cumsum(0)])
    T = int(offsets[-1]) + 5
    x = torch.randn((T, H), generator=g, device=DEV)
    x = (x / x.square().mean(1, keepdim=True).sqrt()).to(dt)

    logits, Y = moep.moe_expert_outputs(x, *full.weights())
    kept = int(moep.prune_enumerate(logits, Y, k, r)[2].item()) & 0xFFFFFFFF
    pruned, start = Layer(E, k, H, F, dtype, seed, kept), Layer(E, k, H, F, dtype, seed, kept)
    teacher = say(full, x, head)
    reference = say(start, x, head)
    answer = torch.arange(T, device=DEV) < offsets[-1]
    losses = {"policy": [], "preference": []}
    for step in range(steps):
        z = say(pruned, x, head)
        if step % 2 == 0:                                   # its own answers, judged by the unpruned layer
            noise = -torch.log(-torch.log(torch.rand(z.shape, generator=g, device=DEV).clamp(1e-9, 1 - 1e-7)))
            tokens = torch.where(answer, (z.float() + noise).argmax(1), -1)
            old = moep.moe_token_logprobs(z, tokens)[0]
            reward = moep.moe_token_logprobs(teacher, tokens)[0]
            advantages = torch.where(answer, (reward - reward[answer].mean()) / reward[answer].std(), 0.0)
            ref = moep.moe_token_logprobs(reference, tokens)[0]
            weights = answer.float() / answer.sum()
            for _ in range(2):                              # two steps on the same answers: the second one's ratios are no longer 1
                loss, _, _, dz = moep.moe_policy_loss(z, tokens, old, advantages, ref, kl=0.02, weights=weights, gradient=True, out=z)
                losses["policy"].append(float((weights * loss).sum()))
                learn(pruned, dz, head, rate)
                z = say(pruned, x, head)
        else:                                               # preferred answers: what the unpruned layer says, against anything
            best = moep.moe_token_logprobs(teacher, torch.full((T,), -1, dtype=torch.int64, device=DEV), 1)[3][:, 0].long()
            anything = torch.randint(0, V, (T,), generator=g, device=DEV)
            tokens = torch.where(torch.arange(T, device=DEV) < offsets[P], best, anything)
            ref = moep.moe_token_logprobs(reference, tokens)[0]
            dz = torch.zeros_like(z)                        # (the padding's rows stay as they are)
            loss, rewards, *_ = moep.moe_preference_loss(z, tokens, offsets, ref, beta=0.05, average=True, gradient=True, out=dz)
            losses["preference"].append(float(loss.mean()))
            learn(pruned, dz / P, head, rate)
    return {"kept": kept, "losses": losses}


if __name__ == "__main__":
    result = align()
    print(f"kept experts {result['kept']:#x}")
    for name, losses in result["losses"].items():
        print(f"{name:>10}: " + "  ".join(f"{x:.4f}" for x in losses))
