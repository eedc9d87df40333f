"""Timed cases of the operators that score, distil and train a pruned model's expert layer.

Three operators, told apart by a case's "kind":

  logprobs   log probabilities of given tokens with the entropy and the K best alternatives of every row of logits
  distill    the distillation loss from a teacher's K best logits, and its gradient: "fused" asks for both in one call with
             the tokens' weights at hand, "split" takes the loss first and the gradient from an upstream one afterwards
  ffn        one expert's gated feed-forward block: "forward" alone, as it is served, or a "step" of training, which returns
             the gradients of its input and of its three weights as well

Ranges: rows 1 .. 8192, vocabularies 257 .. 131072 (any number, odd ones among them; rows may lie further apart than they are
long, and the end of a padded vocabulary may be masked with -inf), K 0 .. 100; blocks of the benchmark's and the tests' layer
shapes and others of the same ranges, H 64 .. 4096, F 64 .. 14336; bf16 and fp32 storage (the fp32 blocks are small ones).
"""
import math

import torch

own = False

DEV = "cuda:0"
MIXTRAL = dict(H=4096, F=14336)
MANY = dict(H=2048, F=5632)
MID = dict(H=1024, F=3584)
SMALL = dict(H=512, F=1024)


def _logprobs(name, T, V, K, dtype="bf16", pad=0, masked=0):
    return dict(name=name, kind="logprobs", T=T, V=V, K=K, dtype=dtype, pad=pad, masked=masked)


def _distill(name, mode, T, V, K, dtype="bf16", tau=1.0, pad=0):
    return dict(name=name, kind="distill", mode=mode, T=T, V=V, K=K, dtype=dtype, tau=tau, pad=pad)


def _ffn(name, mode, T, H, F, dtype="bf16"):
    return dict(name=name, kind="ffn", mode=mode, T=T, H=H, F=F, dtype=dtype)


def listed():
    return [
        # one generated token: its log probability and what else the model might have said
        _logprobs("score_1", 1, 32000, 20),
        # likelihood evaluation of a pruned model, answers scored and checked for being the greedy choice; ragged
        _logprobs("score_1999", 1999, 32000, 1),
        # fp32 logits over an odd vocabulary whose padded end is masked
        _logprobs("score_f32_777", 777, 50001, 5, dtype="f32", pad=79, masked=33),
        # a teacher's alternatives kept for distillation, large vocabulary
        _logprobs("teacher_131072", 2048, 131072, 64),
        # a toy model's step: launches and latency
        _distill("distill_tiny_33", "fused", 33, 1003, 8, dtype="f32"),
        # a training batch against the kept alternatives
        _distill("distill_4096", "fused", 4096, 32000, 64, tau=2.0),
        # loss and gradient apart, as an autograd engine calls them; odd vocabulary
        _distill("distill_split_1001", "split", 1001, 50001, 10, tau=1.5),
        # the large vocabulary
        _distill("distill_131072", "fused", 2048, 131072, 100),
        # one token through one expert as it is served
        _ffn("ffn_token_1", "forward", 1, **MIXTRAL),
        # the rows that routing leaves one expert of a mid-sized layer in a training batch
        _ffn("ffn_step_777", "step", 777, **MID),
        # a small layer kept in fp32
        _ffn("ffn_step_f32_1501", "step", 1501, dtype="f32", **SMALL),
        # a Mixtral-shaped expert on its share of a long batch
        _ffn("ffn_step_8192", "step", 8192, **MIXTRAL),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    while True:
        kind = rng.choice(["logprobs", "distill", "ffn"])
        dtype = "f32" if rng.random() < 0.25 else "bf16"
        if kind == "ffn":
            shape = rng.choice([MIXTRAL, MANY, MID, None])
            if dtype == "f32" or shape is None:
                top = (16, 56) if dtype == "f32" else (64, 224)
                shape = dict(H=64 * _log(rng, 1, top[0]), F=64 * _log(rng, 1, top[1]))
            c = _ffn("", rng.choice(["forward", "step", "step"]), _log(rng, 1, 8192), dtype=dtype, **shape)
        else:
            V = rng.choice([32000, 131072, _log(rng, 257, 131072), _log(rng, 257, 131072)])
            T, pad = _log(rng, 1, 8192), rng.choice([0, 0, 1, 64])
            if kind == "logprobs":
                c = _logprobs("", T, V, rng.choice([0, 1, 5, 20, 64, 100]), dtype=dtype, pad=pad, masked=rng.choice([0, 0, 1, V // 50]))
            else:
                c = _distill("", rng.choice(["fused", "split"]), T, V, rng.choice([4, 10, 64, 100]), dtype=dtype,
                             tau=rng.choice([1.0, 1.5, 2.0]), pad=pad)
        w = work(c)
        limit = (1.0e11, 1.1e9) if dtype == "f32" else (8.7e12, 1.1e9)
        sizes = [c.get(n) for n in ("T", "V", "H", "F")] + [c.get("V", 0) + c.get("pad", 0)]
        if w["flops"] <= limit[0] and w["bytes"] <= limit[1] and 3072 not in sizes:
            del c["name"]
            return c


# ---------------------------------------------------------------- inputs
def _type(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _rows(case, g):
    """Logits as a language model's head gives them: a wide bulk and, in every row, a few tokens well above it."""
    T, V = case["T"], case["V"]
    z = torch.randn((T, V), generator=g, device=DEV).mul_(2.0)
    at = torch.randint(0, V, (T, 12), generator=g, device=DEV)
    z.scatter_add_(1, at, 4.0 + 3.0 * torch.randn((T, 12), generator=g, device=DEV))
    if case.get("masked"):
        z[:, V - case["masked"]:] = -math.inf
    wide = torch.zeros((T, V + case["pad"]), dtype=_type(case), device=DEV)
    wide[:, :V] = z
    return wide[:, :V]


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    T, kind = case["T"], case["kind"]
    if kind == "ffn":
        H, F, dt = case["H"], case["F"], _type(case)
        draw_ = lambda *shape: torch.randn(shape, generator=g, device=DEV)  # noqa: E731
        s = dict(case=case, x=draw_(T, H).to(dt))
        s["W1"], s["W3"] = ((draw_(F, H) / math.sqrt(H)).to(dt) for _ in range(2))
        s["W2"] = (draw_(H, F) / math.sqrt(F)).to(dt)
        if case["mode"] == "step":
            s["dy"] = draw_(T, H).to(dt)
        return s
    V, K = case["V"], case["K"]
    s = dict(case=case, logits=_rows(case, g))
    if kind == "logprobs":
        tokens = torch.randint(0, V - case["masked"], (T,), generator=g, device=DEV)
        prompt = torch.rand((T,), generator=g, device=DEV) < 0.1      # tokens that are not scored
        s["tokens"] = torch.where(prompt & (T > 1), torch.full_like(tokens, -1), tokens)
        return s
    teacher = s["logits"].float() + 0.7 * torch.randn((T, V), generator=g, device=DEV)
    s["teacher"], ids = torch.topk(teacher, K, dim=1)
    short = torch.rand((T, 1), generator=g, device=DEV) < 0.1         # rows for which the teacher kept half as many
    s["ids"] = torch.where(short & (torch.arange(K, device=DEV) >= (K + 1) // 2), torch.full_like(ids, -1), ids).to(torch.int32)
    s["teacher"] = s["teacher"].contiguous()
    answer = torch.rand((T,), generator=g, device=DEV) >= 0.1         # the others' weight is 0: not trained on
    answer[0] = True
    s["weights"] = answer.float() * (0.5 + torch.rand((T,), generator=g, device=DEV)) / T
    return s


# ---------------------------------------------------------------- one pass
def run(state):
    c = state["case"]
    if own:
        return _run_own(c, state)
    return {"logprobs": _plain_logprobs, "distill": _plain_distill, "ffn": _plain_ffn}[c["kind"]](c, state)


def _run_own(c, s):
    import paper_2402_14800_amd as pkg

    if c["kind"] == "logprobs":
        return pkg.moe_token_logprobs(s["logits"], s["tokens"], c["K"])
    if c["kind"] == "distill":
        if c["mode"] == "fused":
            loss, _, grad = pkg.moe_distill_topk(s["logits"], s["ids"], s["teacher"], c["tau"], weights=s["weights"], gradient=True)
            return loss, grad
        loss, lse = pkg.moe_distill_topk(s["logits"], s["ids"], s["teacher"], c["tau"])
        return loss, pkg.moe_distill_topk_backward(s["logits"], s["ids"], s["teacher"], lse, s["weights"], c["tau"])
    if c["mode"] == "forward":
        return pkg.expert_ffn_forward(s["x"], s["W1"], s["W3"], s["W2"])
    y, gate_up = pkg.expert_ffn_forward(s["x"], s["W1"], s["W3"], s["W2"], save=True)
    return (y, *pkg.expert_ffn_backward(s["dy"], s["x"], s["W1"], s["W3"], s["W2"], gate_up))


def _plain_logprobs(c, s):
    z, K = s["logits"].float(), c["K"]
    m = z.amax(1, keepdim=True)
    e = (z - m).exp()
    total = e.sum(1, keepdim=True)
    lse = m + total.log()
    there = e > 0
    entropy = (total.log() - torch.where(there, e * (z - m), 0.0).sum(1, keepdim=True) / total).squeeze(1)
    tokens = s["tokens"]
    given = tokens >= 0
    logprob = torch.where(given, z.gather(1, tokens.clamp(min=0)[:, None]).squeeze(1) - lse.squeeze(1), 0.0)
    # a value and its index in one number, so that ties go to the lowest index
    bits = (z + 0.0).view(torch.int32).long()
    order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits)
    keys = (order << 32) | (c["V"] - 1 - torch.arange(c["V"], device=z.device))
    best = c["V"] - 1 - (torch.topk(keys, K, dim=1).values & 0xFFFFFFFF)
    return logprob, entropy, z.gather(1, best) - lse, best.to(torch.int32)


def _plain_distill(c, s):
    """Of a row: tau^2 sum_j q_j (log q_j - log p_j), q the softmax of the teacher's K logits over tau, p that of all the student's;
    the gradient is tau (p - q) times the row's weight."""
    z, tau = s["logits"].float() / c["tau"], c["tau"]
    ids, w = s["ids"].long(), s["weights"]
    there = ids >= 0
    t = torch.where(there, s["teacher"] / tau, -math.inf)
    log_q = t - t.amax(1, keepdim=True)
    q = log_q.exp()
    norm = q.sum(1, keepdim=True)
    q, log_q = q / norm, torch.where(there, log_q - norm.log(), 0.0)
    m = z.amax(1, keepdim=True)
    e = (z - m).exp()
    total = e.sum(1, keepdim=True)
    log_p = z.gather(1, ids.clamp(min=0)) - m - total.log()
    loss = tau * tau * (q * (log_q - log_p)).sum(1)
    grad = (e / total).scatter_add_(1, ids.clamp(min=0), -q) * (tau * w)[:, None]
    if c["mode"] == "fused":
        loss = torch.where(w != 0, loss, 0.0)
    return loss, grad.to(s["logits"].dtype)


def _plain_ffn(c, s):
    dt = s["x"].dtype
    x, W1, W3, W2 = (s[n].float() for n in ("x", "W1", "W3", "W2"))
    g, u = x @ W1.T, x @ W3.T
    sig = 1.0 / (1.0 + (-g).exp())
    h = g * sig * u
    y = (h @ W2.T).to(dt)
    if c["mode"] == "forward":
        return y
    dy = s["dy"].float()
    dh = dy @ W2
    da = dh * u * sig * (1.0 + g * (1.0 - sig))
    db = dh * g * sig
    return y, (da @ W1 + db @ W3).to(dt), (da.T @ x).to(dt), (db.T @ x).to(dt), (dy.T @ h).to(dt)


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    T, size = case["T"], 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "ffn":
        H, F = case["H"], case["F"]
        if case["mode"] == "forward":
            return {"bytes": size * (2 * T * H + 3 * H * F), "flops": 6.0 * T * H * F}
        return {"bytes": size * (4 * T * H + 6 * H * F), "flops": 18.0 * T * H * F}
    V, K = case["V"], case["K"]
    if case["kind"] == "logprobs":
        return {"bytes": T * (V * size + 8 + 8 + 8 * K), "flops": 5.0 * T * V}
    return {"bytes": T * (2 * V * size + 8 * K + 8), "flops": 8.0 * T * V}


# ---------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "ffn":
        return _exact_ffn(case, s)
    outs = []
    rows = max(1, (1 << 27) // case["V"])                              # of 64-bit numbers in hand at a time
    for r in range(0, case["T"], rows):
        part = {n: v[r:r + rows] for n, v in s.items() if n != "case"}
        outs.append((_exact_logprobs if case["kind"] == "logprobs" else _exact_distill)(case, part))
    return tuple(None if o[0] is None else torch.cat(o) for o in zip(*outs))


def _exact_logprobs(case, s):
    logp = torch.log_softmax(s["logits"].double(), 1)
    p = logp.exp()
    entropy = -torch.xlogy(p, p).sum(1)
    tokens = s["tokens"]
    logprob = logp.gather(1, tokens.clamp(min=0)[:, None])[:, 0]
    logprob[tokens < 0] = 0.0
    return logprob, entropy, torch.sort(logp, dim=1, descending=True).values[:, :case["K"]].contiguous(), None


def _exact_distill(case, s):
    tau, ids = case["tau"], s["ids"].long()
    logp = torch.log_softmax(s["logits"].double() / tau, 1)
    q = torch.softmax((s["teacher"].double() / tau).masked_fill(ids < 0, -math.inf), 1)
    at = ids.masked_fill(ids < 0, 0)
    loss = tau ** 2 * (torch.xlogy(q, q) - q * logp.gather(1, at)).sum(1)
    target = torch.zeros_like(logp).scatter_add_(1, at, q)
    w = s["weights"].double()
    if case["mode"] == "fused":
        loss[w == 0] = 0.0
    return loss, tau * w[:, None] * (logp.exp() - target)


def _exact_ffn(case, s):
    x, W1, W3, W2 = (s[n].double() for n in ("x", "W1", "W3", "W2"))
    g, u = torch.mm(x, W1.t()), torch.mm(x, W3.t())
    silu = g * torch.sigmoid(g)
    y = torch.mm(silu * u, W2.t())
    if case["mode"] == "forward":
        return y
    dy = s["dy"].double()
    dh = torch.mm(dy, W2)
    s_ = torch.sigmoid(g)
    da, db = dh * u * (s_ + silu * (1 - s_)), dh * silu
    return y, torch.mm(da, W1) + torch.mm(db, W3), torch.mm(da.t(), x), torch.mm(db.t(), x), torch.mm(dy.t(), silu * u)
