"""The operators that repair and judge a pruned model, as measurable cases.

A program that has pruned a model with this package asks three things of the GPU beyond the layer passes:

  logprobs   what the model says of given tokens: their log probabilities, the entropy of every position and the most
             likely alternatives, with the gradient (perplexity, serving, the teacher's side of a distillation)
  distill    how far the pruned model's distribution is from the original's, of which only the most likely tokens of
             every position are kept, with the gradient
  gated      the gated block silu(X W_gate^T) * (X W_up^T) of the micro-experts that were kept, with its gradients

Vocabularies are those of the language models whose layer shapes the package has (32000, 102400, 151936) or of the same
range; layer sizes are the package's own (``inputs.CONFIGS``) or of the same ranges.
"""
from __future__ import annotations

import math

import torch

own = False

_handle = None


def _camera():
    """The library context; a program makes one and keeps it."""
    global _handle
    if _handle is None:
        from paper_2508_02322_amd import binding
        _handle = binding.Camera(device=0)
    return _handle


# ---- the cases ---------------------------------------------------------------------------------------------------
def _logits(op, direction, n, vocab, top_k, dtype="bf16", temperature=1.0, masked=0.0, ignored=0.0, pad=0, tail=False, **kw):
    return dict(op=op, direction=direction, n=n, vocab=vocab, top_k=top_k, dtype=dtype, temperature=temperature,
                masked=masked, ignored=ignored, pad=pad, tail=tail, **kw)


def _gated(direction, n, d_model, d_ff, dtype="bf16", **kw):
    return dict(op="gated", direction=direction, n=n, d_model=d_model, d_ff=d_ff, dtype=dtype, **kw)


def listed():
    return [
        # one position of one sequence being decoded, with the alternatives that an answer shows
        _logits("logprobs", "forward", 1, 151936, 20, name="logprobs-token"),
        # a decoding batch whose grammar rules half of the vocabulary out
        _logits("logprobs", "forward", 64, 102400, 8, temperature=0.7, masked=0.5, name="logprobs-batch-64-masked"),
        # the original model's pass over a chunk of the tokens it teaches: its 64 most likely tokens at every position
        _logits("logprobs", "forward", 4096, 151936, 64, name="logprobs-teacher-4096"),
        # perplexity of a float32 model, a vocabulary of odd size and rows that lie apart
        _logits("logprobs", "forward", 2047, 32003, 0, dtype="f32", pad=5, name="logprobs-perplexity-f32"),
        # the gradient of a fine-tuning step with an entropy bonus; a quarter of the positions is prompt and has no target
        _logits("logprobs", "backward", 2048, 102400, 0, ignored=0.25, name="logprobs-backward-2048"),
        # the distillation loss of a chunk, the unlisted tokens as one class
        _logits("distill", "forward", 4096, 151936, 64, tail=True, name="distill-4096"),
        # its gradient, and that of a smaller chunk over the listed tokens alone
        _logits("distill", "backward", 2048, 151936, 64, tail=True, name="distill-backward-2048"),
        # a float32 step, loss and gradient, of few positions at a raised temperature
        _logits("distill", "step", 65, 50021, 100, dtype="f32", temperature=2.0, pad=3, name="distill-step-f32"),
        # one token through one expert of the Qwen2 shape
        _gated("forward", 1, 3584, 2560, name="gated-token"),
        # a training step of the Qwen2 shape's shared expert
        _gated("step", 8192, 3584, 20480, name="gated-step-8192"),
        # a training step of what pruning left of an expert of the DeepSeek shape: an odd number of micro-experts
        _gated("step", 1021, 2048, 843, name="gated-step-compact"),
        # a float32 block of odd sizes
        _gated("step", 1499, 772, 1033, dtype="f32", name="gated-step-ragged-f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["logprobs", "distill", "gated"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "gated":
        n, d_ff = _log_int(rng, 1, 4096), _log_int(rng, 16, 16384)
        d_model = 8 * _log_int(rng, 16, 512) if dtype == "bf16" else 4 * _log_int(rng, 16, 512)
        if dtype == "f32":
            n, d_ff = min(n, 2048), min(d_ff, 4096)
        return _gated(rng.choice(["forward", "step"]), n, d_model, d_ff, dtype)
    vocab = _log_int(rng, 1000, 200000)
    n = min(_log_int(rng, 1, 4096), (300 if dtype == "bf16" else 150) * 10**6 // vocab)
    temperature = rng.choice([1.0, 0.7, 2.0])
    pad = rng.choice([0, 0, 1, 8, 37])
    if op == "logprobs":
        direction = rng.choice(["forward", "forward", "backward"])
        return _logits(op, direction, n, vocab, rng.choice([0, 1, 5, 20, 64, 256]), dtype, temperature,
                       rng.choice([0.0, 0.0, 0.5]), rng.choice([0.0, 0.3]), pad)
    return _logits(op, rng.choice(["forward", "backward", "step"]), n, vocab, _log_int(rng, 1, 256), dtype, temperature,
                   0.0, rng.choice([0.0, 0.3]), pad, rng.choice([True, False]))


# ---- what a program has in hand ----------------------------------------------------------------------------------
_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _rows(values, pad, dtype):
    """`values` rounded to dtype in rows that lie `pad` elements further apart than they are long."""
    n, vocab = values.shape
    out = torch.empty((n, vocab + pad), dtype=dtype, device=values.device)[:, :vocab]
    return out.copy_(values)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)

    dtype = _TYPES[case["dtype"]]
    s = dict(case)
    n = case["n"]
    if case["op"] == "gated":
        d, f = case["d_model"], case["d_ff"]
        s.update(X=normal(n, d).to(dtype), W_gate=(0.02 * normal(f, d)).to(dtype), W_up=(0.02 * normal(f, d)).to(dtype))
        if case["direction"] == "step":
            s["dH"] = (0.001 * normal(n, f)).to(dtype)
        return s
    vocab, k, temperature = case["vocab"], case["top_k"], case["temperature"]
    # a trained model's logits: a normal bulk, and a few tokens that stand out by an amount of the position's own
    z = 2.0 * normal(n, vocab)
    apart = vocab // 24
    stand_out = torch.arange(24, device="cuda") * apart + torch.randint(0, apart, (n, 24), generator=g, device="cuda")
    z.scatter_(1, stand_out, 8.0 + 3.0 * normal(n, 24).abs())
    if case["masked"] > 0:  # the same tokens at every position; a sixteenth of the vocabulary is always left
        out = torch.rand(vocab, generator=g, device="cuda") < case["masked"]
        out[::16] = False
        z[:, out] = -math.inf
    ignored = torch.rand(n, generator=g, device="cuda") < case["ignored"]
    if case["op"] == "logprobs":
        s["logits"] = _rows(z, case["pad"], dtype)
        pick = torch.rand(n, 1, generator=g, device="cuda") < 0.7  # mostly a likely token, else any
        any_token = torch.randint(0, (vocab + 15) // 16, (n, 1), generator=g, device="cuda") * 16
        likely = s["logits"].argmax(1, keepdim=True)
        s["targets"] = torch.where(ignored[:, None], -100, torch.where(pick, likely, any_token))[:, 0].to(torch.int32)
        if case["direction"] == "backward":
            w = 1.0 / n
            s["grad_logprob"] = (-w * torch.rand(n, generator=g, device="cuda")).masked_fill(ignored, 0.0)
            s["grad_entropy"] = torch.full((n,), -0.01 * w, device="cuda").masked_fill(ignored, 0.0)
            # what the forward call left
            zs = s["logits"].double()
            m = zs.amax(1, keepdim=True)
            d = (zs - m) / temperature
            log_sum = d.exp().sum(1, keepdim=True).log()
            lp = d - log_sum
            s["stats"] = torch.cat([m, log_sum], 1).float()
            s["entropy"] = -(lp.exp() * lp.clamp(min=-1e4)).sum(1).float()
        return s
    # the original model's distribution at its k most likely tokens; the pruned model's logits are near its own
    t = z / temperature
    top = t.topk(k, dim=1)
    s["teacher_idx"] = top.indices.to(torch.int32)
    s["teacher_logprob"] = (top.values - t.logsumexp(1, keepdim=True)).float()
    few = torch.rand(n, generator=g, device="cuda") < 0.02  # positions for which fewer tokens were kept
    if k > 2:
        s["teacher_idx"][few, k // 2:] = -1
    s["logits"] = _rows(z + 0.5 * normal(n, vocab), case["pad"], dtype)
    if case["direction"] != "forward":
        s["grad_loss"] = (torch.rand(n, generator=g, device="cuda") / n).masked_fill(ignored, 0.0)
    if case["direction"] == "backward":  # what the forward call left
        s["stats"] = _distill_rows(s, torch.float64)[1].float()
    return s


# ---- the plain forms ---------------------------------------------------------------------------------------------
def _plain_logprobs(s):
    z, targets, k, temperature = s["logits"].float(), s["targets"].long(), s["top_k"], s["temperature"]
    n, vocab = z.shape
    m = z.amax(1, keepdim=True)
    d = (z - m) / temperature
    e = d.exp()
    total = e.sum(1, keepdim=True)
    log_sum = total.log()
    entropy = log_sum[:, 0] - (e * d.clamp(min=-1e4)).sum(1) / total[:, 0]
    valid = (targets >= 0) & (targets < vocab)
    at = targets.clamp(0, vocab - 1)[:, None]
    logprob = torch.where(valid, (d.gather(1, at) - log_sum)[:, 0], 0.0)
    out = dict(logprob=logprob, entropy=entropy, stats=torch.cat([m, log_sum], 1))
    if k:
        # one whole number a token that orders as (logit, lowest index first) does
        bits = (z + 0.0).view(torch.int32).long()
        order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits)
        key = (order << 32) + torch.arange(vocab - 1, -1, -1, device=z.device)
        idx = vocab - 1 - (key.topk(k, dim=1).values & 0xFFFFFFFF)
        top = d.gather(1, idx)
        out["top_idx"] = torch.where(top == -math.inf, -1, idx).to(torch.int32)
        out["top_logprob"] = top - log_sum
    return out


def _plain_logprobs_backward(s):
    z, targets, temperature = s["logits"].float(), s["targets"].long(), s["temperature"]
    n, vocab = z.shape
    valid = (targets >= 0) & (targets < vocab)
    a = torch.where(valid, s["grad_logprob"], 0.0)[:, None] / temperature
    b = s["grad_entropy"][:, None] / temperature
    lp = ((z - s["stats"][:, :1]) / temperature - s["stats"][:, 1:]).clamp(min=-1e4)
    grad = -lp.exp() * (a + b * (lp + s["entropy"][:, None]))
    grad.scatter_add_(1, targets.clamp(0, vocab - 1)[:, None], a)
    return grad.to(s["logits"].dtype)


def _distill_rows(s, dtype):
    """(loss, what the gradient takes from the loss); the vocabulary's sums in `dtype`."""
    z, t, temperature, tail = s["logits"].to(dtype), s["teacher_logprob"].double(), s["temperature"], s["tail"]
    n, vocab = z.shape
    idx = s["teacher_idx"].long()
    valid = (idx >= 0) & (idx < vocab)
    at = idx.clamp(0, vocab - 1)
    m = z.amax(1, keepdim=True)
    e = ((z - m) / temperature).exp()
    log_sum = e.sum(1, keepdim=True).log().double()
    log_p = (z.gather(1, at).double() - m.double()) / temperature - log_sum
    t = t.masked_fill(~valid, -math.inf)
    norm = torch.zeros_like(log_sum) if tail else (t / temperature).logsumexp(1, keepdim=True)
    log_q = t if tail else t / temperature - norm
    q = log_q.exp()
    loss = (q * (log_q - log_p).masked_fill(~valid, 0.0)).nan_to_num(0.0).sum(1)
    if tail:
        rest = e.scatter(1, torch.where(valid, at, at[:, :1]), 0.0).sum(1, keepdim=True).double()
        log_rest = rest.log() - log_sum
        left = (1.0 - q.sum(1, keepdim=True)).clamp(min=0.0)
        loss = loss + torch.where(left > 0, left * (left.log() - log_rest), 0.0)[:, 0]
        mass = q.sum(1, keepdim=True) + left
        log_ratio = left.log() - log_rest
    else:
        mass = q.sum(1, keepdim=True)
        log_ratio = torch.full_like(mass, -math.inf)
    return loss, torch.cat([m.double(), log_sum, norm, mass, log_ratio], 1)


def _plain_distill(s):
    loss, stats = _distill_rows(s, torch.float32)
    return dict(loss=loss.float(), stats=stats.float())


def _plain_distill_backward(s, stats):
    z, temperature = s["logits"].float(), s["temperature"]
    n, vocab = z.shape
    idx = s["teacher_idx"].long()
    valid = (idx >= 0) & (idx < vocab)
    at = idx.clamp(0, vocab - 1)
    m, log_sum, norm, mass, log_ratio = (stats[:, i:i + 1] for i in range(5))
    g = s["grad_loss"][:, None] / temperature
    p = ((z - m) / temperature - log_sum).exp()
    t = s["teacher_logprob"] if s["tail"] else s["teacher_logprob"] / temperature - norm
    q = t.exp().masked_fill(~valid, 0.0)
    here = (mass * p.gather(1, at) - q).masked_fill(~valid, 0.0)
    grad = torch.cat([p * (mass - log_ratio.exp()), torch.zeros_like(g)], 1)  # a column for the entries that name no token
    grad.scatter_(1, torch.where(valid, at, vocab), here)
    return (g * grad[:, :vocab]).to(s["logits"].dtype)


def _plain_gated(s):
    x, w_gate, w_up = s["X"].float(), s["W_gate"].float(), s["W_up"].float()
    gate, up = x @ w_gate.t(), x @ w_up.t()
    sig = 1.0 / (1.0 + (-gate).exp())
    out = dict(H=(gate * sig * up).to(s["X"].dtype))
    if s["direction"] == "step":
        dh = s["dH"].float()
        d_up = dh * gate * sig
        d_gate = dh * up * (sig * (1.0 + gate * (1.0 - sig)))
        out.update(dX=(d_gate @ w_gate + d_up @ w_up).to(s["X"].dtype),
                   dW_gate=(d_gate.t() @ x).to(s["X"].dtype), dW_up=(d_up.t() @ x).to(s["X"].dtype))
    return out


# ---- the framework's calls ---------------------------------------------------------------------------------------
def _own(s):
    cam = _camera()
    if s["op"] == "gated":
        if s["direction"] == "forward":
            return dict(H=cam.gated_ffn(s["X"], s["W_gate"], s["W_up"]))
        H, pre = cam.gated_ffn(s["X"], s["W_gate"], s["W_up"], want_pre=True)
        dX, dW_gate, dW_up = cam.gated_ffn_backward(s["X"], s["W_gate"], s["W_up"], s["dH"], pre=pre)
        return dict(H=H, dX=dX, dW_gate=dW_gate, dW_up=dW_up)
    temperature = s["temperature"]
    if s["op"] == "logprobs":
        if s["direction"] == "backward":
            return cam.token_logprobs_backward(s["logits"], s["targets"], s["stats"], s["grad_logprob"],
                                               entropy=s["entropy"], grad_entropy=s["grad_entropy"], temperature=temperature)
        return cam.token_logprobs(s["logits"], s["targets"], top_k=s["top_k"], temperature=temperature)
    teacher = s["teacher_idx"], s["teacher_logprob"]
    if s["direction"] == "backward":
        return cam.distill_topk_backward(s["logits"], *teacher, s["stats"], s["grad_loss"], temperature=temperature, tail=s["tail"])
    out = cam.distill_topk(s["logits"], *teacher, temperature=temperature, tail=s["tail"])
    if s["direction"] == "step":
        out["dlogits"] = cam.distill_topk_backward(s["logits"], *teacher, out["stats"], s["grad_loss"], temperature=temperature, tail=s["tail"])
    return out


def run(state):
    if own:
        return _own(state)
    if state["op"] == "gated":
        return _plain_gated(state)
    if state["op"] == "logprobs":
        return _plain_logprobs_backward(state) if state["direction"] == "backward" else _plain_logprobs(state)
    if state["direction"] == "backward":
        return _plain_distill_backward(state, state["stats"])
    out = _plain_distill(state)
    if state["direction"] == "step":
        out["dlogits"] = _plain_distill_backward(state, out["stats"])
    return out


# ---- what a pass cannot do without -------------------------------------------------------------------------------
def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    n = case["n"]
    if case["op"] == "gated":
        d, f = case["d_model"], case["d_ff"]
        once = n * d + 2 * f * d  # X and both matrices
        if case["direction"] == "forward":
            return {"bytes": size * (once + n * f), "flops": 4 * n * d * f}
        return {"bytes": size * (2 * once + 2 * n * f), "flops": 12 * n * d * f}  # and H, dH and the three gradients
    vocab, k = case["vocab"], case["top_k"]
    if case["op"] == "logprobs":
        if case["direction"] == "backward":  # the rows that have a gradient, and every row of it
            return {"bytes": int(size * n * vocab * (2 - case["ignored"])) + 24 * n, "flops": 6 * n * vocab}
        return {"bytes": size * n * vocab + 20 * n + 8 * n * k, "flops": 6 * n * vocab}
    teacher = 8 * n * k
    if case["direction"] == "forward":
        return {"bytes": size * n * vocab + teacher + 24 * n, "flops": 4 * n * vocab}
    read = 1.0 - case["ignored"] if case["direction"] == "backward" else 1.0
    return {"bytes": int(size * n * vocab * (1 + read)) + teacher + 28 * n, "flops": (5 if read < 1 else 8) * n * vocab}


# ---- the same from the definitions, in 64 bits -------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "gated":
        X, Wg, Wu = (s[x].double() for x in ("X", "W_gate", "W_up"))
        G, U = torch.mm(X, Wg.T), torch.mm(X, Wu.T)
        sg = torch.sigmoid(G)
        if case["direction"] == "forward":
            return {"H": G * sg * U}
        dH = s["dH"].double()
        dU = dH * (G * sg)
        dG = dH * U * (sg + G * sg * (1 - sg))
        return {"H": G * sg * U, "dX": torch.mm(dG, Wg) + torch.mm(dU, Wu), "dW_gate": torch.mm(dG.T, X), "dW_up": torch.mm(dU.T, X)}
    scaled = s["logits"].double() / case["temperature"]
    logp = torch.log_softmax(scaled, dim=1)
    vocab = case["vocab"]
    m = s["logits"].double().max(1).values
    lse = torch.logsumexp(scaled, dim=1)
    rows = torch.arange(case["n"], device="cuda")
    if case["op"] == "logprobs":
        H = torch.special.entr(logp.exp()).sum(1)
        target = s["targets"].long()
        has = (target >= 0) & (target < vocab)
        if case["direction"] == "backward":
            # d logprob[t] / dz = (1[t] - p) / T and d entropy / dz = -p (log p + H) / T
            p = logp.exp()
            out = torch.where(p > 0, -p * (logp + H[:, None]), 0.0) * s["grad_entropy"].double()[:, None]
            glp = torch.where(has, s["grad_logprob"].double(), 0.0)
            out -= p * glp[:, None]
            out[rows[has], target[has]] += glp[has]
            return out / case["temperature"]
        lp = torch.where(has, logp[rows, target.clamp(0, vocab - 1)], 0.0)
        out = {"logprob": lp, "entropy": H, "stats": torch.stack([m, lse - m / case["temperature"]], 1)}
        if case["top_k"]:  # equal values keep their order
            value, place = torch.sort(s["logits"].double(), dim=1, descending=True, stable=True)
            place = place[:, :case["top_k"]]
            out["top_idx"] = place.masked_fill(value[:, :case["top_k"]] == -math.inf, -1).int()
            out["top_logprob"] = logp.gather(1, place)
        return out
    # distillation: the teacher's distribution q over its listed tokens (and one class for all others with `tail`)
    idx = s["teacher_idx"].long()
    valid = (idx >= 0) & (idx < vocab)
    t = s["teacher_logprob"].double()
    q = torch.where(valid, t.exp() if case["tail"] else torch.softmax((t / case["temperature"]).masked_fill(~valid, -math.inf), 1), 0.0)
    dense = torch.zeros(case["n"], vocab + 1, dtype=torch.float64, device="cuda")
    dense.scatter_(1, torch.where(valid, idx, vocab), q)
    inside = torch.zeros(case["n"], vocab + 1, dtype=torch.bool, device="cuda")
    inside.scatter_(1, torch.where(valid, idx, vocab), True)
    dense, inside = dense[:, :vocab], inside[:, :vocab]
    p = logp.exp()
    loss = torch.where(dense > 0, dense * (dense.log() - logp), 0.0).sum(1)
    mass, per_unlisted = q.sum(1), torch.zeros(case["n"], dtype=torch.float64, device="cuda")  # an unlisted token's p has mass - per_unlisted
    if case["tail"]:
        q_rest = (1 - q.sum(1)).clamp(min=0)
        p_rest = torch.where(inside, 0.0, p).sum(1)
        loss = loss + torch.special.xlogy(q_rest, q_rest) - torch.special.xlogy(q_rest, p_rest)
        mass, per_unlisted = mass + q_rest, q_rest / p_rest
    norm = torch.zeros_like(mass) if case["tail"] else torch.logsumexp((t / case["temperature"]).masked_fill(~valid, -math.inf), 1)
    out = {"loss": loss, "stats": torch.stack([m, lse - m / case["temperature"], norm, mass, per_unlisted.log()], 1)}
    if case["direction"] == "forward":
        return out
    grad = mass[:, None] * p - dense - torch.where(inside, 0.0, p * per_unlisted[:, None])
    grad *= s["grad_loss"].double()[:, None] / case["temperature"]
    if case["direction"] == "backward":
        return grad
    out["dlogits"] = grad
    return out
