"""What a teacher's temperature means in a repairing step, against the definition written from the original model's logits."""
import math

import pytest
import torch

from paper_2508_02322_amd import pipeline

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: U}


def step64(original, logits, targets, idx, g_lp, g_kl, T):
    """Log probability, divergence over the listed tokens alone, their gradients, and what the tolerances are made of, in float64."""
    n, vocab = logits.shape
    z = logits.double()
    lp, lp_T = torch.log_softmax(z, 1), torch.log_softmax(z / T, 1)
    at = idx.long()
    teacher = torch.log_softmax(original.double() / T, 1).gather(1, at)
    log_q = torch.log_softmax(original.double().gather(1, at) / T, 1)    # renormalised over the listed tokens, at T
    q = log_q.exp()
    apart = log_q - lp_T.gather(1, at)
    kl = (q * apart).sum(1)
    has = targets >= 0
    rows = torch.arange(n, device="cuda")
    to = targets.long().clamp(min=0)
    g1 = torch.where(has, g_lp.double(), 0.0)
    logprob = torch.where(has, lp[rows, to], 0.0)
    a = -lp.exp() * g1[:, None]
    a[rows, to] += g1
    b = lp_T.exp() * (g_kl.double() / T)[:, None]
    q_part = torch.zeros_like(b).scatter_(1, at, q * (g_kl.double() / T)[:, None])
    return dict(logprob=logprob, kl=kl, a=a, b=b - q_part, p_part=b, q_part=q_part, teacher=teacher, apart=apart, lp=lp, lp_T=lp_T, g1=g1)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T", [0.5, 1.0, 2.0, 3.0])
def test_renormalised_teacher_has_its_temperature_once(cam, T, dtype):
    """q = softmax(original / T) over the listed tokens, p = softmax(logits / T).

    Tolerances, u = 2^-24: a log probability is off by (4 |lp| + L + 8) u (L additions one after the other in a row's sum; the
    teacher's values carry that and two roundings more), so log q by e = twice that of the listed ones (itself and the norm), q by e
    relative.  The divergence: q's error times how far the two are apart, and p's.  The gradient: each part's relative error;
    two roundings to the type, each of a value no larger than all parts' magnitudes together."""
    n, vocab, k = 41, 5003, 24
    gen = torch.Generator(device="cuda").manual_seed(5)
    original = (3 * torch.randn((n, vocab), generator=gen, device="cuda")).to(dtype)
    logits = (original.float() + 0.7 * torch.randn((n, vocab), generator=gen, device="cuda")).to(dtype)
    targets = original.float().argmax(1).int()
    targets[::5] = -100
    teacher = pipeline.teacher_of(cam, original, k, T)
    g_lp = torch.full((n,), -0.5 / n, device="cuda")
    g_kl = torch.linspace(0.1, 1.0, n, device="cuda") * (T * T / n)
    out = pipeline.recovery_step(cam, logits, targets, teacher, g_lp, g_kl, tail=False)
    torch.cuda.synchronize()
    w = step64(original, logits, targets, teacher.idx, g_lp, g_kl, T)
    L = vocab / 512 + 40
    err = lambda lp: (4 * lp.abs() + L + 8) * U  # noqa: E731
    e = 2 * (err(w["teacher"]) + 2 * w["teacher"].abs() * U).amax(1)
    e_p = err(w["lp_T"].gather(1, teacher.idx.long())).amax(1)
    tol = e * (w["apart"].abs().amax(1) + 1) + e_p + U * w["kl"].abs()
    assert bool(((out.kl.double() - w["kl"]).abs() <= tol).all()), float(((out.kl.double() - w["kl"]).abs() / tol).max())
    assert bool(((out.logprob.double() - w["logprob"]).abs() <= err(w["logprob"])).all())
    size = w["a"].abs() + w["g1"].abs()[:, None] * w["lp"].exp() + w["p_part"].abs() + w["q_part"].abs()
    tol = (w["g1"].abs()[:, None] * w["lp"].exp() * (err(w["lp"]) + 4 * U) + w["p_part"].abs() * (err(w["lp_T"]) + 8 * U)
           + w["q_part"].abs() * (e[:, None] + 8 * U) + 2 * HALF[dtype] * size + 2.0 ** -126)
    off = (out.dlogits.double() - w["a"] - w["b"]).abs()
    assert bool((off <= tol).all()), float((off / tol).max())


@pytest.mark.parametrize("tail", [False, True])
def test_a_model_is_no_distance_from_itself(cam, tail):
    """At any temperature and in either form: the divergence is 0 to the error of the log probabilities, 2 (4 |lp| + L + 8) u."""
    gen = torch.Generator(device="cuda").manual_seed(6)
    logits = 3 * torch.randn((20, 3001), generator=gen, device="cuda")
    n = logits.shape[0]
    targets = torch.zeros(n, dtype=torch.int32, device="cuda")
    for T in (0.5, 1.0, 2.0):
        # of all tokens that the unlisted class leaves out, none: the renormalised student is the student
        kept = logits.clone()
        if not tail:
            kept.masked_fill_(~torch.zeros_like(kept, dtype=torch.bool).scatter_(1, logits.topk(40, 1).indices, True), -math.inf)
        teacher = pipeline.teacher_of(cam, kept, 40, T)
        out = pipeline.recovery_step(cam, kept, targets, teacher, torch.zeros(n, device="cuda"), torch.ones(n, device="cuda"), tail=tail)
        torch.cuda.synchronize()
        reach = float(teacher.logprob.abs().max())
        assert float(out.kl.abs().max()) < 4 * (4 * reach + 3001 / 512 + 48) * U
        assert float(out.dlogits.abs().max()) < 4 * (4 * reach + 3001 / 512 + 48) * U * max(1.0, 1 / T)


def test_renormalised_step_in_a_graph(cam):
    """Captured once at a temperature of its own and replayed after the logits and the teacher changed, in turn with eager calls."""
    n, vocab, T = 33, 2003, 2.0
    gen = torch.Generator(device="cuda").manual_seed(7)
    logits = torch.randn((n, vocab), generator=gen, device="cuda").to(torch.bfloat16)
    teacher = pipeline.teacher_of(cam, torch.randn((n, vocab), generator=gen, device="cuda").to(torch.bfloat16), 8, T)
    targets = torch.randint(0, vocab, (n,), generator=gen, device="cuda").int()
    g = torch.ones(n, device="cuda")

    def step():
        out = pipeline.recovery_step(cam, logits, targets, teacher, g, g, tail=False)
        return out.logprob, out.entropy, out.kl, out.dlogits
    step()
    torch.cuda.synchronize()
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        with torch.cuda.graph(graph, stream=stream):
            captured = step()
    for trial in range(4):
        if trial:
            logits.copy_(torch.randn(logits.shape, generator=gen, device="cuda"))
            teacher.logprob.copy_(-3 * torch.rand(teacher.logprob.shape, generator=gen, device="cuda"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        kept = [t.clone() for t in captured]
        for a, b in zip(kept, step()):
            assert torch.equal(a, b)
        torch.cuda.synchronize()
