"""Values at the ends of what logits can be: NaN and +Inf are not hidden, and what the definition makes finite is finite and right."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
# rows in parts, whole in long workgroups, whole in short ones
SHAPES = [(12, 9001), (1100, 17001), (1030, 3001)]


def rows_of(n, vocab, dtype, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (3 * torch.randn((n, vocab), generator=gen, device="cuda")).to(TYPES[dtype])


def spoil(z, idx):
    """Rows 1 to 9: NaN at the target, at a listed token, elsewhere, at the last token; all NaN; NaN and ruled out tokens only; +Inf;
    +Inf at a listed token; NaN and +Inf."""
    nan, vocab = float("nan"), z.shape[1]
    z = z.clone()
    z[1, 0] = nan
    z[2, idx[2, 3].long()] = nan
    z[3, 777] = nan
    z[4, vocab - 1] = nan
    z[5] = nan
    z[6] = -math.inf
    z[6, vocab // 2] = nan
    z[7, 2222] = math.inf
    z[8, idx[8, 0].long()] = math.inf
    z[9, 5] = nan
    z[9, 6] = math.inf
    return z


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,vocab", SHAPES)
def test_log_probabilities_show_nan(cam, n, vocab, dtype):
    z = rows_of(n, vocab, dtype, 1)
    targets = torch.zeros(n, dtype=torch.int32, device="cuda")
    top = cam.token_logprobs(z, targets, top_k=10)
    bad = spoil(z, top["top_idx"])
    out, plain = cam.token_logprobs(bad, targets, top_k=10), cam.token_logprobs(bad, targets)
    ones = torch.ones(n, device="cuda")
    grad = cam.token_logprobs_backward(bad, targets, out["stats"], ones, out["entropy"], ones)
    want = cam.token_logprobs_backward(z, targets, top["stats"], ones, top["entropy"], ones)
    only = cam.token_logprobs_backward(bad, targets, out["stats"], ones)
    torch.cuda.synchronize()
    spoiled = torch.zeros(n, dtype=torch.bool, device="cuda")
    spoiled[1:10] = True
    for o in (out, plain):
        for key in ("logprob", "entropy"):
            assert torch.equal(o[key].isnan(), spoiled), key
        assert torch.equal(o["stats"][:, 1].isnan(), spoiled)
    for g in (grad, only):
        assert bool(g[spoiled].isnan().all()) and not bool(g[~spoiled].isnan().any())
    for key in top:
        assert torch.equal(out[key][~spoiled], top[key][~spoiled]), key
    assert torch.equal(grad[~spoiled], want[~spoiled])
    assert bool(((out["top_idx"] >= -1) & (out["top_idx"] < vocab)).all())
    # a row without gradient stays without one
    none = cam.token_logprobs_backward(bad, targets, out["stats"], torch.zeros(n, device="cuda"))
    torch.cuda.synchronize()
    assert not bool(none.any())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("n,vocab", SHAPES)
def test_distillation_shows_nan(cam, n, vocab, tail, dtype):
    z = rows_of(n, vocab, dtype, 2)
    top = cam.token_logprobs(rows_of(n, vocab, dtype, 3), top_k=10)
    teacher = top["top_idx"], top["top_logprob"]
    bad = spoil(z, top["top_idx"])
    ones = torch.ones(n, device="cuda")
    good, out = cam.distill_topk(z, *teacher, tail=tail), cam.distill_topk(bad, *teacher, tail=tail)
    want = cam.distill_topk_backward(z, *teacher, good["stats"], ones, tail=tail)
    got = cam.distill_topk_backward(bad, *teacher, out["stats"], ones, tail=tail)
    torch.cuda.synchronize()
    spoiled = torch.zeros(n, dtype=torch.bool, device="cuda")
    spoiled[1:10] = True
    assert torch.equal(out["loss"].isnan(), spoiled)
    assert bool(got[spoiled].isnan().all()) and not bool(got[~spoiled].isnan().any())
    for key in good:
        assert torch.equal(out[key][~spoiled], good[key][~spoiled]), key
    assert torch.equal(got[~spoiled], want[~spoiled])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1.0, 0.5, 2.0])
@pytest.mark.parametrize("n,vocab", SHAPES)
def test_unlisted_class_next_to_impossible(cam, n, vocab, T, dtype):
    """The student keeps the listed tokens and gives all others a mask's value (rows: -50, -200, -1e3, -1e4, -1e9, the type's lowest,
    the last two with a few tokens less ruled out), the teacher has a quarter of its probability there.  The unlisted tokens' gradient is
    p - q_r softmax(unlisted): about -1 / (4 unlisted) each, whatever the mask.

    Tolerance, relative to the two terms: L additions in each sum, 4 u per unit of the exponents that are taken, d from the class's largest
    logit, w = log q_r - log sum exp d; where the class is within e^-256 its ratio to q_r goes through float32 as a logarithm, 4 u each unit."""
    k = 8
    z = rows_of(n, vocab, dtype, 4)
    gen = torch.Generator(device="cuda").manual_seed(5)
    idx = torch.stack([torch.randperm(vocab, generator=gen, device="cuda")[:k] for _ in range(8)]).repeat(-(-n // 8), 1)[:n].int()
    lowest = torch.finfo(TYPES[dtype]).min
    masks = [-50.0, -200.0, -1e3, -1e4, -1e9, lowest, -1e9, lowest]
    listed = torch.zeros((n, vocab), dtype=torch.bool, device="cuda").scatter_(1, idx.long(), True)
    some = torch.rand(vocab, generator=gen, device="cuda") < 0.3
    noise = 2 * torch.rand((n, vocab), generator=gen, device="cuda")
    for i, value in enumerate(masks):
        fill = torch.full((vocab,), value, device="cuda")
        if value > -1e5:
            fill = fill - noise[i]                         # not all alike where the type can tell
        elif i >= 6:
            fill[some] = value / 2
        z[i::8] = torch.where(listed[i::8], z[i::8], fill.to(TYPES[dtype]))
    share = torch.rand((n, k), generator=gen, device="cuda") + 0.1
    val = (0.75 * share / share.sum(1, keepdim=True)).log()
    g = torch.linspace(0.5, 2.0, n, device="cuda")
    out = cam.distill_topk(z, idx, val, temperature=T, tail=True)
    got = cam.distill_topk_backward(z, idx, val, out["stats"], g, temperature=T, tail=True)
    added = cam.distill_topk_backward(z, idx, val, out["stats"], g, temperature=T, tail=True, dlogits=torch.zeros_like(z), accumulate=True)
    torch.cuda.synchronize()

    d = z.double().masked_fill(listed, -math.inf)
    m_r = d.amax(1, keepdim=True)
    d = (d - m_r) / T
    log_s = torch.logsumexp(d, 1, keepdim=True)
    here = z.double().gather(1, idx.long()) / T
    log_sum = torch.logaddexp(torch.logsumexp(here, 1, keepdim=True), m_r / T + log_s)
    q = val.double().exp()
    q_r = 1 - q.sum(1, keepdim=True)
    log_rest = m_r / T + log_s - log_sum
    loss = (q * (val.double() - (here - log_sum))).sum(1) + (q_r * (q_r.log() - log_rest))[:, 0]
    L = vocab / 128 + 40
    fits = loss < 3e38
    assert bool(((out["loss"].double() - loss).abs()[fits] <= ((L + 32) * U + 4 * U * loss.abs())[fits]).all())
    within = (d - log_s).exp()                              # of the class; 0 at the listed tokens
    unlisted = within * log_rest.exp() - q_r * within
    p = torch.zeros_like(unlisted).scatter_(1, idx.long(), (here - log_sum).exp())
    dense = torch.zeros_like(unlisted).scatter_(1, idx.long(), q)
    want = torch.where(listed, p - dense, unlisted) * (g.double() / T)[:, None]
    w = (q_r.log() - log_s).abs()
    log_ratio = q_r.log() - log_rest
    steps = L + 16 + 4 * d.clamp(min=-1e4).abs() + 4 * w + torch.where(log_ratio.abs() < 300, 8 * log_ratio.abs(), 0.0)
    small = (within * log_rest.exp() + q_r * within) * steps * U
    tol = torch.where(listed, (p + dense) * (4 * 40 + L + 16) * U, small) * (g.double() / T)[:, None]
    half = torch.finfo(TYPES[dtype]).eps / 2
    for name, x in (("alone", got), ("added", added)):
        off = (x.double() - want).abs()
        bound = tol + half * (want.abs() + tol) + 2.0 ** -126
        assert bool(torch.isfinite(x).all()), name
        assert bool((off <= bound).all()), (name, float((off / bound).max()), int((off / bound).amax(1).argmax()) % 8)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("value", [-1e4, -1e9, "lowest", -math.inf])
@pytest.mark.parametrize("left,k", [(1, 4), (5, 20), (30, 64), (60, 64)])
@pytest.mark.parametrize("n,vocab", SHAPES)
def test_both_models_masked_alike(cam, n, vocab, left, k, value, dtype):
    """A mask leaves the same few tokens to both models, fewer than the list is long: nothing is left for the unlisted class but the
    rounding of the teacher's log probabilities, and the divergence is that of the few tokens, whatever number the mask is.

    Tolerance: the teacher's and the student's log probabilities are off by (4 |lp| + L + 8) u each, L = left additions of numbers
    that are not 0 and 4 levels of the join."""
    mask = torch.finfo(TYPES[dtype]).min if value == "lowest" else value
    original, z = rows_of(n, vocab, dtype, 7), rows_of(n, vocab, dtype, 8)
    out = torch.ones(vocab, dtype=torch.bool, device="cuda")
    out[torch.randperm(vocab, generator=torch.Generator(device="cuda").manual_seed(9), device="cuda")[:left]] = False
    original[:, out] = mask
    z[:, out] = mask
    g = torch.ones(n, device="cuda")
    for T in (1.0, 2.0):
        top = cam.token_logprobs(original, top_k=k, temperature=T)
        teacher = top["top_idx"], top["top_logprob"]
        kd = cam.distill_topk(z, *teacher, temperature=T, tail=True)
        got = cam.distill_topk_backward(z, *teacher, kd["stats"], g, temperature=T, tail=True)
        torch.cuda.synchronize()
        lq, lp = (torch.log_softmax(x[:, ~out].double() / T, 1) for x in (original, z))
        off = lambda t: (4 * t.abs() + left + 12) * U  # noqa: E731
        kl = (lq.exp() * (lq - lp)).sum(1)
        tol = (lq.exp() * (off(lq) * (1 + (lq - lp).abs()) + off(lp))).sum(1) + U * kl.abs() + 2.0 ** -20
        assert bool(((kd["loss"].double() - kl).abs() <= tol).all()), (T, float((kd["loss"].double() - kl).abs().max()))
        want = torch.zeros((n, vocab), dtype=torch.float64, device="cuda")
        want[:, ~out] = (lp.exp() - lq.exp()) / T
        size = torch.zeros_like(want)
        size[:, ~out] = (lp.exp() * off(lp) + lq.exp() * off(lq) + 8 * U) / T
        half = torch.finfo(TYPES[dtype]).eps / 2
        # q_r is at most 2^-20, over the unlisted tokens, where it is not told from rounding
        bound = size + half * (want.abs() + size) + 2.0 ** -20 / T
        assert bool(((got.double() - want).abs() <= bound).all()), float((got.double() - want).abs().max())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [3e38, 1e30, 1e-30, 5e-39])
@pytest.mark.parametrize("n,vocab", SHAPES)
def test_temperatures_at_the_ends(cam, n, vocab, T, dtype):
    """All tokens that are left alike, or the largest alone; ruled out ones stay so.  log of up to 17001 terms of 1: (L + 8) u off,
    16 u for a value below 16, and the same for the distance from the largest's difference, 0."""
    z = rows_of(n, vocab, dtype, 6)
    z[:, 7::3] = -math.inf
    z[:, 100] = 40.0
    left = (z[0] != -math.inf).sum().double()
    targets = torch.full((n,), 100, dtype=torch.int32, device="cuda")
    idx = torch.tensor([[100, 0, 1]], dtype=torch.int32, device="cuda").repeat(n, 1)
    val = torch.full((n, 3), -math.log(4.0), device="cuda")
    out = cam.token_logprobs(z, targets, top_k=3, temperature=T)
    g = torch.ones(n, device="cuda") * min(T, 1.0)                     # the gradient is 1 / T long
    grad = cam.token_logprobs_backward(z, targets, out["stats"], g, temperature=T)
    kd = [cam.distill_topk(z, idx, val, temperature=T, tail=tail) for tail in (False, True)]
    kd_grad = [cam.distill_topk_backward(z, idx, val, o["stats"], g, temperature=T, tail=tail) for o, tail in zip(kd, (False, True))]
    torch.cuda.synchronize()
    want = -math.log(left) if T > 1 else 0.0
    tol = (vocab / 128 + 40 + 8 + 16) * U * 2
    assert float((out["logprob"].double() - want).abs().max()) <= tol and float((out["entropy"].double() + want).abs().max()) <= 16 * tol
    assert bool((out["top_idx"][:, 0] == 100).all())
    for x in (grad, *kd_grad):
        assert bool(torch.isfinite(x).all()) and not bool(x[z == -math.inf].any())
    if T > 1:
        assert float((kd[0]["loss"].double() - (math.log(left) - math.log(3.0))).abs().max()) <= 2 * tol
        assert float((kd[1]["loss"].double() - (math.log(left) - math.log(4.0) - 0.25 * math.log(left - 3.0))).abs().max()) <= 2 * tol


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("offset", [0.0, -10.0, -20.0, 100.0, 1e4, -1e6, 1e7])
@pytest.mark.parametrize("n,vocab", SHAPES)
def test_renormalised_teacher_far_from_zero(cam, n, vocab, offset, dtype):
    """The teacher's values shifted by a constant (whole numbers, so that the shift is exact) are the same distribution: the same loss
    and gradient.  q_j is off by 4 u per unit of its exponent, at most 36 here, and k / 64 + 6 additions and 16 u for exp and the norm."""
    k, T = 100, 0.5
    z = rows_of(n, vocab, dtype, 10)
    gen = torch.Generator(device="cuda").manual_seed(11)
    idx = torch.stack([torch.randperm(vocab, generator=gen, device="cuda")[:k] for _ in range(8)]).repeat(-(-n // 8), 1)[:n].int()
    value = torch.randint(-9, 10, (n, k), generator=gen, device="cuda").float()
    g = torch.linspace(0.5, 2.0, n, device="cuda")
    out = cam.distill_topk(z, idx, value + offset, temperature=T)
    got = cam.distill_topk_backward(z, idx, value + offset, out["stats"], g, temperature=T)
    torch.cuda.synchronize()
    log_q = torch.log_softmax(value.double() / T, 1)
    q = log_q.exp()
    lp = torch.log_softmax(z.double() / T, 1)
    here = lp.gather(1, idx.long())
    loss = (q * (log_q - here)).sum(1)
    L = vocab / 128 + 40
    assert bool(((out["loss"].double() - loss).abs() <= (4 * here.abs().amax(1) + L + 16) * U + U * loss.abs()).all())
    dense = torch.zeros_like(lp).scatter_(1, idx.long(), q)
    want = (lp.exp() - dense) * (g.double() / T)[:, None]
    tol = (lp.exp() * (4 * lp.abs() + L + 16) * U + dense * (4 * 36 + 2 + 6 + 16) * U) * (g.double() / T)[:, None]
    half = torch.finfo(TYPES[dtype]).eps / 2
    bound = tol + half * (want.abs() + tol) + 2.0 ** -126
    off = (got.double() - want).abs()
    assert bool((off <= bound).all()), float((off / bound).max())
