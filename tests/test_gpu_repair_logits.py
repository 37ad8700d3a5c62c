"""Log probabilities, distillation and their gradients against the definitions in float64, at the sizes, strides, masks and ties
where they can go wrong.

Tolerances.  u = 2^-24 is half a step of float32, relative to the value.  A row's sum of exponentials goes through at most
vocab / 512 + 40 additions one after the other (a thread's stripe, then the joins), each off by u; call that L.  A log
probability lp is a difference of a value off by 4 u |lp| (subtraction, scaling, the exponent's argument) and the logarithm of
that sum, so |lp - exact| <= (4 |lp| + L + 8) u, which is also the relative error of exp(lp).  The entropy is the sum of two
terms, neither larger than itself, each with the sums' error: (1 + 2 H) L u and the exponents' 8 u.  A value rounded to its type t is off by
half a step more, finfo(t).eps / 2 relative.
"""
import itertools
import math

import pytest
import torch

from paper_2508_02322_amd import binding

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def chain(vocab):
    return vocab / 512 + 40


def lp_error(lp, vocab):
    return (4 * torch.where(lp == -math.inf, 0.0, lp).abs() + chain(vocab) + 8) * U


def make_logits(n, vocab, dtype, seed, pad=0, offset=0, spread=3.0):
    """[n, vocab] in rows vocab + pad apart, the first `offset` elements into the buffer; the rest of the buffer is NaN."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    buf = torch.full((offset + n * (vocab + pad) + 16,), float("nan"), dtype=TYPES[dtype], device="cuda")
    rows = buf[offset:offset + n * (vocab + pad)].view(n, vocab + pad)[:, :vocab]
    rows.copy_(spread * torch.randn((n, vocab), generator=g, device="cuda"))
    return rows


def log_softmax64(logits, temperature):
    # relative to the largest logit first: beside values of 1e38, float64 too would lose the logarithm of the sum
    d = (logits.double() - logits.double().amax(1, keepdim=True)) / float(torch.tensor(temperature, dtype=torch.float32))
    return torch.where(logits == -math.inf, -math.inf, d - torch.logsumexp(d, 1, keepdim=True))


def top64(logits, k):
    """Indices and values of the k largest, equal values in rising index order; -1 where the value is -inf."""
    value, idx = torch.sort(logits.double() + 0.0, dim=1, descending=True, stable=True)
    value, idx = value[:, :k], idx[:, :k]
    return idx.masked_fill(value == -math.inf, -1).int()


def check_logprobs(cam, logits, targets, top_k, temperature):
    n, vocab = logits.shape
    out = cam.token_logprobs(logits, targets, top_k=top_k, temperature=temperature)
    torch.cuda.synchronize()
    lp = log_softmax64(logits, temperature)
    H = torch.special.entr(lp.exp()).sum(1)
    tol = (1 + 2 * H) * chain(vocab) * U + 8 * U
    assert torch.all((out["entropy"].double() - H).abs() <= tol), float((out["entropy"].double() - H).abs().max())
    assert torch.equal(out["stats"][:, 0], logits.float().amax(1))
    if targets is not None:
        has = (targets >= 0) & (targets < vocab)
        want = torch.where(has, lp[torch.arange(n, device="cuda"), targets.long().clamp(0, vocab - 1)], 0.0)
        finite = want > -math.inf
        assert torch.all((out["logprob"].double() - want).abs()[finite] <= lp_error(want, vocab)[finite])
        assert torch.all(out["logprob"][~finite] == -math.inf)
    if top_k:
        idx = top64(logits, top_k)
        assert torch.equal(out["top_idx"], idx)
        want = torch.where(idx >= 0, lp.gather(1, idx.long().clamp(min=0)), -math.inf)
        finite = want > -math.inf
        assert torch.all((out["top_logprob"].double() - want).abs()[finite] <= lp_error(want, vocab)[finite])
        assert torch.all(out["top_logprob"][~finite] == -math.inf)
    return out


def random_targets(n, vocab, seed, ignored=0.2):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.randint(0, vocab, (n,), generator=g, device="cuda")
    t[torch.rand(n, generator=g, device="cuda") < ignored] = -100
    if n > 3:
        t[3] = vocab      # just outside
    return t.int()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,vocab,top_k,pad,offset", [
    (1, 1, 1, 0, 0), (1, 2, 2, 0, 1), (3, 7, 7, 0, 3), (1, 8, 3, 0, 0), (2, 9, 0, 5, 0), (5, 511, 20, 0, 5), (4, 513, 256, 3, 0),
    (1, 4096, 5, 0, 0), (1, 4097, 64, 0, 1), (3, 5000, 256, 7, 2), (70, 12345, 33, 0, 0), (1, 151936, 20, 0, 0), (9, 50257, 1, 0, 0),
    (2050, 3001, 8, 1, 0), (300, 32003, 100, 0, 7)])
def test_logprobs_sizes_and_strides(cam, n, vocab, top_k, pad, offset, dtype):
    logits = make_logits(n, vocab, dtype, 11 + n + vocab, pad, offset)
    check_logprobs(cam, logits, random_targets(n, vocab, 5), top_k, 1.0)


@pytest.mark.parametrize("temperature", [0.25, 0.7, 3.0])
def test_logprobs_temperature(cam, temperature):
    logits = make_logits(6, 20011, "f32", 3)
    check_logprobs(cam, logits, random_targets(6, 20011, 5), 16, temperature)


def test_logprobs_without_targets(cam):
    logits = make_logits(6, 2001, "bf16", 3)
    out = check_logprobs(cam, logits, None, 3, 1.0)
    assert "logprob" not in out
    assert "top_idx" not in cam.token_logprobs(logits)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [40, 3000, 70001])
def test_logprobs_masks_and_ties(cam, vocab, dtype):
    """Rows: one token left; none left; fewer left than alternatives; the type's lowest value as the mask; a constant row; two
    values only; rising; falling; zeros of both signs; huge logits; one token far above the rest."""
    dt = TYPES[dtype]
    z = make_logits(12, vocab, dtype, 7)
    low = torch.finfo(dt).min
    z[0] = -math.inf
    z[0, vocab // 3] = 2.0
    z[1] = -math.inf
    z[2, 5:] = -math.inf
    z[3, 4:] = low
    z[4] = 1.5
    z[5] = (torch.arange(vocab, device="cuda") % 3 == 1).to(dt)
    z[6] = torch.linspace(-5, 5, vocab, device="cuda").to(dt)
    z[7] = torch.linspace(5, -5, vocab, device="cuda").to(dt)
    z[8] = 0.0
    z[8, ::2] = -0.0
    z[9] = low
    z[10] *= 1e30
    z[11, vocab - 1] = 300.0
    targets = torch.tensor([vocab // 3, 2, 3, 2, vocab - 1, 1, 0, 0, 1, 5, 3, vocab - 1], dtype=torch.int32, device="cuda")
    k = min(vocab, 30)
    out = cam.token_logprobs(z, targets, top_k=k)
    torch.cuda.synchronize()
    assert torch.equal(out["top_idx"], top64(z, k))
    # the empty row
    assert out["entropy"][1] == 0 and out["logprob"][1] == -math.inf and torch.all(out["top_logprob"][1] == -math.inf)
    assert out["stats"][1, 0] == -math.inf and out["stats"][1, 1] == 0
    # all others by the definition (the wide row's probabilities are 0 or 1: its log probabilities are its differences)
    rows = [i for i in range(12) if i != 1]
    for i in rows:
        check_logprobs(cam, z[i:i + 1], targets[i:i + 1], k, 1.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 1024])
def test_more_candidates_than_room(cam, n, dtype):
    """Thousands of values reach the bound: all equal; equal but for a few larger ones, behind and among them; different in their last
    bits only; larger ones in a few stripes, more of them than wanted; equal ones that begin late; the same with every second ruled out."""
    vocab, vec = (16000, 8 if dtype == "bf16" else 4)
    at = torch.arange(vocab, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(2)
    noise = torch.rand(vocab, generator=g, device="cuda")
    rows = [torch.ones(vocab, device="cuda"), 1.0 + 1e-3 * noise,
            torch.where(at % 3001 == 7, 3.0 + at / vocab, torch.full_like(noise, 0.5)),
            torch.where((at // vec) % 128 < 5, 2.0 + noise, torch.full_like(noise, 0.5)),
            torch.where((at // vec) % 512 < 10, 2.0 + noise, torch.full_like(noise, 0.5)),
            torch.where(at > 9000, 1.0, -1.0), torch.where(at % 2 == 0, -math.inf, 0.25), torch.where(noise < 0.5, 0.25, 0.25 + 2.0 ** -24)]
    z = torch.stack(rows).to(TYPES[dtype])
    if n > len(rows):
        z = z.repeat(n // len(rows), 1)
    for k in (1, 20, 64, 256):
        for part in ([z] if n > 1 else [z[i:i + 1] for i in range(len(rows))]):
            out = cam.token_logprobs(part, top_k=k)
            torch.cuda.synchronize()
            assert torch.equal(out["top_idx"], top64(part, k)), (n, k)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab,top_k", [(1, 1), (5, 5), (63, 63), (500, 64), (513, 64), (4097, 20), (16384, 64), (16384, 65), (16385, 64)])
def test_many_short_rows(cam, vocab, top_k, dtype):
    """1030 rows in short workgroups (and just beyond where they are used): rows with ties, masks and nothing left among ordinary ones."""
    n = 1030
    z = make_logits(n, vocab, dtype, 13, pad=3)
    z[::7] = -math.inf
    z[::7, vocab // 2:vocab // 2 + 9] = 1.0
    z[3::7] = 0.25
    z[5::7] = torch.finfo(TYPES[dtype]).min
    z[5::7, vocab // 3] = -2.0
    z[6::7] = torch.linspace(-4, 4, vocab, device="cuda").to(TYPES[dtype])
    z[1024] = -math.inf
    out = cam.token_logprobs(z, random_targets(n, vocab, 3), top_k=top_k)
    rest = torch.arange(n, device="cuda") != 1024
    check_logprobs(cam, z[rest], random_targets(n, vocab, 3)[rest], top_k, 1.0)
    torch.cuda.synchronize()
    assert torch.equal(out["top_idx"], top64(z, top_k)) and out["entropy"][1024] == 0


def test_logprobs_do_not_depend_on_the_cut(cam):
    """One row by itself is cut into many parts, among many rows into few: the same tokens, and sums equal to their rounding."""
    logits = make_logits(2048, 9001, "bf16", 1)
    targets = random_targets(2048, 9001, 2, ignored=0.0)
    whole = cam.token_logprobs(logits, targets, top_k=50)
    for i in (0, 7, 2047):
        one = cam.token_logprobs(logits[i:i + 1], targets[i:i + 1], top_k=50)
        assert torch.equal(one["top_idx"], whole["top_idx"][i:i + 1])
        assert abs(float(one["entropy"][0] - whole["entropy"][i])) <= float((2 + 4 * whole["entropy"][i]) * chain(9001) * U)
    again = cam.token_logprobs(logits, targets, top_k=50)
    for key in whole:
        assert torch.equal(whole[key], again[key]), key


def test_logprobs_bad_rows_leave_the_others(cam):
    """NaN and +inf in a row: its indices stay tokens or -1, and the other rows do not change."""
    logits = make_logits(5, 6007, "f32", 4)
    good = cam.token_logprobs(logits, top_k=9)
    bad = logits.clone()
    bad[1, 17] = float("nan")
    bad[3, 4000] = math.inf
    bad[3, 4001] = float("nan")
    out = cam.token_logprobs(bad, top_k=9)
    torch.cuda.synchronize()
    for i in (0, 2, 4):
        assert torch.equal(out["top_idx"][i], good["top_idx"][i]) and out["entropy"][i] == good["entropy"][i]
    assert torch.all((out["top_idx"] >= -1) & (out["top_idx"] < 6007))


def logprob_gradient64(logits, targets, g_lp, g_h, temperature):
    n, vocab = logits.shape
    T = float(torch.tensor(temperature, dtype=torch.float32))
    lp = log_softmax64(logits, temperature)
    p = lp.exp()
    H = torch.special.entr(p).sum(1, keepdim=True)
    has = torch.zeros(n, dtype=torch.bool, device="cuda") if targets is None else (targets >= 0) & (targets < vocab)
    one = torch.zeros(n, 1, dtype=torch.float64, device="cuda") if g_lp is None else torch.where(has, g_lp.double(), 0.0)[:, None]
    two = torch.zeros(n, 1, dtype=torch.float64, device="cuda") if g_h is None else g_h.double()[:, None]
    inner = torch.where(p > 0, lp + H, 0.0)
    want = -p * (one + two * inner)
    size = p * (one.abs() + two.abs() * inner.abs())     # what the rounding errors are relative to
    # the entropy's own error, and that of lp, inside the bracket
    slack = p * two.abs() * ((1 + 2 * H) * chain(vocab) * U + lp_error(lp, vocab))
    if targets is not None:
        rows = torch.nonzero(has)[:, 0]
        want[rows, targets[rows].long()] += one[rows, 0]
        size[rows, targets[rows].long()] += one[rows, 0].abs()
    return want / T, (size * (lp_error(lp, vocab) + 4 * U) + slack) / T


def check_gradient(got, want, tol, dtype):
    half = torch.finfo(TYPES[dtype]).eps / 2
    tiny = float(torch.finfo(torch.float32).tiny)        # below it float32 (and bf16) lose bits
    err = (got.double() - want).abs()
    bad = err > tol + half * (want.abs() + tol) + tiny
    assert not bool(bad.any()), (float(err[bad].max()), int(bad.sum()), float(want.abs().max()))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,vocab,pad,pad_out,which,temperature", [
    (1, 1, 0, 0, "both", 1.0), (2, 7, 0, 3, "lp", 1.0), (3, 4099, 5, 0, "entropy", 0.5), (4, 16384, 0, 0, "both", 1.0),
    (3, 16385, 1, 2, "both", 2.0), (65, 3001, 0, 0, "lp", 1.0), (2, 151937, 0, 0, "both", 1.0)])
def test_logprobs_gradient(cam, n, vocab, pad, pad_out, which, temperature, dtype):
    logits = make_logits(n, vocab, dtype, n + vocab, pad)
    if vocab > 100:
        logits[n - 1, 20:40] = -math.inf
    targets = random_targets(n, vocab, 9)
    targets[targets.eq(25)] = 3
    g = torch.Generator(device="cuda").manual_seed(1)
    g_lp = torch.randn(n, generator=g, device="cuda") if which != "entropy" else None
    g_h = torch.randn(n, generator=g, device="cuda") if which != "lp" else None
    fwd = cam.token_logprobs(logits, targets, temperature=temperature)
    buf = torch.full((n, vocab + pad_out), 77.0, dtype=TYPES[dtype], device="cuda")
    got = cam.token_logprobs_backward(logits, targets, fwd["stats"], g_lp, fwd["entropy"] if g_h is not None else None, g_h,
                                      temperature, dlogits=buf[:, :vocab])
    torch.cuda.synchronize()
    assert got.data_ptr() == buf.data_ptr() and torch.all(buf[:, vocab:] == 77.0)
    want, tol = logprob_gradient64(logits, targets, g_lp, g_h, temperature)
    check_gradient(got, want, tol, dtype)


def test_logprobs_gradient_against_differences(cam):
    """The gradient of sum(a logprob + b entropy) by central differences of the float64 definition."""
    n, vocab, T = 2, 37, 0.8
    logits = make_logits(n, vocab, "f32", 6)
    targets = torch.tensor([5, 30], dtype=torch.int32, device="cuda")
    a, b = torch.tensor([0.7, -1.3], device="cuda"), torch.tensor([0.4, 0.9], device="cuda")
    fwd = cam.token_logprobs(logits, targets, temperature=T)
    got = cam.token_logprobs_backward(logits, targets, fwd["stats"], a, fwd["entropy"], b, T)

    def f(z):
        lp = torch.log_softmax(z / float(torch.tensor(T, dtype=torch.float32)), 1)
        H = -(lp.exp() * lp).sum(1)
        return (a.double() * lp[torch.arange(n, device="cuda"), targets.long()] + b.double() * H).sum()
    z, h = logits.double(), 1e-5
    want = torch.zeros_like(z)
    for i, v in itertools.product(range(n), range(vocab)):
        e = torch.zeros_like(z)
        e[i, v] = h
        want[i, v] = (f(z + e) - f(z - e)) / (2 * h)
    # differences: h^2 and 1e-16 / h; float32: a few steps of values below 1
    assert float((got.double() - want).abs().max()) < 1e-8 + 64 * U


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradient_in_place_and_added(cam, dtype):
    n, vocab = 5, 20001
    logits = make_logits(n, vocab, dtype, 8, pad=3)
    targets = random_targets(n, vocab, 9)
    g = torch.linspace(-1, 1, n, device="cuda")          # one row has no gradient
    fwd = cam.token_logprobs(logits, targets)
    plain = cam.token_logprobs_backward(logits, targets, fwd["stats"], g, fwd["entropy"], g)
    old = torch.randn((n, vocab), device="cuda").to(TYPES[dtype])
    added = cam.token_logprobs_backward(logits, targets, fwd["stats"], g, fwd["entropy"], g, dlogits=old.clone(), accumulate=True)
    want, tol = logprob_gradient64(logits, targets, g, g, 1.0)
    check_gradient(added, want + old.double(), tol + U * (want.abs() + old.double().abs()), dtype)
    assert torch.equal(added[2], old[2]) and not bool(plain[2].any())
    same = logits
    got = cam.token_logprobs_backward(same, targets, fwd["stats"], g, fwd["entropy"], g, dlogits=same)
    torch.cuda.synchronize()
    assert torch.equal(got, plain)


# ---- distillation --------------------------------------------------------------------------------------------------
def make_teacher(n, vocab, k, temperature, seed, tail, spread=3.0):
    z = make_logits(n, vocab, "f32", seed, spread=spread).double() / temperature
    top = z.topk(min(k, vocab), dim=1)
    lp = top.values - torch.logsumexp(z, 1, keepdim=True)
    idx = torch.full((n, k), -1, dtype=torch.int32, device="cuda")
    val = torch.full((n, k), 0.5, dtype=torch.float32, device="cuda")
    idx[:, :top.indices.shape[1]] = top.indices.int()
    val[:, :top.indices.shape[1]] = (lp if tail else lp * temperature).float()
    return idx, val


def distill64(logits, idx, val, temperature, tail):
    """(loss, mass, factor, gradient per grad_loss, q per token, p, lp, marks) by the definition; the first entry that names a token counts."""
    n, vocab = logits.shape
    T = float(torch.tensor(temperature, dtype=torch.float32))
    lp = log_softmax64(logits, temperature)
    p = lp.exp()
    k = idx.shape[1]
    ok = (idx >= 0) & (idx < vocab) & (val > -math.inf)
    for j in range(1, k):
        ok[:, j] &= ~(idx[:, :j] == idx[:, j:j + 1]).any(1)
    t = val.double().masked_fill(~ok, -math.inf)
    if tail:
        q = t.exp()
        norm = torch.zeros(n, 1, dtype=torch.float64, device="cuda")
    else:
        norm = torch.logsumexp(t / T, 1, keepdim=True)
        q = torch.where(ok, (t / T - norm).exp(), 0.0)
        norm = torch.where(norm == -math.inf, 0.0, norm)
    at = idx.long().clamp(0, vocab - 1)
    dense = torch.zeros(n, vocab, dtype=torch.float64, device="cuda").scatter_add_(1, at, torch.where(ok, q, 0.0))
    marks = torch.zeros(n, vocab, dtype=torch.float64, device="cuda").scatter_add_(1, at, ok.double()) > 0
    loss = torch.where(dense > 0, dense * (dense.log() - lp), 0.0).sum(1)
    mass = q.sum(1)
    factor = mass.clone()
    rest = torch.where(marks, -math.inf, lp)
    log_rest = torch.logsumexp(rest, 1)
    ratio = torch.zeros_like(mass)
    if tail:
        left = (1 - mass).clamp(min=0)
        has = (log_rest > -math.inf) & (left > 0)
        loss = loss + torch.where(has, left * (left.clamp(min=1e-300).log() - torch.where(has, log_rest, 0.0)), 0.0)
        ratio = torch.where(has, left * (-torch.where(has, log_rest, 0.0)).exp(), 0.0)
        mass = mass + torch.where(log_rest > -math.inf, left, 0.0)
        factor = mass - ratio
    grad = torch.where(marks, mass[:, None] * p - dense, p * factor[:, None]) / T
    return dict(loss=loss, mass=mass, factor=factor, ratio=ratio, grad=grad, q=dense, p=p, lp=lp, marks=marks, norm=norm[:, 0], T=T,
                log_rest=log_rest)


def check_distill(cam, logits, idx, val, temperature, tail, dtype, g=None, **kw):
    n, vocab = logits.shape
    out = cam.distill_topk(logits, idx, val, temperature=temperature, tail=tail)
    if g is None:
        g = torch.randn(n, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
    got = cam.distill_topk_backward(logits, idx, val, out["stats"], g, temperature=temperature, tail=tail, **kw)
    torch.cuda.synchronize()
    w = distill64(logits, idx, val, temperature, tail)
    L = chain(vocab)
    reach = torch.where(w["marks"] & (w["lp"] > -math.inf), w["lp"].abs(), 0.0).amax(1) + torch.where(w["log_rest"] > -math.inf, w["log_rest"].abs(), 0.0)
    finite = w["loss"] < math.inf
    tol = (4 * reach + 2 * L + 16) * U + U * w["loss"].abs()
    assert torch.all((out["loss"].double() - w["loss"]).abs()[finite] <= tol[finite]), float(((out["loss"].double() - w["loss"]).abs() / tol)[finite].max())
    assert torch.all(out["loss"][~finite] == math.inf)
    st = out["stats"].double()
    assert torch.all((st[:, 3] - w["mass"]).abs() <= 4 * U)
    has = w["ratio"] > 0
    log_ratio = torch.where(has, w["ratio"], 1.0).log()
    assert torch.all((st[:, 4] - log_ratio).abs()[has] <= ((2 * L + 4 * reach + 8) * U + U * log_ratio.abs())[has])
    assert torch.all(st[:, 4][~has] == -math.inf)
    ratio_tol = w["ratio"] * (2 * L + 4 * reach + 8 + 4 * log_ratio.abs()) * U
    # the gradient
    rel = lp_error(w["lp"], vocab)
    lq = 4 * (val.double().clamp(min=-1e4).abs().amax(1, keepdim=True) / w["T"] + w["norm"].abs()[:, None] + 4) * U
    unlisted = w["p"] * (w["factor"].abs()[:, None] * (rel + 8 * U) + ratio_tol[:, None] + 2 * U * (w["mass"] + w["ratio"])[:, None])
    listed = w["p"] * w["mass"][:, None] * (rel + 8 * U) + w["q"] * lq
    tol = torch.where(w["marks"], listed, unlisted) / w["T"] * g.double().abs()[:, None]
    return out, got, w["grad"] * g.double()[:, None], tol


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("n,vocab,k,pad,offset,temperature", [
    (1, 1, 1, 0, 0, 1.0), (2, 7, 3, 1, 1, 1.0), (3, 7, 7, 0, 0, 2.0), (2, 5, 9, 0, 0, 1.0), (4, 4097, 64, 0, 3, 1.0),
    (1, 50021, 256, 0, 0, 0.5), (65, 9001, 20, 3, 0, 2.0), (2049, 1500, 5, 0, 0, 1.0), (1024, 16384, 256, 0, 1, 1.0), (1024, 300, 256, 0, 0, 1.0), (1100, 16385, 7, 0, 0, 1.0), (3, 151936, 100, 0, 0, 1.0), (2, 300001, 30, 0, 0, 1.0)])
def test_distill_loss_and_gradient(cam, n, vocab, k, pad, offset, temperature, tail, dtype):
    idx, val = make_teacher(n, vocab, k, temperature, 21, tail)
    logits = make_logits(n, vocab, dtype, 22 + vocab, pad, offset)
    _, got, want, tol = check_distill(cam, logits, idx, val, temperature, tail, dtype)
    check_gradient(got, want, tol, dtype)


@pytest.mark.parametrize("tail", [False, True])
def test_distill_entries_that_do_not_count(cam, tail):
    """Rows: as made; ids outside the vocabulary; the same id three times; no entry at all; entries of probability 0; one entry; all of
    the student's probability on the listed tokens; the student rules listed and unlisted tokens out; the student rules everything out."""
    n, vocab, k = 10, 3003, 12
    idx, val = make_teacher(n, vocab, k, 1.0, 31, tail)
    z = make_logits(n, vocab, "f32", 32)
    idx[1, ::2] = torch.tensor([-1, vocab, 2 ** 31 - 1, -2 ** 31, -5, vocab + 1], dtype=torch.int32, device="cuda")
    idx[2, 4], idx[2, 9] = idx[2, 1], idx[2, 1]
    idx[3] = -1
    val[4, 2:6] = -math.inf
    idx[5, 1:] = -7
    z[6] = -200.0
    z[6, idx[6].long()] = 3.0
    z[7, 1000:] = -math.inf
    idx[7] = torch.arange(5, 5 + k, device="cuda").int()
    z[8] = -math.inf
    z[9, idx[9, 0].long()] = -math.inf                     # a token the teacher wants
    out, got, want, tol = check_distill(cam, z[:8], idx[:8], val[:8], 1.0, tail, "f32")
    check_gradient(got, want, tol, "f32")
    if not tail:
        assert out["loss"][3] == 0 and not bool(got[3].any())
    out = cam.distill_topk(z, idx, val, tail=tail)
    got = cam.distill_topk_backward(z, idx, val, out["stats"], torch.ones(n, device="cuda"), tail=tail)
    torch.cuda.synchronize()
    assert out["loss"][9] == math.inf and out["loss"][8] == math.inf and not bool(got[8].any())
    assert bool(torch.isfinite(got[9]).all())


def test_distill_tail_against_differences(cam):
    n, vocab, k, T = 2, 23, 4, 1.5
    idx, val = make_teacher(n, vocab, k, T, 41, True)
    logits = make_logits(n, vocab, "f32", 42)
    g = torch.tensor([0.8, -1.1], device="cuda")
    for tail in (True, False):
        out = cam.distill_topk(logits, idx, val, T, tail)
        got = cam.distill_topk_backward(logits, idx, val, out["stats"], g, T, tail)
        z, h = logits.double(), 1e-5
        want = torch.zeros_like(z)
        for i, v in itertools.product(range(n), range(vocab)):
            e = torch.zeros_like(z)
            e[i, v] = h
            want[i, v] = ((distill64(z + e, idx, val, T, tail)["loss"] - distill64(z - e, idx, val, T, tail)["loss"]) * g.double()).sum() / (2 * h)
        assert float((got.double() - want).abs().max()) < 1e-8 + 64 * U


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_distill_gradient_in_place_and_added(cam, dtype):
    n, vocab, k = 4, 40003, 50
    idx, val = make_teacher(n, vocab, k, 1.0, 51, True)
    logits = make_logits(n, vocab, dtype, 52, pad=5)
    g = torch.tensor([0.5, 0.0, -2.0, 1.0], device="cuda")
    _, plain, want, tol = check_distill(cam, logits, idx, val, 1.0, True, dtype, g=g)
    check_gradient(plain, want, tol, dtype)
    assert not bool(plain[1].any())
    old = torch.randn((n, vocab), device="cuda").to(TYPES[dtype])
    _, added, want, tol = check_distill(cam, logits, idx, val, 1.0, True, dtype, g=g, dlogits=old.clone(), accumulate=True)
    check_gradient(added, want + old.double(), tol + U * (want.abs() + old.double().abs()), dtype)
    assert torch.equal(added[1], old[1])
    stats = cam.distill_topk(logits, idx, val, tail=True)["stats"]
    got = cam.distill_topk_backward(logits, idx, val, stats, g, tail=True, dlogits=logits)
    torch.cuda.synchronize()
    assert got.data_ptr() == logits.data_ptr() and torch.equal(got, plain)


def test_distill_of_the_same_model_is_zero(cam):
    """A teacher against itself, its alternatives straight from token_logprobs: the loss is 0 and so is the gradient, to the
    rounding of the alternatives' log probabilities."""
    logits = make_logits(20, 30011, "bf16", 61)
    for T in (1.0, 2.0):
        top = cam.token_logprobs(logits, top_k=40, temperature=T)
        out = cam.distill_topk(logits, top["top_idx"], top["top_logprob"], temperature=T, tail=True)
        assert float(out["loss"].abs().max()) < 2 * (chain(30011) + 4 * 40 + 8) * U
        grad = cam.distill_topk_backward(logits, top["top_idx"], top["top_logprob"], out["stats"], torch.ones(20, device="cuda"), temperature=T, tail=True)
        assert float(grad.float().abs().max()) < 2 * (chain(30011) + 4 * 40 + 8) * U


# ---- streams, graphs, far rows -------------------------------------------------------------------------------------
def test_logit_calls_on_another_stream_and_in_a_graph(cam):
    n, vocab, k = 3, 20003, 10
    logits = make_logits(n, vocab, "bf16", 71)
    targets = random_targets(n, vocab, 1, ignored=0.0)
    idx, val = make_teacher(n, vocab, k, 1.0, 72, True)
    g = torch.ones(n, device="cuda")

    def step():
        lp = cam.token_logprobs(logits, targets, top_k=k)
        kd = cam.distill_topk(logits, idx, val, tail=True)
        d = cam.token_logprobs_backward(logits, targets, lp["stats"], -g)
        cam.distill_topk_backward(logits, idx, val, kd["stats"], g, tail=True, dlogits=d, accumulate=True)
        return lp["logprob"], lp["top_idx"], kd["loss"], d
    step()
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        aside = step()
    stream.synchronize()
    for a, b in zip(aside, step()):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        with torch.cuda.graph(graph, stream=stream):
            captured = step()
    gen = torch.Generator(device="cuda").manual_seed(7)
    for trial in range(4):
        if trial:
            logits.copy_(3 * torch.randn(logits.shape, generator=gen, device="cuda"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        kept = [x.clone() for x in captured]
        for a, b in zip(kept, step()):
            assert torch.equal(a, b)
        torch.cuda.synchronize()


def test_two_graphs_on_one_workspace(cam):
    """Two captured calls that cut their rows share the context's workspace: replayed in turn, each gives its own result."""
    def capture(n, vocab, k, seed):
        z = make_logits(n, vocab, "bf16", seed)
        cam.token_logprobs(z, top_k=k)
        torch.cuda.synchronize()
        stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        with torch.cuda.stream(stream):
            with torch.cuda.graph(graph, stream=stream):
                out = cam.token_logprobs(z, top_k=k)
        torch.cuda.synchronize()
        return z, k, graph, out
    cam.token_logprobs(make_logits(2, 9000, "bf16", 1), top_k=40)      # the workspace has its size before the first capture
    both = [capture(2, 50000, 40, 1), capture(5, 30001, 17, 2)]
    for trial in range(3):
        for z, k, graph, out in both:
            graph.replay()
        torch.cuda.synchronize()
        for z, k, graph, out in both:
            assert torch.equal(out["top_idx"], top64(z, k))
            for key, want in cam.token_logprobs(z, top_k=k).items():
                assert torch.equal(out[key], want), key
            z.copy_(-z)


def test_rows_beyond_32_bit_offsets(cam):
    """Rows that start more than 2^31 elements into the buffer."""
    vocab, apart = 5003, (1 << 30) + 12345
    buf = torch.empty(2 * apart + vocab, dtype=torch.bfloat16, device="cuda")
    logits = buf.as_strided((3, vocab), (apart, 1))
    logits.copy_(make_logits(3, vocab, "bf16", 81))
    near = logits.contiguous()
    targets = random_targets(3, vocab, 1, ignored=0.0)
    far_out, near_out = cam.token_logprobs(logits, targets, top_k=4), cam.token_logprobs(near, targets, top_k=4)
    g = torch.ones(3, device="cuda")
    want = cam.token_logprobs_backward(near, targets, near_out["stats"], g)
    got = cam.token_logprobs_backward(logits, targets, far_out["stats"], g, dlogits=logits)
    torch.cuda.synchronize()
    for key in near_out:
        assert torch.equal(far_out[key], near_out[key]), key
    assert torch.equal(got.contiguous(), want)


def test_no_rows(cam):
    e = torch.empty((0, 11), dtype=torch.bfloat16, device="cuda")
    out = cam.token_logprobs(e, torch.empty(0, dtype=torch.int32, device="cuda"), top_k=3)
    assert out["logprob"].shape == (0,) and out["top_idx"].shape == (0, 3)
    out = cam.distill_topk(e, torch.empty((0, 2), dtype=torch.int32, device="cuda"), torch.empty((0, 2), device="cuda"))
    assert out["loss"].shape == (0,)


def test_binding_refuses_what_the_library_cannot_see(cam):
    z = make_logits(4, 100, "f32", 1)
    idx, val = make_teacher(4, 100, 3, 1.0, 2, True)
    for call in (lambda: cam.token_logprobs(z.t()), lambda: cam.token_logprobs(z.cpu()), lambda: cam.distill_topk(z.cpu(), idx.cpu(), val.cpu()),
                 lambda: cam.token_logprobs_backward(z, None, torch.zeros((4, 2), device="cuda"), torch.zeros(4), dlogits=z.cpu()), lambda: cam.token_logprobs(z, torch.zeros(3, dtype=torch.int32, device="cuda")),
                 lambda: cam.token_logprobs(z, torch.zeros(4, dtype=torch.int64, device="cuda")),
                 lambda: cam.distill_topk(z, idx[:, ::2], val[:, ::2]), lambda: cam.distill_topk(z, idx, val.double()),
                 lambda: cam.token_logprobs_backward(z, None, torch.zeros((4, 2), device="cuda"), None),
                 lambda: cam.token_logprobs_backward(z, None, torch.zeros((4, 2), device="cuda"), None, accumulate=True),
                 lambda: cam.token_logprobs(z, top_k=101), lambda: cam.token_logprobs(z, temperature=0.0)):
        with pytest.raises(binding.CameraError):
            call()
    for call in (lambda: cam.distill_topk(z, idx[:, 0], val[:, 0]),
                 lambda: cam.distill_topk_backward(z, idx[:, 0], val[:, 0], torch.zeros((4, 5), device="cuda"), torch.zeros(4, device="cuda"))):
        with pytest.raises(binding.CameraError, match="teacher_idx"):
            call()
