"""The gated block and its gradients against the definition in float64: odd widths, one token to many, strides, outputs left out.

Tolerances.  u = 2^-24.  A product's sum over K terms is off by at most K u times the sum of their magnitudes (float32 accumulation;
products of two bf16 are exact in it).  silu and silu' are at most 1.1 steep.  A result rounded to its type is off by half a step,
finfo(t).eps / 2 relative.  With bf16, dG and dU are rounded before their products: independent errors of at most half a step h = 2^-8,
hence a standard deviation of h / sqrt(3) each, so a sum over c of dG_c w_c is off by less than six standard deviations,
6 h / sqrt(3) sqrt(sum (dG_c w_c)^2) (one in 5e8 beyond).
"""
import math

import pytest
import torch

from paper_2508_02322_amd import binding

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def make(n, d, f, dtype, seed, ldx_pad=0, spread=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = TYPES[dtype]
    X = torch.full((n, d + ldx_pad), float("nan"), dtype=dt, device="cuda")[:, :d]
    X.copy_(spread * torch.randn((n, d), generator=g, device="cuda"))
    W = [(torch.randn((f, d), generator=g, device="cuda") / math.sqrt(d)).to(dt) for _ in range(2)]
    dH = torch.randn((n, f), generator=g, device="cuda").to(dt)
    return X, W[0], W[1], dH


def reference(X, Wg, Wu, dH, dtype):
    x, wg, wu, dh = (t.double().contiguous() for t in (X, Wg, Wu, dH))
    d, f, n = x.shape[1], wg.shape[0], x.shape[0]
    half = torch.finfo(TYPES[dtype]).eps / 2
    G, Up = x @ wg.t().contiguous(), x @ wu.t().contiguous()
    eG, eU = d * U * (x.abs() @ wg.abs().t().contiguous()), d * U * (x.abs() @ wu.abs().t().contiguous())
    s = torch.sigmoid(G)
    silu, dsilu = G * s, s * (1 + G * (1 - s))
    H = silu * Up
    tol_H = 1.1 * eG * Up.abs() + silu.abs() * eU + 1.1 * eG * eU + 16 * U * H.abs()
    dU, dG = dh * silu, dh * Up * dsilu
    eDU = dh.abs() * (1.1 * eG + 16 * U * silu.abs())
    eDG = dh.abs() * (dsilu.abs() * eU + Up.abs() * (0.5 * eG + 32 * U) + eG * eU)   # |silu''| <= 1/2
    h2 = (half / math.sqrt(3)) ** 2 if dtype == "bf16" else 0.0

    def product(a, ea, b):          # a [m, k] off by ea (then rounded), b [k, p]
        k = a.shape[1]
        b = b.contiguous()
        out = a @ b
        return out, ea @ b.abs() + k * U * (a.abs() @ b.abs()) + 6 * torch.sqrt(h2 * (a * a) @ (b * b))

    t = lambda m: m.t().contiguous()  # noqa: E731
    x1, e1 = product(dG, eDG, wg)
    x2, e2 = product(dU, eDU, wu)
    g1, eg = product(t(dG), t(eDG), x)
    u1, eu = product(t(dU), t(eDU), x)
    return {"H": (H, tol_H), "dX": (x1 + x2, e1 + e2), "dW_gate": (g1, eg), "dW_up": (u1, eu), "pre": ((G, eG), (Up, eU))}


def close(got, want, tol, dtype, what):
    half = torch.finfo(TYPES[dtype]).eps / 2
    err = (got.double() - want).abs()
    bound = tol + half * (want.abs() + tol) + 2.0 ** -126
    assert bool(torch.isfinite(got).all()), what
    assert bool((err <= bound).all()), (what, float((err / bound).max()))


def check(cam, n, d, f, dtype, seed=1, ldx_pad=0, spread=1.0, pre=True):
    X, Wg, Wu, dH = make(n, d, f, dtype, seed, ldx_pad, spread)
    w = reference(X, Wg, Wu, dH, dtype)
    H, kept = cam.gated_ffn(X, Wg, Wu, want_pre=True)
    alone = cam.gated_ffn(X, Wg, Wu)
    grads = cam.gated_ffn_backward(X, Wg, Wu, dH, pre=kept if pre else None)
    torch.cuda.synchronize()
    close(H, *w["H"], dtype, "H")
    close(alone, *w["H"], dtype, "H alone")
    for i, name in enumerate(("gate", "up")):
        close(kept[:, i, :f], *w["pre"][i], "f32", name)
    for got, name in zip(grads, ("dX", "dW_gate", "dW_up")):
        close(got, *w[name], dtype, name)
    return X, Wg, Wu, dH, H, kept, grads


@pytest.mark.parametrize("n,d,f", [(1, 8, 1), (1, 64, 7), (2, 72, 8), (33, 128, 31), (64, 64, 64), (65, 264, 129), (257, 200, 843), (256, 512, 256),
                                   (1, 2048, 1408), (700, 2048, 131), (1021, 136, 520)])
def test_bf16_block(cam, n, d, f):
    check(cam, n, d, f, "bf16")


# How dX is computed: tiles, and whether K is in parts.
FORMS = {(40, 128, 5000, "bf16"): ("small", True), (700, 256, 200, "bf16"): ("small", False), (2500, 2048, 300, "bf16"): ("smallest", False), (4096, 2048, 200, "bf16"): ("full", False),
         (2048, 3584, 4000, "bf16"): ("full", True), (300, 772, 517, "f32"): ("full", True), (300, 772, 40, "f32"): ("full", False)}


@pytest.mark.parametrize("n,d,f,dtype", list(FORMS))
def test_every_form(cam, n, d, f, dtype):
    check(cam, n, d, f, dtype)


@pytest.mark.parametrize("n,d,f", [(3, 128, 4100), (17, 128, 4100), (64, 72, 4096), (16, 40, 9), (1, 8200, 40)])
def test_bf16_few_tokens(cam, n, d, f):
    """By rows and in tiles, on both sides of where they meet."""
    check(cam, n, d, f, "bf16")


@pytest.mark.parametrize("n,d,f", [(1, 4, 1), (3, 12, 5), (64, 32, 32), (65, 260, 33), (300, 772, 517)])
def test_f32_block(cam, n, d, f):
    check(cam, n, d, f, "f32")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_apart_and_projections_made_again(cam, dtype):
    X, Wg, Wu, dH, H, kept, grads = check(cam, 130, 96, 203, dtype, ldx_pad=16, pre=False)
    again = cam.gated_ffn_backward(X, Wg, Wu, dH, pre=kept)
    for a, b in zip(grads, again):
        assert torch.equal(a, b)
    # gradients left out
    for want in ((True, False, False), (False, True, False), (False, False, True), (True, False, True), (False, True, True)):
        some = cam.gated_ffn_backward(X, Wg, Wu, dH, pre=kept, want=want)
        for a, b, w in zip(some, grads, want):
            assert (a is None) if not w else torch.equal(a, b)
    # dH and H in rows of their own, at any element
    buf = torch.full((130 * 211 + 3,), 9.0, dtype=TYPES[dtype], device="cuda")
    far = buf[3:].view(130, 211)[:, :203]
    far.copy_(dH)
    for a, b in zip(cam.gated_ffn_backward(X, Wg, Wu, far, pre=kept), grads):
        assert torch.equal(a, b)
    wide = torch.full((130, 224), 9.0, dtype=TYPES[dtype], device="cuda")
    cam.gated_ffn(X, Wg, Wu, H=wide[:, :203])
    torch.cuda.synchronize()
    pad = 208 if dtype == "bf16" else 204
    assert torch.equal(wide[:, :203], cam.gated_ffn(X, Wg, Wu)) and not bool(wide[:, 203:pad].any()) and bool((wide[:, pad:] == 9.0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_saturated_gates(cam, dtype):
    """Gates far from zero on both sides: exp overflows to inf or vanishes, the gradient stays finite."""
    check(cam, 40, 64, 48, dtype, spread=60.0)


def test_gradient_against_differences(cam):
    n, d, f = 3, 8, 5
    X, Wg, Wu, dH = make(n, d, f, "f32", 5)
    grads = cam.gated_ffn_backward(X, Wg, Wu, dH)

    def loss(x, wg, wu):
        g, u = x @ wg.t(), x @ wu.t()
        return (dH.double() * (g * torch.sigmoid(g) * u)).sum()
    args = [X.double(), Wg.double(), Wu.double()]
    h = 1e-5
    for i, got in enumerate(grads):
        want = torch.zeros_like(args[i])
        for j in range(want.numel()):
            e = torch.zeros_like(want).view(-1)
            e[j] = h
            e = e.view_as(want)
            up = [a + e if m == i else a for m, a in enumerate(args)]
            down = [a - e if m == i else a for m, a in enumerate(args)]
            want.view(-1)[j] = (loss(*up) - loss(*down)) / (2 * h)
        # differences: 1e-9; float32: sums of up to 10 terms below 10
        assert float((got.double() - want).abs().max()) < 1e-8 + 400 * U


def test_operands_beyond_32_bit_offsets(cam):
    """The rows of [dG | dU], and those of their transpose, are more than 2 GiB; the last rows of every result against the definition."""
    n, d, f = 30000, 8, 18000
    X, Wg, Wu, _ = make(n, d, f, "bf16", 11)
    dH = torch.randn((n, f), generator=torch.Generator(device="cuda").manual_seed(12), device="cuda", dtype=torch.bfloat16)
    H, pre = cam.gated_ffn(X, Wg, Wu, want_pre=True)
    dX, dWg, dWu = cam.gated_ffn_backward(X, Wg, Wu, dH, pre=pre)
    torch.cuda.synchronize()
    few = slice(n - 40, n)
    w = reference(X[few], Wg, Wu, dH[few], "bf16")
    close(H[few], *w["H"], "bf16", "H")
    close(dX[few], *w["dX"], "bf16", "dX")
    few = slice(f - 40, f)
    w = reference(X, Wg[few], Wu[few], dH[:, few], "bf16")
    close(dWg[few], *w["dW_gate"], "bf16", "dW_gate")
    close(dWu[few], *w["dW_up"], "bf16", "dW_up")


def test_packed_expert(cam):
    """The rows that a pruning leaves of one expert, where they lie in the packed matrices."""
    g = torch.Generator(device="cuda").manual_seed(3)
    counts = [37, 90, 11]
    packed = [torch.randn((sum(counts), 128), generator=g, device="cuda").to(torch.bfloat16) / 8 for _ in range(2)]
    X = torch.randn((50, 128), generator=g, device="cuda").to(torch.bfloat16)
    at = 0
    for c in counts:
        Wg, Wu = packed[0][at:at + c], packed[1][at:at + c]
        dH = torch.randn((50, c), generator=g, device="cuda").to(torch.bfloat16)
        w = reference(X, Wg, Wu, dH, "bf16")
        close(cam.gated_ffn(X, Wg, Wu), *w["H"], "bf16", "H")
        for got, name in zip(cam.gated_ffn_backward(X, Wg, Wu, dH), ("dX", "dW_gate", "dW_up")):
            close(got, *w[name], "bf16", name)
        at += c


def test_no_tokens(cam):
    X, Wg, Wu, dH = make(0, 64, 24, "bf16", 1)
    assert cam.gated_ffn(X, Wg, Wu).shape == (0, 24)
    dX, dWg, dWu = cam.gated_ffn_backward(X, Wg, Wu, dH)
    torch.cuda.synchronize()
    assert dX.shape == (0, 64) and not bool(dWg.any()) and not bool(dWu.any())


def test_on_another_stream_and_in_a_graph(cam):
    X, Wg, Wu, dH = make(70, 128, 100, "bf16", 4)

    def step():
        H, pre = cam.gated_ffn(X, Wg, Wu, want_pre=True)
        return (H, *cam.gated_ffn_backward(X, Wg, Wu, dH, pre=pre))
    step()
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        aside = step()
    stream.synchronize()
    for a, b in zip(aside, step()):
        assert torch.equal(a, b)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        with torch.cuda.graph(graph, stream=stream):
            captured = step()
    gen = torch.Generator(device="cuda").manual_seed(7)
    for trial in range(4):
        if trial:
            X.copy_(torch.randn(X.shape, generator=gen, device="cuda"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        kept = [x.clone() for x in captured]
        for a, b in zip(kept, step()):
            assert torch.equal(a, b)
        torch.cuda.synchronize()


def test_binding_refuses_what_the_library_cannot_see(cam):
    X, Wg, Wu, dH = make(4, 64, 24, "bf16", 1)
    for call in (lambda: cam.gated_ffn(X, Wg.t(), Wu.t()), lambda: cam.gated_ffn(X, Wg, Wu[:20]), lambda: cam.gated_ffn(X, Wg.float(), Wu.float()),
                 lambda: cam.gated_ffn(X[:, ::2], Wg, Wu), lambda: cam.gated_ffn(X, Wg, Wu, H=torch.empty((4, 23), dtype=X.dtype, device="cuda")),
                 lambda: cam.gated_ffn(X.cpu(), Wg.cpu(), Wu.cpu()), lambda: cam.gated_ffn_backward(X, Wg, Wu, dH[:, :20]), lambda: cam.gated_ffn_backward(X, Wg, Wu, dH, pre=dH.float())):
        with pytest.raises(binding.CameraError):
            call()
    short = torch.empty(3 * 32 + 20, dtype=X.dtype, device="cuda")          # the last row's zeros would lie behind the buffer
    with pytest.raises(binding.CameraError, match="last row"):
        cam.gated_ffn(X, Wg[:20].contiguous(), Wu[:20].contiguous(), H=short.as_strided((4, 20), (32, 1)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_row_has_no_stride(cam, dtype):
    """torch leaves any number as the row stride of a single row, here an odd one and one of 0; only the address counts."""
    X, Wg, Wu, dH = make(1, 64, 24, dtype, 3)
    H, pre = cam.gated_ffn(X, Wg, Wu, want_pre=True)
    want = cam.gated_ffn_backward(X, Wg, Wu, dH, pre=pre)
    for stride in (0, 1, 67):
        x, dh = X.as_strided((1, 64), (stride, 1)), dH.as_strided((1, 24), (stride, 1))
        assert x.stride(0) == stride
        assert torch.equal(cam.gated_ffn(x, Wg, Wu), H)
        for a, b in zip(cam.gated_ffn_backward(x, Wg, Wu, dh, pre=pre), want):
            assert torch.equal(a, b)
