"""Calls of the operators that judge and repair a pruned model which are refused on the host, each for the argument that it names; every
other argument is one that the call takes."""
import pytest
import torch

from paper_2508_02322_amd import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_of_a_given_block_that_lie_on_each_other(cam, dtype):
    X, W = torch.randn((4, 64), device="cuda").to(dtype), torch.randn((64, 64), device="cuda").to(dtype)
    behind = torch.full((4 * 64,), 9.0, dtype=dtype, device="cuda")
    for H in (behind[:64].view(1, 64).expand(4, 64), behind.as_strided((4, 64), (8, 1)), behind.as_strided((4, 64), (1, 1))):
        with pytest.raises(binding.CameraError, match="ldh"):
            cam.gated_ffn(X, W, W, H=H)
    torch.cuda.synchronize()
    assert bool((behind == 9.0).all())
    whole = behind.view(4, 64)
    assert torch.equal(cam.gated_ffn(X, W, W, H=whole), cam.gated_ffn(X, W, W))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_given_row_of_one_token(cam, dtype):
    """Taken whatever its stride; refused where the last vector would lie behind the buffer."""
    X, W = torch.randn((1, 64), device="cuda").to(dtype), torch.randn((20, 64), device="cuda").to(dtype)
    whole = 24 if dtype == torch.bfloat16 else 20
    want = cam.gated_ffn(X, W, W)
    for stride in (0, 1, 20, 67):
        buf = torch.full((40,), 9.0, dtype=dtype, device="cuda")
        H = buf.as_strided((1, 20), (stride, 1))
        assert cam.gated_ffn(X, W, W, H=H) is H
        torch.cuda.synchronize()
        assert torch.equal(buf[:20], want[0]) and not bool(buf[20:whole].any()) and bool((buf[whole:] == 9.0).all())
    if dtype == torch.bfloat16:
        with pytest.raises(binding.CameraError, match="last row"):
            cam.gated_ffn(X, W, W, H=torch.empty((1, 20), dtype=dtype, device="cuda"))


def logit_arguments(n=4, vocab=100, k=3):
    z = torch.randn((n, vocab), device="cuda")
    stats = torch.zeros((n, 2), device="cuda")
    return dict(logits=z, targets=torch.zeros(n, dtype=torch.int32, device="cuda"), stats=stats, grad_logprob=torch.ones(n, device="cuda"),
                entropy=torch.ones(n, device="cuda"), grad_entropy=torch.ones(n, device="cuda"), dlogits=torch.empty_like(z),
                teacher_idx=torch.zeros((n, k), dtype=torch.int32, device="cuda"), teacher_logprob=torch.zeros((n, k), device="cuda"),
                distill_stats=torch.zeros((n, 5), device="cuda"), grad_loss=torch.ones(n, device="cuda"))


CALLS = {
    "token_logprobs": lambda cam, a, **kw: cam.token_logprobs(a["logits"], a["targets"], **kw),
    "token_logprobs_backward": lambda cam, a, **kw: cam.token_logprobs_backward(
        a["logits"], a["targets"], a["stats"], a["grad_logprob"], a["entropy"], a["grad_entropy"], dlogits=a["dlogits"], **kw),
    "distill_topk": lambda cam, a, **kw: cam.distill_topk(a["logits"], a["teacher_idx"], a["teacher_logprob"], **kw),
    "distill_topk_backward": lambda cam, a, **kw: cam.distill_topk_backward(
        a["logits"], a["teacher_idx"], a["teacher_logprob"], a["distill_stats"], a["grad_loss"], dlogits=a["dlogits"], **kw)}
TAKES = {"token_logprobs": ["logits", "targets"],
         "token_logprobs_backward": ["logits", "targets", "stats", "grad_logprob", "entropy", "grad_entropy", "dlogits"],
         "distill_topk": ["logits", "teacher_idx", "teacher_logprob"],
         "distill_topk_backward": ["logits", "teacher_idx", "teacher_logprob", "distill_stats", "grad_loss", "dlogits"]}


def reported(name):
    return "stats" if name == "distill_stats" else name


@pytest.mark.parametrize("call", list(CALLS))
def test_every_tensor_of_the_calls_on_logits(cam, call):
    """One at a time: on the host, of another type, a row short, every second column or value.  With all of them right the call works."""
    CALLS[call](cam, logit_arguments())
    torch.cuda.synchronize()
    for name in TAKES[call]:
        t = logit_arguments()[name]
        other = {torch.float32: torch.float64, torch.int32: torch.int64}[t.dtype]
        apart = torch.cat([t, t], -1)[..., ::2]
        for how, bad in (("host", t.cpu()), ("type", t.to(other)), ("short", t[:3]), ("apart", apart)):
            a = logit_arguments()
            a[name] = bad
            # a row less of the logits themselves is a matter of whatever comes with them; their type, of what the library takes
            match = {("logits", "short"): "must be", ("logits", "type"): "dtype"}.get((name, how), f"{reported(name)}:")
            with pytest.raises((binding.CameraError, TypeError, ValueError), match=match):
                CALLS[call](cam, a)


@pytest.mark.parametrize("call", ["token_logprobs_backward", "distill_topk_backward"])
def test_accumulating_takes_a_gradient_of_its_own(cam, call):
    a = logit_arguments()
    a["dlogits"] = None
    with pytest.raises(binding.CameraError, match="accumulate"):
        CALLS[call](cam, a, accumulate=True)
    a["dlogits"] = a["logits"]
    with pytest.raises(binding.CameraError, match="dlogits"):
        CALLS[call](cam, a, accumulate=True)


@pytest.mark.parametrize("call", ["token_logprobs_backward", "distill_topk_backward"])
def test_gradient_rows_on_each_other(cam, call):
    a = logit_arguments()
    a["dlogits"] = torch.empty((1, 100), device="cuda").expand(4, 100)
    with pytest.raises(binding.CameraError, match="ldd"):
        CALLS[call](cam, a)


@pytest.mark.parametrize("name", ["X", "W_gate", "W_up", "dH", "pre", "H"])
def test_every_tensor_of_the_gated_block(cam, name):
    def tensors():
        bf16 = torch.bfloat16
        t = dict(X=torch.zeros((4, 64), dtype=bf16, device="cuda"), W_gate=torch.zeros((24, 64), dtype=bf16, device="cuda"),
                 W_up=torch.zeros((24, 64), dtype=bf16, device="cuda"), dH=torch.zeros((4, 24), dtype=bf16, device="cuda"),
                 H=torch.zeros((4, 24), dtype=bf16, device="cuda"))
        t["pre"] = cam.gated_ffn(t["X"], t["W_gate"], t["W_up"], want_pre=True)[1]
        return t

    def call(t):
        if name == "H":
            return cam.gated_ffn(t["X"], t["W_gate"], t["W_up"], H=t["H"])
        return cam.gated_ffn_backward(t["X"], t["W_gate"], t["W_up"], t["dH"], pre=t["pre"])
    call(tensors())
    torch.cuda.synchronize()
    good = tensors()[name]
    for how, bad in (("host", good.cpu()), ("type", good.to(torch.float64)), ("short", good[:3]), ("apart", torch.cat([good, good], -1)[..., ::2])):
        t = tensors()
        t[name] = bad
        # of X, which the others are compared with, a row less or another type is found at one of them
        match = {("X", "short"): "dH", ("X", "type"): "dtype"}.get((name, how), f"{name}:")
        if name in ("W_gate", "W_up") and how == "short":
            match = "W_gate / W_up"
        with pytest.raises((binding.CameraError, TypeError, ValueError), match=match):
            call(t)
