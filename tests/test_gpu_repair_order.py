"""The order of the sums over a row, as far as the calls promise it."""
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,vocab", [(3, 9001), (1024, 3001), (1024, 16384), (1030, 17001)])
def test_sums_do_not_depend_on_the_alternatives(cam, n, vocab, dtype):
    """The same to the last bit with any number of alternatives up to 64, and with any beyond; on rows of another kind than many short
    ones, with any at all."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    z = (3 * torch.randn((n, vocab), generator=gen, device="cuda")).to(TYPES[dtype])
    targets = torch.randint(0, vocab, (n,), generator=gen, device="cuda").int()
    out = {k: cam.token_logprobs(z, targets, top_k=k) for k in (0, 1, 20, 64, 65, 128, 256)}
    torch.cuda.synchronize()
    short = n >= 1024 and vocab <= 16384
    for k, o in out.items():
        same = out[65 if short and k > 64 else 0]
        for key in ("logprob", "entropy", "stats"):
            assert torch.equal(o[key], same[key]), (k, key)
        if k:
            assert torch.equal(o["top_logprob"], out[256]["top_logprob"][:, :k]) or (short and k <= 64), k
            assert torch.equal(o["top_idx"], out[256]["top_idx"][:, :k]), k
