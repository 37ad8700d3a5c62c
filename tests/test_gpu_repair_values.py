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
