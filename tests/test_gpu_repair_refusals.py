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
