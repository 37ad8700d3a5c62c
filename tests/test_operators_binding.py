"""What the binding hands to the library of the tensors that it is given, without a GPU: the library's call is replaced by one that
notes its arguments."""
import pytest
import torch

from paper_2508_02322_amd import binding


class Noted:
    def __init__(self, lib):
        self.lib, self.args = lib, None

    def camera_gated_ffn(self, ctx, stream, X, dtype, n, d_model, ldx, W_gate, W_up, d_ff, H, ldh, pre):
        self.args = dict(n=n, d_ff=d_ff, H=H, ldh=ldh)
        return 0

    def __getattr__(self, name):
        return getattr(self.lib, name)


@pytest.fixture()
def host(monkeypatch):
    cam = binding.Camera(device=0)
    cam.device = torch.device("cpu")
    cam.lib = Noted(cam.lib)
    monkeypatch.setattr(binding, "_stream_handle", lambda device: 0)
    return cam


def block(n, d_ff, dtype):
    X, W = torch.zeros((n, 64), dtype=dtype), torch.zeros((d_ff, 64), dtype=dtype)
    return X, W, W.clone()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d_ff", [64, 24, 20, 13])
def test_a_given_block_is_not_written_beyond_its_buffer(host, d_ff, dtype):
    """Rows that lie on each other (a stride of 0, or one shorter than they are) have no room of their own: the stride that reaches the
    library is theirs, and the library refuses it, or the binding does."""
    n, v = 4, 128 // torch.finfo(dtype).bits
    whole = -(-d_ff // v) * v
    one_row = torch.zeros((1, whole), dtype=dtype)
    for H in (one_row[:, :d_ff].expand(n, d_ff), torch.zeros(4 * whole, dtype=dtype).as_strided((n, d_ff), (v, 1)),
              torch.zeros(4 * whole, dtype=dtype).as_strided((n, d_ff), (1, 1)), torch.zeros((n, whole), dtype=dtype)[:, :d_ff],
              torch.zeros((n, whole + v), dtype=dtype)[:, :d_ff], torch.zeros((n, whole + 3), dtype=dtype)[:, :d_ff]):
        host.lib.args = None
        try:
            host.gated_ffn(*block(n, d_ff, dtype), H=H)
        except binding.CameraError:
            continue
        a = host.lib.args
        refused = a["ldh"] < d_ff or a["ldh"] % v != 0           # the library's own check of ldh
        room = H.untyped_storage().nbytes() // H.element_size() - H.storage_offset()
        assert refused or (n - 1) * a["ldh"] + whole <= room, (tuple(H.stride()), a["ldh"])
        assert refused == (H.stride(0) < d_ff or H.stride(0) % v != 0)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_single_row_has_no_stride(host, dtype):
    """Whatever torch leaves as the stride of one row: its address counts, and that a whole number of vectors fits behind it."""
    v = 128 // torch.finfo(dtype).bits
    for d_ff in (20, 13, 24):
        whole = -(-d_ff // v) * v
        buf = torch.zeros(whole, dtype=dtype)
        for stride in (0, 1, d_ff, whole, 67):
            host.gated_ffn(*block(1, d_ff, dtype), H=buf.as_strided((1, d_ff), (stride, 1)))
            assert host.lib.args["ldh"] >= d_ff and host.lib.args["ldh"] % v == 0, stride
        if whole > d_ff:
            with pytest.raises(binding.CameraError, match="last row"):
                host.gated_ffn(*block(1, d_ff, dtype), H=torch.zeros(d_ff, dtype=dtype).view(1, d_ff))
    host.gated_ffn(*block(0, 13, dtype), H=torch.zeros((0, 13), dtype=dtype))
    assert host.lib.args["ldh"] % v == 0
