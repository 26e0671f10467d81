"""A workspace that is not what the kernels take for one, on another device or with gaps between its elements, is refused by every call
of the binding before the library is reached."""
import pytest
import torch

from paper_2512_06989_amd import mhffn


def calls(device):
    t = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device=device)  # noqa: E731
    X, P, W, Wr = t(8, 256), t(256, 256), [t(2, 3, 64, 128) for _ in range(3)], t(2, 128, 3)
    return {"forward": lambda ws: mhffn.forward(X, *W, Wr, workspace=ws),
            "backward": lambda ws: mhffn.backward(X, *W, Wr, X, workspace=ws),
            "reference_unfused": lambda ws: mhffn.reference_unfused(X, *W, Wr, workspace=ws),
            "module_forward": lambda ws: mhffn.module_forward(X, P, *W, Wr, P, workspace=ws),
            "module_backward": lambda ws: mhffn.module_backward(X, P, *W, Wr, P, X, X, X, workspace=ws),
            "linear_forward": lambda ws: mhffn.linear_forward(X, P, workspace=ws),
            "linear_backward": lambda ws: mhffn.linear_backward(X, P, X, workspace=ws)}


CALLS = ("forward", "backward", "reference_unfused", "module_forward", "module_backward", "linear_forward", "linear_backward")


@pytest.mark.parametrize("name", CALLS)
def test_another_device(name):
    with pytest.raises(ValueError, match="workspace is on meta, expected cpu"):
        calls("cpu")[name](torch.empty(1 << 20, dtype=torch.uint8, device="meta"))


@pytest.mark.parametrize("name", CALLS)
def test_gaps(name):
    for ws in (torch.zeros(1, dtype=torch.uint8).expand(1 << 20), torch.zeros(1 << 12, 2, dtype=torch.uint8)[:, 0]):
        with pytest.raises(ValueError, match="workspace must be contiguous"):
            calls("cpu")[name](ws)


@pytest.mark.gpu
@pytest.mark.parametrize("name", CALLS)
def test_host_memory(name):
    call = calls("cuda")[name]
    with pytest.raises(ValueError, match="workspace is on cpu, expected cuda:0"):
        call(torch.empty(1 << 20, dtype=torch.uint8))
    call(torch.empty(1 << 24, dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
