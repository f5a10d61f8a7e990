"""A call's tensors, its workspace and its stream are on one device, the current one: anything else is refused before a kernel could
be given another device's memory.  Tensors without memory (FakeTensor) stand for those of a second GPU."""
import pytest
import torch
from torch._subclasses import fake_tensor

from paper_2605_01255_b200 import binding as B

from test_host_calls import OPS, built, calls  # noqa: F401


@pytest.fixture
def on(monkeypatch):
    """on(device): the operators' arguments as test_host_calls makes them, on a device that need not exist."""
    monkeypatch.setattr(fake_tensor, "init_gpu_context", lambda device: None, raising=False)

    def make(device):
        with fake_tensor.FakeTensorMode():
            return calls(device), torch.empty(1 << 20, dtype=torch.uint8, device=device)

    return make


@pytest.mark.parametrize("op", OPS)
def test_a_tensor_on_another_device_is_refused(op, on):
    f, desc, args, kw = on("cuda:0")[0][op]
    others, ws = on("cuda:1")
    _, _, other, other_kw = others[op]
    for name in args:
        with pytest.raises(ValueError, match=r"cuda:[01], the tensors before it on cuda:[01]"):
            f(desc, *[other[k] if k == name else a for k, a in args.items()], **kw)
    for name, t in kw.items():
        if isinstance(t, torch.Tensor):
            with pytest.raises(ValueError, match="on cuda:"):
                f(desc, *args.values(), **dict(kw, **{name: other_kw[name]}))
    if op in (5, 6, 7):
        with pytest.raises(ValueError, match="workspace is on cuda:1"):
            f(desc, *args.values(), **dict(kw, ws=ws))


class Stream:
    cuda_stream, device_index = 0, 1


@pytest.mark.parametrize("op", OPS)
def test_a_stream_of_another_device_is_refused(op, on):
    f, desc, args, kw = on("cuda:0")[0][op]
    with pytest.raises(ValueError, match="stream is on cuda:1, the tensors on cuda:0"):
        f(desc, *args.values(), **dict(kw, stream=Stream()))


@pytest.mark.gpu
@pytest.mark.parametrize("op", OPS)
def test_tensors_of_a_device_that_is_not_current_are_refused(op, on):
    assert torch.cuda.current_device() == 0
    f, desc, args, kw = on("cuda:1")[0][op]
    launches = B.acx_kernel_launches()
    for stream in (None, Stream()):
        with pytest.raises(ValueError, match="the tensors are on cuda:1, the current device is cuda:0"):
            f(desc, *args.values(), **dict(kw, stream=stream))
    assert B.acx_kernel_launches() == launches
