"""The operators between hidden states and tokens take tensors of the GPU that the call runs on: the stream's where one is given, else the current
one.  With stand-ins for tensors and streams of two GPUs, on the host; and what the stand-ins stand for, on the GPU."""
import pytest
import torch

import paper_2605_06534_amd as R
from paper_2605_06534_amd import binding


class Of:
    """A tensor, or a stream, of a GPU."""

    def __init__(self, gpu):
        self.gpu = gpu

    def get_device(self):
        return self.gpu


@pytest.fixture
def two_gpus(monkeypatch):
    monkeypatch.setattr(binding, "_gpus", 2)
    monkeypatch.setattr(binding, "_device_of", lambda stream: 0 if stream is None else stream.gpu, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0)


@pytest.mark.parametrize("stream,tensors,fine", [
    (None, (0, 0), True), (None, (1, 1), False), (None, (0, 1), False), (None, (0, None, 0), True), (0, (0, 0), True), (0, (1, 1), False), (0, (0, 1), False),
    (1, (1, 1), True), (1, (0, 0), False), (1, (1, 0), False), (1, (0, 1), False), (1, (1, None, 1), True)], ids=str)
def test_tensors_of_the_stream_s_gpu(two_gpus, stream, tensors, fine):
    call = lambda: binding._one_device("norm", None if stream is None else Of(stream), *(None if t is None else Of(t) for t in tensors))  # noqa: E731
    if fine:
        call()
        return
    with pytest.raises(R.RoseError) as e:
        call()
    assert e.value.status == binding.ERR_SHAPE


@pytest.mark.gpu
def test_the_gpu_of_a_stream():
    print("case: streams' GPU", flush=True)
    here = torch.cuda.current_device()
    for stream in (None, torch.cuda.Stream(), torch.cuda.current_stream(), torch.cuda.default_stream(), torch.cuda.Stream().cuda_stream, 0):
        assert binding._device_of(stream) == here


@pytest.mark.gpu
def test_calls_on_a_stream_of_another_gpu_are_refused(monkeypatch):
    print("case: a stream of another GPU", flush=True)
    g = dict(device="cuda")
    x, w, f, ws = torch.ones(4, 8, **g), torch.ones(8, **g), torch.ones(4, **g), torch.empty(1 << 20, dtype=torch.uint8, **g)
    ids, t, u = torch.zeros(4, 3, dtype=torch.int64, **g), torch.zeros(4, 3, **g), torch.zeros(4, **g)
    tokens, offsets, out, accepted = torch.zeros(3, dtype=torch.int64, **g), torch.tensor([0, 3], **g), torch.zeros(4, dtype=torch.int64, **g), torch.zeros(1, dtype=torch.int32, **g)
    a = R.Adapters(torch.zeros(2, 3, 8, dtype=torch.bfloat16, **g), torch.zeros(2, 5, 3, dtype=torch.bfloat16, **g))
    chosen, o, d = torch.zeros(4, dtype=torch.int32, **g), torch.zeros(4, 5, **g), torch.zeros(4, 8, **g)
    calls = (lambda s: R.layer_norm(x, w, d, stream=s), lambda s: R.layer_norm_grad(x, x, w, f, d, w.clone(), ws, stream=s),
             lambda s: R.distill_loss(x, ids, t, f, f.clone(), ws, stream=s), lambda s: R.distill_grad(x, ids, t, f, f, d, stream=s),
             lambda s: R.distill_loss_grad(x, ids, t, f, f.clone(), f.clone(), d, ws, stream=s),
             lambda s: R.draft_verify(x, None, tokens, offsets, u, out, accepted, ws, stream=s), lambda s: R.adapter_linear(x.bfloat16(), a, chosen, o, ws, stream=s))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    monkeypatch.setattr(binding, "_gpus", 2)
    for call in calls:                            # (of this one they are not)
        call(stream)
        call(None)
    torch.cuda.synchronize()
    monkeypatch.setattr(binding, "_device_of", lambda stream: 1)
    for call in calls:
        with pytest.raises(R.RoseError) as e:
            call(stream)
        assert e.value.status == binding.ERR_SHAPE
