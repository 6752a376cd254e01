"""The calls of ``train`` by name and with the stream by place, on the GPU."""
import inspect

import pytest
import torch

from paper_2512_05831_amd import train

pytestmark = pytest.mark.gpu


def calls(device):
    g = torch.Generator(device=device).manual_seed(1)
    x, y = torch.randn(6, 40, generator=g, device=device), torch.randn(6, 40, generator=g, device=device)
    mean, rstd = torch.zeros(6, device=device), torch.ones(6, device=device)
    slots = torch.arange(6, dtype=torch.int32, device=device).view(3, 2)
    return [(train.layer_norm, dict(x=x, weight=None, statistics=True)), (train.layer_norm_backward, dict(dy=y, x=x, rstd=rstd, mean=mean)),
            (train.activation, dict(v=x)), (train.activation_backward, dict(dh=y[:, :20], v=x)),
            (train.dispatch, dict(x=x, tokens=slots.view(-1))), (train.combine, dict(y=x, slots=slots)),
            (train.combine_backward, dict(dout=y[:3], y=x, slots=slots)), (train.weight_gradient, dict(dy=y.half(), x=x.half()))]


def tensors(r):
    return [t for t in (r if isinstance(r, tuple) else (r,)) if t is not None]


@pytest.mark.parametrize("which", range(8))
def test_the_same_however_they_are_given(which, device):
    call, kw = calls(device)[which]
    want = tensors(call(*kw.values()) if call not in (train.layer_norm, train.layer_norm_backward) else call(**kw))
    torch.cuda.synchronize()
    side = torch.cuda.Stream(device)
    parameters = list(inspect.signature(call).parameters.values())
    assert parameters[-1].name == "stream"
    placed = [kw.get(p.name, p.default) for p in parameters[:-1]]
    with_stream = call(*placed, side)
    side.synchronize()
    first = parameters[0].name
    rest = {k: v for k, v in kw.items() if k != first}
    for got in (call(**kw), call(kw[first], **rest), call(*placed), call(*placed, stream=None), call(*placed, None), with_stream):
        torch.cuda.synchronize()
        got = tensors(got)
        assert len(got) == len(want) and all(torch.equal(a, b) for a, b in zip(got, want))
