"""The calls of ``train`` take their arguments by name and by place, as their signatures show them (no GPU: all are refused
for tensors that are not on one, after their arguments are bound)."""
import inspect

import pytest
import torch

from paper_2512_05831_amd import train

CALLS = [train.layer_norm, train.layer_norm_backward, train.activation, train.activation_backward, train.dispatch, train.combine,
         train.combine_backward, train.weight_gradient]


@pytest.mark.parametrize("call", CALLS, ids=lambda f: f.__name__)
def test_by_name_and_by_place(call):
    x = torch.zeros(4, 8)
    parameters = inspect.signature(call).parameters
    needed = [name for name, p in parameters.items() if p.default is p.empty]
    for named in range(len(needed) + 1):  # the last so many by name
        args, kw = [x] * (len(needed) - named), {name: x for name in needed[len(needed) - named:]}
        for also in ({}, {"stream": None}):
            with pytest.raises(ValueError, match="expected device tensors"):
                call(*args, **kw, **also)
    # all by place, the stream among them
    with pytest.raises(ValueError, match="expected device tensors"):
        call(*([x] * len(needed)), *(p.default for p in list(parameters.values())[len(needed):]))
    with pytest.raises(TypeError, match="missing"):
        call()
    with pytest.raises(TypeError, match="unexpected keyword"):
        call(*([x] * len(needed)), nothing=1)
    with pytest.raises(TypeError, match="multiple values"):
        call(*([x] * len(needed)), **{needed[0]: x})
    with pytest.raises(TypeError):
        call(*([x] * (len(parameters) + 1)))
