"""A weight is mostly a torch.nn.Parameter: its calls go the short way too, and are the same."""
from __future__ import annotations

import pytest
import torch

import paper_2607_20538_gb300 as cg
from test_short_calls import ARGS, KW, NAMES, PYTHON, calls  # noqa: F401  (a fixture)


@pytest.mark.parametrize("name", NAMES)
def test_same_call(name, calls):  # noqa: F811
    kw = KW[name]()
    short, python = calls.both(name, kw, PYTHON[name])
    for key, value in kw.items():
        if not isinstance(value, torch.Tensor):
            continue
        one = dict(kw, **{key: torch.nn.Parameter(value, requires_grad=False)})
        got, longer = calls.both(name, one, PYTHON[name])
        assert len(got) == 1 and got == longer == short == python, key


def test_other_subclasses_take_the_longer_way(calls):  # noqa: F811
    class Other(torch.Tensor):
        pass

    class Weight(torch.nn.Parameter):
        pass

    kw = KW["block8_matmul"]()
    for t in (Other, Weight):
        assert calls.module.block8_matmul(*ARGS["block8_matmul"](dict(kw, w=kw["w"].as_subclass(t)))) is None


def test_a_parameter_that_does_not_fit(calls):  # noqa: F811
    kw = KW["block8_matmul"]()
    wrong = torch.nn.Parameter(torch.empty(130, 256, dtype=kw["w"].dtype), requires_grad=False)
    assert calls.module.block8_matmul(*ARGS["block8_matmul"](dict(kw, w=wrong))) is None
    with pytest.raises(cg.CodecGaugeError, match="w:"):
        cg.block8_matmul(**dict(kw, w=wrong))
