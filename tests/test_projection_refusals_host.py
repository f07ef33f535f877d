"""A sampler's steps refuse a projection that does not fit before anything of the step is launched, dense ones as sparse ones (without a GPU: the layer
has nothing but its shape, so that any launch would fail in another way)."""
import types

import pytest

from paper_2506_23858_b200 import binding as vb
from paper_2506_23858_b200.layer import SteppedAttention, VmobaLayer


def stepped():
    layer = VmobaLayer.__new__(VmobaLayer)
    layer.shape = vb.make_shape(1, 2, 64, (2, 4, 4), (1, 2, 2), "bf16")
    s = SteppedAttention.__new__(SteppedAttention)
    s.layer, s.tau, s.schedule, s._one_block = layer, 0.5, [True, False], layer.shape
    return s


def linear(*args, **kw):
    return types.SimpleNamespace(shape=vb.make_linear_shape(*args, **kw))


@pytest.mark.parametrize("step", [0, 1])
@pytest.mark.parametrize("projection,projected", [
    (linear(1, 32, 128, 64, "bf16", heads=2), None),
    (linear(1, 32, 128, 64, "bf16", heads=2), {"bias": 1}),
    (linear(1, 32, 128, 64, "bf16"), {"weight": 1}),
    (linear(1, 32, 128, 64, "f32", heads=2), {"weight": 1}),
    (linear(2, 32, 128, 64, "bf16", heads=2), {"weight": 1}),
    (linear(1, 32, 128, 64, "bf16", heads=1), {"weight": 1}),
])
def test_a_projection_that_does_not_fit_is_refused_first(step, projection, projected):
    with pytest.raises(ValueError):
        stepped().forward(step, None, None, None, None, projection=projection, projected=projected)
