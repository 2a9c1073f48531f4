"""The native module takes no object for one of another class: what it would read as a descriptor is somebody else's memory."""
import ctypes

import pytest

import paper_2602_05367_b200 as rabit
from paper_2602_05367_b200 import binding


def _made(cls, **attributes):
    """An object of the class without a device: its address is that of zeros."""
    o = cls.__new__(cls)
    memory = ctypes.create_string_buffer(4096)
    for name in attributes.pop("addresses"):
        setattr(o, name, ctypes.addressof(memory))
    for name, v in dict(attributes, _keep=memory, _device=0, dev_buf=None, _handle=None, N=32, M=32, rank=1).items():
        setattr(o, name, v)
    return o


ADAPTERS = _made(rabit.RabitAdapters, addresses=["_addr"])
GRADIENTS = _made(rabit.RabitGradients, addresses=["_gradients_addr"])
GRADIENTS.free = lambda: None
LAYER = _made(rabit.RabitLayer, addresses=["_layer_addr"])


@pytest.mark.parametrize("other", [ADAPTERS, LAYER, None, 7], ids=["adapters", "layer", "None", "int"])
def test_clipping_needs_gradients(other):
    with pytest.raises(TypeError, match="RabitGradients"):
        rabit.rabit_clip_gradients(other, 1.0, None, 0)


@pytest.mark.parametrize("other", [GRADIENTS, LAYER, None], ids=["gradients", "layer", "None"])
def test_factor_gradients_need_adapters(other):
    with pytest.raises(TypeError, match="RabitAdapters"):
        rabit.rabit_adapter_gradients(other, None, None, None, None, None)


@pytest.mark.parametrize("other", [ADAPTERS, GRADIENTS, None], ids=["adapters", "gradients", "None"])
def test_calls_of_layers_need_layers(other):
    with pytest.raises(TypeError, match="RabitLayer"):
        rabit.rabit_linear_group([other], [None], [None])
    with pytest.raises(TypeError, match="RabitLayer"):
        rabit.rabit_linear_group_adapted([other], [None], [None], None, [None])


def test_what_was_freed_is_said_to_be():
    layer = _made(rabit.RabitLayer, addresses=[])
    layer._layer_addr = None
    with pytest.raises(binding.RabitError, match="freed"):
        rabit.rabit_linear_group([layer], [None], [None])
