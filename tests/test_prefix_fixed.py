"""What a Prefix or Rotary was made of cannot be replaced behind the library's back: its structure holds the first one's address and size."""
import pytest
import torch

import paper_2407_11550_amd as adakv
from paper_2407_11550_amd import binding


@pytest.fixture
def made(lib, monkeypatch):
    monkeypatch.setattr(binding, "_ptr", lambda t, name, dtype=None: t.data_ptr())     # (host tensors: nothing is called with them)
    layer = adakv.Layer(torch.bfloat16, 8, 2, 64, 1, 7, 0.2, [5], [12])
    K = torch.zeros(12, 64, dtype=torch.bfloat16)
    prefix = adakv.Prefix(layer, torch.zeros(3, dtype=torch.int32), 0, K, K.clone(), torch.zeros(2, dtype=torch.int32), [0, -1, 0])
    return prefix, adakv.Rotary(64, freq=torch.ones(32, dtype=torch.float64))


def test_sequences_of_a_prefix(made):
    """A longer list would let a layer of more sequences through than the library's array has."""
    prefix, _ = made
    assert list(prefix.of) == [0, -1, 0]
    with pytest.raises(AttributeError):
        prefix.of.append(0)
    with pytest.raises(AttributeError):
        prefix.of = [0] * 64
    assert len(prefix.of) == len(prefix._of) == 3


def test_tensors(made):
    prefix, rotation = made
    with pytest.raises(TypeError):
        prefix.tensors["K_cache"] = torch.zeros(12, 64, dtype=torch.bfloat16)
    for x, name in ((prefix, "tensors"), (prefix, "headroom"), (prefix, "layer"), (rotation, "freq"), (rotation, "dims"), (rotation, "magnitude")):
        with pytest.raises(AttributeError):
            setattr(x, name, None)
    assert rotation.c.freq == rotation.freq.data_ptr() and prefix.c.K_cache == prefix.tensors["K_cache"].data_ptr()
