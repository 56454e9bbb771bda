"""Kv4Cache holds on to the tensors that its calls use, on one device (no GPU: tensors that say they are on one)."""
import pytest
import torch


def made(device_of, slots=64):
    """The four tensors of a cache of 1 kv head of 64, each of which reports a device."""
    class OnDevice(torch.Tensor):
        is_cuda = property(lambda self: True)
        device = property(lambda self: torch.device(device_of[id(self)]))

    names, out = [], []
    for i, (width, dtype) in enumerate(((32, torch.uint8), (2, torch.int16)) * 2):
        t = torch.zeros(1, 1, slots, width, dtype=dtype).as_subclass(OnDevice)
        names.append(id(t))
        out.append(t)
    return names, out


@pytest.fixture(autouse=True)
def lib():
    from paper_2607_15865_gb300 import build
    build.build()


def test_its_tensors_cannot_be_replaced():
    from paper_2607_15865_gb300.kv4 import Kv4Cache
    where = {}
    ids, t = made(where)
    where.update({i: "cuda:0" for i in ids})
    c = Kv4Cache(64, *t)
    for name, mine in zip(("k_codes", "k_scales", "v_codes", "v_scales"), t):
        with pytest.raises(AttributeError):
            setattr(c, name, mine.clone())
        assert getattr(c, name) is mine and getattr(c.struct, name) == mine.data_ptr()


@pytest.mark.parametrize("other", range(4))
def test_tensors_of_two_devices_are_refused(other):
    from paper_2607_15865_gb300.kv4 import Kv4Cache
    where = {}
    ids, t = made(where)
    where.update({i: "cuda:0" for i in ids})
    Kv4Cache(64, *t)
    where[ids[other]] = "cuda:1"
    with pytest.raises(ValueError, match="cuda:1"):
        Kv4Cache(64, *t)
