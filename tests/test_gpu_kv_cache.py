"""KVCodes keeps the tensors that the library was told of."""
import pytest
import torch

import paper_1402_3788_amd as km

pytestmark = pytest.mark.gpu

BF = torch.bfloat16
NAMES = ("k_centres", "v_centres", "k_codes", "v_codes")


def make():
    dev = torch.device("cuda:0")
    g = torch.Generator().manual_seed(0)
    centres = [torch.randn(2, 16, 256, 4, generator=g).to(BF).to(dev) for _ in range(2)]
    return km.KVCodes.empty(*centres, 3, 16)


@pytest.mark.parametrize("name", NAMES)
def test_another_tensor_in_its_place_is_refused(name):
    cache = make()
    was = getattr(cache, name)
    with pytest.raises(AttributeError, match="another"):
        setattr(cache, name, was.clone())
    assert getattr(cache, name) is was
    setattr(cache, name, was)                   # as `cache.k_codes += 1` ends
    with pytest.raises(AttributeError):
        delattr(cache, name)


@pytest.mark.parametrize("name,value", [("pages", 1 << 20), ("page", 64), ("heads", 4), ("dim", 128),
                                        ("sub", 8), ("K", 3), ("dtype", torch.float16),
                                        ("device", torch.device("cpu")), ("index", -1)])
def test_sizes_are_what_the_library_was_told(name, value):
    cache = make()
    was = getattr(cache, name)
    with pytest.raises(AttributeError, match="another"):
        setattr(cache, name, value)
    assert getattr(cache, name) == was


def test_written_to_in_place():
    cache = make()
    slots = torch.arange(48, device="cuda:0")
    cache.k_codes += 7
    cache.v_codes.fill_(9)
    cache.k_centres *= 2
    k, v = km.kmeans_kv_read(cache, slots)
    assert torch.equal(k, cache.k_centres[:, :, 7].reshape(1, 2, 64).expand(48, 2, 64))
    assert torch.equal(v, cache.v_centres[:, :, 9].reshape(1, 2, 64).expand(48, 2, 64))
