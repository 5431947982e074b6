"""A PagedCache works on the tensors that it was made around: it keeps them, and another one in their place is refused."""
import gc
import weakref

import pytest
import torch


@pytest.fixture(scope="module")
def a2sf():
    from paper_2407_20485_b200 import build

    build.build()
    from paper_2407_20485_b200 import binding

    return binding


NAMES = ("k_pages", "v_pages", "scores", "positions", "page_table", "past", "start")


@pytest.mark.parametrize("name", NAMES)
def test_a_tensor_is_not_replaced(a2sf, name):
    """The kernels have its address: another tensor would be ignored, and the old one's memory given to somebody else."""
    cache = a2sf.PagedCache(2, 3, 64, torch.bfloat16, 16, 10, 4, device="cpu")
    old = getattr(cache, name)
    with pytest.raises(AttributeError, match=name):
        setattr(cache, name, torch.zeros_like(old))
    with pytest.raises(AttributeError, match=name):
        delattr(cache, name)
    assert getattr(cache, name) is old
    seen = weakref.ref(old)
    del old
    gc.collect()
    assert seen() is not None


def test_tensors_change_in_place(a2sf):
    cache = a2sf.PagedCache(2, 3, 64, torch.bfloat16, 16, 10, 4, device="cpu")
    at = cache.past.data_ptr()
    cache.past += 3
    cache.past.add_(1)
    cache.scores *= 0.5
    cache.page_table[1] = 2
    cache.note = "other attributes are free"
    assert cache.past.tolist() == [4, 4] and cache.past.data_ptr() == at and cache.page_table[1].tolist() == [2] * 4
