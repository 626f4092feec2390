"""A KVCache is of the tensor and sizes that it was made of, for good: the calls go by a
description made of them, and another tensor in their place would leave it pointing at
memory that may have been freed."""

import copy

import pytest
import torch


@pytest.fixture()
def cache(duo_lib):
    data = torch.zeros((5, 2, duo_lib.kv_page_bytes(32, 2, 64, "int4") // 2), dtype=torch.uint8)
    return duo_lib.KVCache(data, 32, 2, 64, "int4")


@pytest.mark.parametrize("name,value", [("data", torch.zeros(1, dtype=torch.uint8)), ("page_size", 16), ("kv_heads", 1),
                                        ("head_dim", 128), ("fmt", "bf16")])
def test_nothing_can_be_replaced(cache, name, value):
    before = getattr(cache, name)
    with pytest.raises(AttributeError):
        setattr(cache, name, value)
    assert getattr(cache, name) is before


def test_description(cache):
    for c in (cache, copy.copy(cache)):
        assert (c.page_size, c.kv_heads, c.head_dim, c.fmt) == (32, 2, 64, "int4")
        assert c.c.data == c.data.data_ptr() == cache.data.data_ptr()
        assert (c.c.num_pages, c.c.page_size, c.c.kv_heads, c.c.head_dim, c.c.format) == (5, 32, 2, 64, 2)
