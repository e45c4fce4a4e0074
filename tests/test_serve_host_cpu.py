"""Host-side rules of the serving operators that need no GPU: what the binding and the layer refuse, fix or allocate."""
from __future__ import annotations

import copy

import pytest
import torch

from paper_2410_07505_b200 import cq


# ----------------------------------------------------------------------------- cache
FIELDS = ("k_codes", "v_codes", "k_scale", "v_scale", "k_col", "v_col", "bits", "pages", "page_size", "heads", "head_dim", "device")


@pytest.mark.parametrize("name", FIELDS)
def test_a_caches_fields_cannot_be_replaced(name):
    """The calls use addresses taken when the cache is made: a replaced tensor would be ignored and the old one's memory freed."""
    cache = object.__new__(cq.KVCache)
    with pytest.raises(AttributeError):
        setattr(cache, name, torch.zeros(1))
    with pytest.raises(AttributeError):
        delattr(cache, name)


def test_a_cache_cannot_be_copied():
    """A copy would hold new tensors and the old ones' addresses."""
    cache = object.__new__(cq.KVCache)
    object.__setattr__(cache, "k_codes", torch.zeros(2))
    object.__setattr__(cache, "_args", (1, 2))
    for how in (copy.copy, copy.deepcopy):
        with pytest.raises((AttributeError, TypeError)):
            how(cache)
