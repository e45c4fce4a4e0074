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


# ----------------------------------------------------------------------------- scales of activations
def storage_end(t: torch.Tensor) -> int:
    return t.untyped_storage().nbytes() // t.element_size() - t.storage_offset()


@pytest.mark.parametrize("nb,T", ((1, 1), (1, 4), (2, 5), (3, 7), (64, 130)))
def test_rows_of_activation_scales_are_whole(nb, T):
    """The product copies scales in groups of four: the last row too has to be there up to a multiple of 4."""
    up = -(-T // 4) * 4
    made = cq._act_scale(nb, T, "cpu")
    assert made.shape == (nb, T) and made.stride() == (up, 1) and storage_end(made) >= nb * up
    assert cq._whole_rows(made) is made
    short = torch.empty_strided((nb, T), (up, 1))
    short.copy_(torch.arange(nb * T).view(nb, T))
    whole = cq._whole_rows(short)
    assert torch.equal(whole, short) and whole.stride(0) % 4 == 0 and storage_end(whole) >= (nb - 1) * whole.stride(0) + up
    assert (whole is short) == (T == up)
    wide = torch.zeros(nb, up + 4)[:, :T]
    assert cq._whole_rows(wide) is wide


# ----------------------------------------------------------------------------- workspaces
def test_a_workspace_has_to_be_contiguous_memory_of_the_calls_device():
    here = torch.zeros(64, dtype=torch.float32)
    assert cq._workspace_of(here, -1) == (here.data_ptr(), 256)          # bytes, whatever the type
    for bad, dev in ((here, 0), (here[::2], -1), (torch.zeros(1).expand(1 << 20), -1)):
        with pytest.raises(ValueError):
            cq._workspace_of(bad, dev)


# ----------------------------------------------------------------------------- shapes of a cache
@pytest.mark.parametrize("page_size,heads,head_dim,bits", ((16, 2, 80, 8), (16, 2, 256, 8), (16, 2, 65, 4), (16, 2, 129, 4), (16, 2, 0, 8),
                                                           (8, 2, 64, 8), (24, 2, 64, 8), (8192, 2, 64, 8), (0, 2, 64, 8), (16, 0, 64, 8),
                                                           (16, 5000, 64, 8)))
def test_a_cache_of_a_shape_that_no_call_takes_is_refused_when_it_is_made(page_size, heads, head_dim, bits):
    with pytest.raises(cq.CQError) as e:
        cq.KVCache.empty(2, page_size, heads, head_dim, bits, device="cpu")
    assert e.value.status == 2
    if head_dim % 2 == 0:
        codes = torch.zeros(2, heads, page_size, head_dim if bits == 8 else head_dim // 2, dtype=torch.int8 if bits == 8 else torch.uint8)
        scale = torch.zeros(2, heads, page_size)
        with pytest.raises(cq.CQError):
            cq.KVCache(codes, codes, scale, scale, bits)


def test_a_cache_of_more_rows_than_a_call_can_count_is_refused_when_it_is_made():
    with pytest.raises(cq.CQError):
        cq.KVCache.empty(1 << 26, 16, 2, 64, device="meta")


# ----------------------------------------------------------------------------- pitches
def test_the_pitch_of_a_single_row_does_not_matter():
    codes = torch.zeros(4, 264, dtype=torch.uint8).view(torch.float8_e4m3fn)
    assert cq._codes_pitch(codes[:1, :100], 1, 100, -1, "a") == 112
    assert cq._codes_pitch(codes[:, :100], 4, 100, -1, "a") == 264         # the library refuses this one
    scale = torch.zeros(3, 9)
    assert cq._act_scale_pitch(scale[:1, :5], 1, 5, -1, "a") == 8
    assert cq._act_scale_pitch(scale[:, :5], 3, 5, -1, "a") == 9
