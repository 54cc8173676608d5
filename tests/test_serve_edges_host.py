"""Calls of the long-context operators that do nothing or are refused, without
a GPU: none gets as far as a HIP call."""
import ctypes

import pytest

mlkv = pytest.importorskip("paper_2406_09297_amd")
torch = pytest.importorskip("torch")

P = 0x10000  # stands for device memory: 16-byte aligned, never read


def test_a_prefill_of_no_tokens_needs_no_tensors():
    """A tensor of T = 0 tokens has no address."""
    mp = mlkv.Map.uniform(12, 12, 4, 1)
    cache = ctypes.byref(mlkv._Cache(P, P, 4, 2, 64, 64))
    assert torch.empty((2, 0, 12, 64)).data_ptr() == 0
    f = mlkv.lib().mlkv_prefill_attention_window
    assert f(0, None, cache, mp.handle, None, 0, 8, 1, None, 0, None) == mlkv.MLKV_OK
    for args in ((12, 0, 8, 0), (0, 0, -1, 0), (0, 0, 8, 7)):  # layer, T, window, out_dtype
        layer, T, window, dtype = args
        assert mlkv.STATUS_NAMES[f(layer, None, cache, mp.handle, None, T, window, 1, None, dtype,
                                   None)] == "MLKV_ERR_INVALID_ARG"
