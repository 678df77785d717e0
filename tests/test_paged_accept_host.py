"""Acceptance of draft trees: caches of more heads than it counts in (no GPU; nothing is launched)."""
import ctypes

import pytest

from tests.test_paged_host import ARG, X, _batch, _cache, lib  # noqa: F401


@pytest.mark.parametrize("heads", [2 ** 20 + 1, 2 ** 23, 2 ** 24, 2 ** 31 - 1])
def test_heads_beyond_the_count(lib, heads):  # noqa: F811
    """With 2^23 heads of 128 fp32 a row's units passed 2^31, and no key was moved."""
    cache = _cache(n_kv_heads=heads, page_size=1, head_stride=128, token_stride=128, page_stride=128 * heads)
    assert lib.esp_paged_accept(4, ctypes.byref(cache), ctypes.byref(_batch()), X, X, X, X, None, 4, X, 7 * X, None) == ARG
    # none to look at: what is refused does not go by that
    assert lib.esp_paged_accept(4, ctypes.byref(cache), ctypes.byref(_batch(batch=0)), X, X, X, X, None, 4, X, 7 * X, None) == ARG


def test_as_many_as_the_append_takes(lib):  # noqa: F811
    cache = _cache(n_kv_heads=2 ** 20, page_size=1, head_stride=128, token_stride=128, page_stride=128 * 2 ** 20)
    assert lib.esp_paged_accept(4, ctypes.byref(cache), ctypes.byref(_batch(batch=0)), X, X, X, X, None, 4, X, 7 * X, None) == 0
