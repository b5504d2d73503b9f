"""Scales of the scores that would not be finite in base 2."""
import pytest

from test_kv4 import _attn, _cache, lib  # noqa: F401


@pytest.mark.parametrize("scale", [2.4e38, 2.9e38, 3.3e38, float("inf")])
def test_attention_refuses_scales_past_fp32_in_base_2(lib, scale):  # noqa: F811
    """scale * log2(e) enters the kernels: an infinite one makes NaN of scores of zero."""
    assert lib.buddy_kv4_attention(_cache(), _attn(scale=scale), None, None) == 1
