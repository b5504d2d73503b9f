"""Scales of the scores that would not be finite in base 2."""
import pytest

from test_kv4 import _attn, _cache, lib  # noqa: F401


@pytest.mark.parametrize("scale", [2.4e38, 2.9e38, 3.3e38, float("inf")])
def test_attention_refuses_scales_past_fp32_in_base_2(lib, scale):  # noqa: F811
    """scale * log2(e) enters the kernels: an infinite one makes NaN of scores of zero."""
    assert lib.buddy_kv4_attention(_cache(), _attn(scale=scale), None, None) == 1


@pytest.mark.parametrize("n_tok", [2 ** 31 - 1, 2 ** 31 - 256, 2 ** 31 - 512])
def test_attention_refuses_rows_next_to_2_to_the_31(lib, n_tok):  # noqa: F811
    """Rows are counted in 32 bits in tiles of up to 256: the last tile's end has to fit as well."""
    from paper_2606_09514_gb300 import binding as B
    bad = _attn(n_tok=n_tok, max_new=n_tok, n_q_heads=1, row_start=4096)
    assert lib.buddy_kv4_attention(_cache(n_kv_heads=1), bad, None, None) == B.BUDDY_ERR_RANGE
