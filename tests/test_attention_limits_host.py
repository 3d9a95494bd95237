"""Limits of the attention calls that hold before a device is touched."""
import pytest

import paper_2506_05413_amd as sr
from test_attention_host import prefill


@pytest.mark.parametrize("tokens,status", [((1 << 31) - 1, sr.SR_ERR_SHAPE), ((1 << 31) - (1 << 10) + 1, sr.SR_ERR_SHAPE), ((1 << 31) - (1 << 10), sr.SR_ERR_NULL)])
def test_tokens_whose_last_tile_ends_beyond_32_bits(tokens, status):
    """(The last one goes on to the check of its pointers.)"""
    assert prefill(Tk=tokens, K=None) == prefill(Tq=tokens, H=2, Q=None) == status


@pytest.mark.parametrize("page", [24, 48, 100, 8, 0, -16, 1 << 21])
def test_no_workspace_for_pages_that_are_refused(page):
    assert sr.sr_attn_decode_workspace_bytes(1, 32, 8, 128, 512, 32) > 0
    assert sr.sr_attn_decode_workspace_bytes(1, 32, 8, 128, 512, page) == 0
