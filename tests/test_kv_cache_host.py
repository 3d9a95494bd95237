"""Clipping ratios that the cache's writer refuses, before a device is touched."""
import pytest

import paper_2506_05413_amd as sr
from test_attention_host import A, append, cache


@pytest.mark.parametrize("clip", [2.0 ** -65, 1e-30, 1e-45, -0.5, 1.0000001])
def test_ratios_that_are_refused(clip):
    assert append(clip=clip) == append(clip=clip, T=0) == sr.SR_ERR_ARG
    assert append(cache(type=sr.SR_KV_F16, K_params=None, V_params=None), clip=clip, T=0) == sr.SR_OK       # not looked at


def test_the_smallest_ratio():
    assert append(clip=2.0 ** -64, T=0) == sr.SR_OK and append(clip=2.0 ** -64, slots=A + 0, K=None) == sr.SR_ERR_NULL
