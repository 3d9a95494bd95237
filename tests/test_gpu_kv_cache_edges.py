"""sr_rope_kv_append where the quantiser's numbers leave the ordinary: clipping ratios far below 1."""
import numpy as np
import pytest
import torch

from oracle import attention_oracle as ao
from test_gpu_kv_cache import dev, inputs, make_cache, rows_of

pytestmark = pytest.mark.gpu


def edge_rows(d):
    """Rows around zero, rows whose every value is far from it beside their range, rows of the smallest numbers."""
    rng = np.random.default_rng(d)
    v = np.zeros((12, 1, d), np.float16)
    v[:4] = rng.standard_normal((4, 1, d))
    v[4] = np.linspace(1000, 1001, d)
    v[5] = -np.linspace(1000, 1001, d)
    v[6, 0, ::2], v[6, 0, 1::2] = 65504, 65472               # one step apart at the end of fp16's range
    v[7] = -v[6]
    v[8] = rng.uniform(-65504, 65504, d)
    v[9] = 3.25
    v[10] = 6e-8
    v[10, 0, 3] = -6e-8
    v[11, 0, 7] = 65504
    return v


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("clip", [0.3, 0.01, 1e-3, 1e-6, 1e-12, 2.0 ** -64])
def test_small_clips(gpu, d, clip):
    """A small ratio makes a small step: quotients go up to 2^15 / clip, and all but the smallest values take code 0 or 15."""
    v = edge_rows(d)
    clip = float(np.float32(clip))
    slots = np.arange(len(v), dtype=np.int64)
    cache = make_cache(1, 1, 16, d, True)
    V = dev(v.reshape(len(v), -1))
    gpu.sr_rope_kv_append(None, V, V, None, dev(slots), None, cache, clip=clip)
    torch.cuda.synchronize()
    codes, scale, zero = ao.quantise_heads(v, clip, np.float32)
    for side in (0, 1):
        np.testing.assert_array_equal(ao.unpack_uint4(rows_of(cache[side], slots, 16)), codes)
        np.testing.assert_array_equal(rows_of(cache[2 + side], slots, 16), np.stack([scale, zero], -1))
