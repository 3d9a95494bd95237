"""sr_rope_kv_append where the quantiser's numbers leave the ordinary: clipping ratios far below 1, rows that hold a NaN or an
infinity, or reach one; and tables of angles without a row."""
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


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_rows_that_are_not_finite(gpu, d, bad):
    """A head of a token with such a value stands for NaN as a whole: read back, and in the attention of the query heads that
    read it.  Every other row, head and sequence is what it is without it."""
    rng = np.random.default_rng(d)
    T, KV, H, page = 70, 2, 4, 16
    k, v = inputs(rng, T, KV, d), inputs(rng, T, KV, d)
    q = (1.5 * rng.standard_normal((2, H * d))).astype(np.float16)
    slots = np.arange(T, dtype=np.int64)                     # sequence 0: pages 0 .. 2, 40 tokens; sequence 1: pages 3 and 4
    table, lens = dev(np.array([[0, 1, 2], [3, 4, -1]], np.int32)), dev(np.array([40, 22], np.int32))

    def through(k, v):
        cache = make_cache(5, KV, page, d, True)
        gpu.sr_rope_kv_append(None, dev(k.reshape(T, -1)), dev(v.reshape(T, -1)), None, dev(slots), None, cache)
        gk, gv = gpu.sr_kv_gather(dev(slots), cache)
        o = gpu.sr_attn_decode(dev(q), cache, table, lens)
        torch.cuda.synchronize()
        return (*(rows_of(t, slots, page) for t in cache), *(t.cpu().numpy().reshape(T, KV, d) for t in (gk, gv)), o.cpu().numpy().reshape(2, H, d))

    clean = through(k, v)
    k[5, 0, 3] = bad                                         # read by heads 0 and 1 of sequence 0
    k[60, 1, d - 1] = bad                                    # by heads 2 and 3 of sequence 1
    v[61, 1, 0], v[61, 1, 1] = bad, -bad
    got = through(k, v)
    is_bad = np.zeros((2, T, KV), bool)
    is_bad[0, 5, 0] = is_bad[0, 60, 1] = is_bad[1, 61, 1] = True
    for side in (0, 1):
        rows, params, back = got[side], got[2 + side], got[4 + side]
        assert np.isnan(params[is_bad[side]][:, 0]).all() and np.isfinite(params[is_bad[side]][:, 1]).all() and np.isnan(back[is_bad[side]]).all()
        for a, b in ((rows, clean[side]), (params, clean[2 + side]), (back, clean[4 + side])):
            np.testing.assert_array_equal(a[~is_bad[side]], b[~is_bad[side]])
    o = got[6]
    assert np.isnan(o[0, :2]).all() and np.isnan(o[1, 2:]).all()
    np.testing.assert_array_equal(o[0, 2:], clean[6][0, 2:])
    np.testing.assert_array_equal(o[1, :2], clean[6][1, :2])


@pytest.mark.parametrize("d", [64, 128])
def test_keys_that_the_transform_takes_out_of_range(gpu, d):
    """Finite keys whose transform does not fit fp16."""
    rng = np.random.default_rng(1)
    k, v = inputs(rng, 9, 1, d), inputs(rng, 9, 1, d)
    k[4] = 65504                                             # the first value becomes 65504 sqrt(d), the others 0
    slots = np.arange(9, dtype=np.int64)
    cache = make_cache(1, 1, 16, d, True)
    K_out = torch.zeros((9, d), dtype=torch.float16, device="cuda")
    gpu.sr_rope_kv_append(None, dev(k.reshape(9, -1)), dev(v.reshape(9, -1)), None, dev(slots), None, cache, hadamard=True, K_out=K_out)
    gk, gv = gpu.sr_kv_gather(dev(slots), cache)
    torch.cuda.synchronize()
    with np.errstate(over="ignore"):
        want = ao.rotate_heads_by_position(k, None, None, hadamard=True, dtype=np.float32).astype(np.float16)
    np.testing.assert_array_equal(K_out.cpu().numpy().reshape(9, 1, d), want)
    there = np.arange(9) != 4
    assert np.isinf(want[4, 0, 0]) and np.isfinite(want[there]).all()
    codes, scale, zero = ao.quantise_heads(want[there], 0.95, np.float32)
    np.testing.assert_array_equal(ao.unpack_uint4(rows_of(cache[0], slots, 16))[there], codes)
    np.testing.assert_array_equal(rows_of(cache[2], slots, 16)[there], np.stack([scale, zero], -1))
    assert np.isnan(gk[4].cpu().numpy()).all() and torch.isfinite(gk[there]).all() and torch.isfinite(gv).all()


def test_a_16_bit_cache_takes_rows_as_they_are(gpu):
    rng = np.random.default_rng(2)
    k, v = inputs(rng, 5, 2, 64), inputs(rng, 5, 2, 64)
    k[1, 0, 5], k[2, 1, 0], v[3, 0, 63] = np.nan, np.inf, -np.inf
    slots = np.arange(5, dtype=np.int64)
    cache = make_cache(1, 2, 16, 64, False)
    gpu.sr_rope_kv_append(None, dev(k.reshape(5, -1)), dev(v.reshape(5, -1)), None, dev(slots), None, cache)
    gk, gv = gpu.sr_kv_gather(dev(slots), cache)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(gk.cpu().numpy().reshape(k.shape), k)
    np.testing.assert_array_equal(gv.cpu().numpy().reshape(v.shape), v)


def test_a_table_without_a_row_is_refused(gpu):
    """It has no address, which must not read as "no rotation"."""
    x = torch.ones((3, 64), dtype=torch.float16, device="cuda")
    at = torch.zeros(3, dtype=torch.int32, device="cuda")
    cache = make_cache(1, 1, 16, 64, False)
    with pytest.raises(ValueError):
        gpu.sr_rope_kv_append(x, x, x, at, at.long(), torch.empty((0, 64), device="cuda"), cache)
    torch.cuda.synchronize()
    assert torch.isnan(cache[0]).all()
