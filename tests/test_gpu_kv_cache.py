"""sr_rope_kv_append and sr_kv_gather against the oracle.  The numbers that go into the cache are promised bit for bit (the
formula in fp32, every operation rounded); the formula in fp32 is held to the one in 64 bits on the CPU
(test_attention_host.py)."""
import numpy as np
import pytest
import torch

from oracle import attention_oracle as ao

pytestmark = pytest.mark.gpu


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def make_cache(pages, kv, page, d, i4, seed=0):
    """A cache full of bytes that no call may touch unasked: NaN, or odd codes and NaN parameters."""
    if i4:
        K = torch.full((pages, kv, page, d // 2), 0xA5, dtype=torch.uint8, device="cuda")
        P = torch.full((pages, kv, page, 2), float("nan"), device="cuda")
        return K, K.clone(), P, P.clone()
    K = torch.full((pages, kv, page, d), float("nan"), dtype=torch.float16, device="cuda")
    return K, K.clone(), None, None


def rows_of(t, slots, page):
    """[T, kv, ..] of the cache tensor's slots."""
    a = t.cpu().numpy()
    return a[slots // page, :, slots % page]


def inputs(rng, T, heads, d, offset=0.0):
    return (rng.standard_normal((T, heads, d)) + offset * rng.standard_normal((heads, d))).astype(np.float16)


def check_append(sr, T, H, KV, d, page, i4, pairs, hadamard, clip=0.95, with_table=True, seed=0, with_k_out=True):
    rng = np.random.default_rng(seed + T)
    print("case append", T, H, KV, d, page, i4, pairs, hadamard, flush=True)
    q, k, v = inputs(rng, T, H, d), inputs(rng, T, KV, d, 2.0), inputs(rng, T, KV, d, 0.3)
    # columns of one fused projection, with a gap behind them
    fused = torch.full((T, (H + 2 * KV) * d + 24), float("nan"), dtype=torch.float16, device="cuda")
    for a, at in ((q, 0), (k, H * d), (v, (H + KV) * d)):
        fused[:, at:at + a.shape[1] * d] = dev(a.reshape(T, -1))
    Q, K, V = fused[:, :H * d], fused[:, H * d:(H + KV) * d], fused[:, (H + KV) * d:(H + 2 * KV) * d]
    table = ao.angles(300, d) if with_table else None
    positions = rng.integers(-3, 305, T).astype(np.int32)           # some outside the table
    pages = -(-T // page) + 2
    slots = rng.permutation(pages * page)[:T].astype(np.int64)
    gone = rng.random(T) < 0.2
    gone[0] = T > 4 and gone[0]
    asked = np.where(gone, rng.choice([-1, -5, pages * page, 1 << 40], T), slots)
    cache = make_cache(pages, KV, page, d, i4)
    before = [None if t is None else t.clone() for t in cache]
    K_out = torch.full((T, KV * d + 8), float("nan"), dtype=torch.float16, device="cuda")[:, :KV * d] if with_k_out else None
    got = sr.sr_rope_kv_append(Q, K, V, dev(positions) if with_table else None, dev(asked), None if table is None else dev(table), cache,
                               hadamard=hadamard, pairs=pairs, clip=clip, K_out=K_out)
    torch.cuda.synchronize()

    want_q = ao.rotate_heads_by_position(q, positions, table, pairs, hadamard, np.float32).astype(np.float16)
    want_k = ao.rotate_heads_by_position(k, positions, table, pairs, hadamard, np.float32).astype(np.float16)
    np.testing.assert_array_equal(got.cpu().numpy().reshape(T, H, d), want_q)
    if with_k_out:
        np.testing.assert_array_equal(K_out.cpu().numpy().reshape(T, KV, d), want_k)
    there = slots[~gone]
    for side, rows in ((0, want_k), (1, v)):
        rows = rows[~gone]
        if i4:
            codes, scale, zero = ao.quantise_heads(rows, clip, np.float32)
            np.testing.assert_array_equal(ao.unpack_uint4(rows_of(cache[side], there, page)), codes)
            np.testing.assert_array_equal(rows_of(cache[2 + side], there, page), np.stack([scale, zero], -1))
        else:
            np.testing.assert_array_equal(rows_of(cache[side], there, page), rows)
    # every other slot is as it was
    for t, b in zip(cache, before):
        if t is not None:
            t, b = (x.view(torch.uint8) if x.dtype == torch.uint8 else x.view(torch.int16 if x.dtype == torch.float16 else torch.int32) for x in (t, b))
            mask = torch.ones(pages * page, dtype=torch.bool)
            mask[torch.from_numpy(there)] = False
            mask = mask.view(pages, 1, page, 1).cuda()
            assert torch.equal(torch.where(mask, t, 0), torch.where(mask, b, 0))
    # and back
    gk, gv = sr.sr_kv_gather(dev(asked), cache)
    torch.cuda.synchronize()
    for rows, g in ((want_k, gk), (v, gv)):
        want = rows.astype(np.float32)
        if i4:
            codes, scale, zero = ao.quantise_heads(rows, clip, np.float32)
            want = (codes.astype(np.float32) - zero[..., None]) * scale[..., None]
        want[gone] = 0
        np.testing.assert_array_equal(g.cpu().numpy().reshape(T, KV, d), want.astype(np.float16))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("i4", [False, True])
@pytest.mark.parametrize("pairs,hadamard", [(False, False), (True, False), (False, True), (True, True)])
def test_append_and_gather(gpu, d, i4, pairs, hadamard):
    check_append(gpu, 37, 6, 2, d, 16, i4, pairs, hadamard)


@pytest.mark.parametrize("T,H,KV,d,page,i4", [(1, 32, 8, 128, 16, True), (1, 1, 1, 64, 16, False), (2, 5, 5, 128, 1024, True),
                                             (5, 3, 1, 64, 32, True), (700, 20, 4, 128, 64, True), (513, 7, 7, 64, 128, False)])
def test_append_shapes(gpu, T, H, KV, d, page, i4):
    check_append(gpu, T, H, KV, d, page, i4, False, T % 2 == 0, clip=1.0 if T == 5 else 0.95, seed=9)


@pytest.mark.parametrize("T,H,KV,d,i4,pairs,hadamard", [(5501, 40, 4, 128, True, False, False), (6001, 36, 4, 64, False, False, False), (5801, 31, 7, 64, True, True, False),
                                                        (5601, 41, 3, 128, False, True, False), (5503, 40, 4, 128, True, False, True)])
def test_append_of_many_rows(gpu, T, H, KV, d, i4, pairs, hadamard):
    """From 262144 rows on they are dealt out in the order of the tokens, unless the transform is asked for."""
    check_append(gpu, T, H, KV, d, 64, i4, pairs, hadamard, seed=3)


def test_append_without_rotation(gpu):
    check_append(gpu, 19, 4, 2, 128, 16, True, False, False, with_table=False, with_k_out=False)
    check_append(gpu, 19, 4, 2, 64, 16, False, False, True, with_table=False)


def test_append_in_place_and_without_queries(gpu):
    rng = np.random.default_rng(1)
    T, H, KV, d = 33, 4, 2, 128
    q, k, v = inputs(rng, T, H, d), inputs(rng, T, KV, d), inputs(rng, T, KV, d)
    table, positions, slots = ao.angles(64, d), np.arange(T, dtype=np.int32), np.arange(T, dtype=np.int64)
    Q, K, V = (dev(a.reshape(T, -1)) for a in (q, k, v))
    cache = make_cache(3, KV, 16, d, True)
    got = gpu.sr_rope_kv_append(Q, K, V, dev(positions), dev(slots), dev(table), cache, Q_out=Q, K_out=K)
    assert got is Q or got.data_ptr() == Q.data_ptr()
    other = make_cache(3, KV, 16, d, True)
    assert gpu.sr_rope_kv_append(None, dev(k.reshape(T, -1)), V, dev(positions), dev(slots), dev(table), other) is None
    torch.cuda.synchronize()
    np.testing.assert_array_equal(Q.cpu().numpy().reshape(T, H, d), ao.rotate_heads_by_position(q, positions, table, dtype=np.float32).astype(np.float16))
    np.testing.assert_array_equal(K.cpu().numpy().reshape(T, KV, d), ao.rotate_heads_by_position(k, positions, table, dtype=np.float32).astype(np.float16))
    for a, b in zip(cache, other):
        x, y = a.cpu().numpy()[:2], b.cpu().numpy()[:2]
        np.testing.assert_array_equal(x, y)


def test_quantiser_edges(gpu):
    """Constant rows, rows that do not straddle zero (zeros far outside 0..15), the largest numbers, a tie at the middle."""
    d, KV = 128, 1
    v = np.zeros((8, KV, d), np.float16)
    v[1] = 3.25
    v[2] = -7.0
    v[3] = np.linspace(1000, 1001, d)
    v[4] = np.linspace(-65504, 65504, d)
    v[5] = np.linspace(-1, 1, d)                          # symmetric: lo / step = -7.5 but for the clip's rounding
    v[6] = 6e-8
    v[6, 0, 3] = -6e-8
    v[7, 0, 100] = 65504
    slots = np.arange(8, dtype=np.int64)
    for clip in (0.95, 1.0):
        cache = make_cache(1, KV, 16, d, True)
        V = dev(v.reshape(8, -1))
        gpu.sr_rope_kv_append(None, V, V, None, dev(slots), None, cache, clip=clip)
        torch.cuda.synchronize()
        codes, scale, zero = ao.quantise_heads(v, clip, np.float32)
        for side in (0, 1):
            np.testing.assert_array_equal(ao.unpack_uint4(rows_of(cache[side], slots, 16)), codes)
            np.testing.assert_array_equal(rows_of(cache[2 + side], slots, 16), np.stack([scale, zero], -1))


def test_agrees_with_the_group_quantiser(gpu):
    """The cache's codes are those of sr_kv_quant_asym with one group per head, but for rounding boundaries."""
    rng = np.random.default_rng(4)
    T, KV, d = 256, 8, 128
    v = dev(inputs(rng, T, KV, d, 0.5).reshape(T, -1))
    cache = make_cache(T // 64, KV, 64, d, True)
    gpu.sr_rope_kv_append(None, v, v, None, dev(np.arange(T, dtype=np.int64)), None, cache)
    Q, scale, zero = gpu.sr_kv_quant_asym(v, d, 0.95)
    torch.cuda.synchronize()
    a = cache[1].permute(0, 2, 1, 3).reshape(T, -1).cpu().numpy()
    p = cache[3].permute(0, 2, 1, 3).reshape(T, KV, 2).cpu().numpy()
    np.testing.assert_allclose(p[..., 0], scale.cpu().numpy(), rtol=1e-6)
    # Both steps are within 5e-7 of the quotient (three roundings, and a reciprocal's unit in the last place), so both quotients
    # v / step and lo / step, at most 16 in size here, are within 8e-6 of the true ones: codes differ only where a quotient lies
    # that near to a boundary, and only in rows whose lo / step does do all codes.  (A row whose largest value is the negative
    # of its smallest has lo / step = -7.5: fp16 rows do that now and then.)
    x = v.cpu().numpy().reshape(T, KV, d)
    _, step, _ = ao.quantise_heads(x, 0.95)
    near = lambda t: np.abs(t - np.floor(t) - 0.5) < 1e-5
    row_tie = near(float(np.float32(0.95)) * x.astype(np.float64).min(-1) / step)
    code_tie = near(x / step[..., None])
    differ = (ao.unpack_uint4(a) != ao.unpack_uint4(Q.cpu().numpy())).reshape(T, KV, d)
    assert not (differ & ~code_tie & ~row_tie[..., None]).any()
    assert not ((p[..., 1] != zero.cpu().numpy()) & ~row_tie).any()
    assert row_tie.mean() < 0.02 and code_tie.mean() < 0.001


def test_far_slots_and_repeats_in_gather(gpu):
    """A cache whose rows lie more than 2^31 bytes apart; the same slot asked for several times."""
    KV, d, page = 8, 128, 1024
    pages = (5 << 30) // (KV * page * d * 2)
    K = torch.empty((pages, KV, page, d), dtype=torch.float16, device="cuda")
    V = torch.empty_like(K)
    cache = (K, V, None, None)
    rng = np.random.default_rng(2)
    slots = np.array([0, pages * page - 1, pages * page // 2 + 17, 5], np.int64)
    k, v = inputs(rng, 4, KV, d), inputs(rng, 4, KV, d)
    gpu.sr_rope_kv_append(None, dev(k.reshape(4, -1)), dev(v.reshape(4, -1)), None, dev(slots), None, cache)
    ask = np.array([1, 1, 3, 0, 2, 1], np.int64)
    gk, gv = gpu.sr_kv_gather(dev(slots[ask]), cache)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(gk.cpu().numpy().reshape(6, KV, d), k[ask])
    np.testing.assert_array_equal(gv.cpu().numpy().reshape(6, KV, d), v[ask])
    np.testing.assert_array_equal(K[-1, :, -1].cpu().numpy(), k[1])


def test_nothing_to_do(gpu):
    cache = make_cache(1, 2, 16, 64, True)
    e = torch.empty((0, 128), dtype=torch.float16, device="cuda")
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    assert gpu.sr_rope_kv_append(e, e, e, None, none, None, cache).shape == (0, 128)
    k, v = gpu.sr_kv_gather(none, cache)
    assert k.shape == v.shape == (0, 128)
