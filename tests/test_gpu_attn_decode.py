"""sr_attn_decode against 64-bit attention over what the cache stands for."""
import numpy as np
import pytest
import torch

from attention_bounds import attention_bound, check_attention
from oracle import attention_oracle as ao
from oracle.smoothrot_oracle import pack_uint4

pytestmark = pytest.mark.gpu


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


class Batch:
    """Sequences in a shuffled paged cache; every slot that no token holds is NaN (codes: anything, parameters NaN)."""

    def __init__(self, lens, KV, d, page, i4, seed=0, spread=1.0, offset=0.0, width=None, spare=2):
        rng = np.random.default_rng(seed)
        self.lens, self.KV, self.d, self.page, self.i4 = list(lens), KV, d, page, i4
        used = [-(-n // page) for n in lens]
        width = width or max(1, max(used))
        pages = sum(used) + spare
        order = rng.permutation(pages)
        self.table = rng.integers(-(1 << 31), 1 << 31, (len(lens), width)).astype(np.int32)     # not looked at behind the length
        cols = d // 2 if i4 else d
        cache = [rng.integers(0, 256, (pages, KV, page, cols)).astype(np.uint8) if i4 else np.full((pages, KV, page, cols), np.nan, np.float16) for _ in range(2)]
        params = [np.full((pages, KV, page, 2), np.nan, np.float32) for _ in range(2)]
        self.k, self.v, self.k_size, self.v_size = [], [], [], []
        at = 0
        for b, n in enumerate(lens):
            mine = order[at:at + used[b]]
            at += used[b]
            self.table[b, :used[b]] = mine
            slots = (mine[:, None] * page + np.arange(page)).reshape(-1)[:n]
            for side, (values, sizes) in enumerate(((self.k, self.k_size), (self.v, self.v_size))):
                x = (spread * (rng.standard_normal((n, KV, d)) + offset)).astype(np.float16)
                if i4:
                    codes, scale, zero = ao.quantise_heads(x, 0.95, np.float32) if n else (np.zeros((0, KV, d), np.uint8), np.zeros((0, KV), np.float32), np.zeros((0, KV), np.float32))
                    cache[side][slots // page, :, slots % page] = pack_uint4(codes)
                    params[side][slots // page, :, slots % page] = np.stack([scale, zero], -1)
                    values.append(ao.values_of(codes, scale, zero))
                    sizes.append((codes + np.abs(zero.astype(np.float64))[..., None]) * scale[..., None].astype(np.float64))
                else:
                    cache[side][slots // page, :, slots % page] = x
                    values.append(x.astype(np.float64))
                    sizes.append(np.abs(x.astype(np.float64)))
        self.cache = (dev(cache[0]), dev(cache[1]), dev(params[0]) if i4 else None, dev(params[1]) if i4 else None)
        self.table_dev, self.lens_dev = dev(self.table), dev(np.array(lens, np.int32))

    def want(self, q, scale, b, h, gone=None):
        """(o, bound) of query rows q [n, d] of sequence b over head h; gone: tokens left out."""
        k, v = self.k[b][:, h], self.v[b][:, h]
        seen = np.ones((len(q), len(k)), bool)
        if gone is not None:
            seen[:, gone] = False
        o, p, s = ao.attend(q, k, v, scale, seen)
        return o, attention_bound(q.astype(np.float64), self.k_size[b][:, h], v, self.v_size[b][:, h], o, p, s, scale)

    def check(self, got, q, scale, what="", gone=None):
        """got, q: [B, H, d]."""
        G = q.shape[1] // self.KV
        worst = 0.0
        for b in range(len(self.lens)):
            for h in range(self.KV):
                rows = slice(h * G, h * G + G)
                o, bound = self.want(q[b, rows], scale, b, h, None if gone is None else gone[b])
                worst = max(worst, check_attention(got[b, rows], o, bound, "%s sequence %d (%d tokens) head %d" % (what, b, self.lens[b], h)))
        return worst


def queries(B, H, d, seed=1, spread=1.5):
    return (spread * np.random.default_rng(seed).standard_normal((B, H, d))).astype(np.float16)


def run(sr, batch, q, scale=None, **more):
    B, H, d = q.shape
    got = sr.sr_attn_decode(dev(q.reshape(B, -1)), batch.cache, batch.table_dev, batch.lens_dev, scale, **more)
    torch.cuda.synchronize()
    return got.cpu().numpy().reshape(B, H, d)


LENS = [0, 1, 15, 16, 17, 31, 32, 33, 127, 128, 129, 300, 511]


@pytest.mark.parametrize("i4", [True, False])
@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("H,KV", [(32, 8), (3, 3), (16, 1), (20, 1), (40, 2), (16, 2), (5, 1), (6, 2)])
def test_lengths_and_heads(gpu, i4, d, H, KV):
    print("case decode", H, KV, d, i4, flush=True)
    batch = Batch(LENS, KV, d, 16, i4, seed=H)
    q = queries(len(LENS), H, d)
    batch.check(run(gpu, batch, q), q, 1 / np.sqrt(d))


@pytest.mark.parametrize("i4", [True, False])
@pytest.mark.parametrize("page,H", [(16, 8), (64, 8), (4096, 8), (16, 2), (64, 14), (32, 24), (16, 34)])
def test_long_sequences_are_split_and_joined(gpu, i4, page, H):
    print("case decode long", page, H, i4, flush=True)
    for lens in ([5001], [3, 4097, 0, 2500]):
        batch = Batch(lens, 2, 128, page, i4, seed=page)
        assert gpu.sr_attn_decode_workspace_bytes(len(lens), H, 2, 128, batch.table.shape[1], page, int(i4)) > 0
        q = queries(len(lens), H, 128)
        batch.check(run(gpu, batch, q), q, 1 / np.sqrt(128))


@pytest.mark.parametrize("i4", [True, False])
@pytest.mark.parametrize("n,longest,shares", [(1, 380, False), (1, 1000, True), (16, 760, False), (16, 3200, True), (7, 300, False), (33, 380, False)])
def test_both_sides_of_the_choice(gpu, i4, n, longest, shares):
    """One workgroup per sequence, and shares of them: few sequences and many."""
    lens = [longest] + [int(x) for x in np.random.default_rng(n).integers(0, longest, n - 1)]
    batch = Batch(lens, 8, 128, 16, i4, seed=n)
    assert (gpu.sr_attn_decode_workspace_bytes(n, 16, 8, 128, batch.table.shape[1], 16, int(i4)) > 0) == shares
    q = queries(n, 16, 128)
    batch.check(run(gpu, batch, q), q, 1 / np.sqrt(128))


@pytest.mark.parametrize("i4", [True, False])
def test_a_table_wider_than_the_lengths(gpu, i4):
    batch = Batch([0, 1, 70, 128], 2, 64, 16, i4, width=700)
    q = queries(4, 4, 64)
    batch.check(run(gpu, batch, q), q, 1 / 8)


def test_lengths_outside_the_table_are_cut(gpu):
    batch = Batch([64, 64, 64], 2, 128, 16, True)
    q = queries(3, 8, 128)
    want = run(gpu, batch, q)
    batch.lens_dev = dev(np.array([64, 1 << 30, -7], np.int32))
    got = run(gpu, batch, q)
    np.testing.assert_array_equal(got[:2], want[:2])
    assert (got[2] == 0).all()


@pytest.mark.parametrize("i4", [True, False])
def test_tokens_of_missing_pages_are_left_out(gpu, i4):
    lens = [100, 48, 700, 33]
    batch = Batch(lens, 2, 128, 16, i4)
    gone = [np.zeros(n, bool) for n in lens]
    for b, page, entry in ((0, 0, -1), (0, 6, 1 << 30), (2, 9, -(1 << 31)), (2, 43, batch.cache[0].shape[0]), (1, 0, -1), (1, 1, -1), (1, 2, -1)):
        batch.table[b, page] = entry
        gone[b][16 * page:16 * page + 16] = True
    batch.table_dev = dev(batch.table)
    q = queries(4, 8, 128)
    got = run(gpu, batch, q)
    batch.check(got, q, 1 / np.sqrt(128), gone=gone)
    assert (got[1] == 0).all()


@pytest.mark.parametrize("i4", [True, False])
@pytest.mark.parametrize("spread,offset", [(1e-3, 0.0), (2e3, 0.0), (1.0, 30.0), (0.02, 400.0)])
def test_small_large_and_shifted_values(gpu, i4, spread, offset):
    """Values far from 1, and rows far from zero beside their range."""
    batch = Batch([200, 37], 2, 128, 32, i4, spread=spread, offset=offset)
    q = queries(2, 8, 128, spread=1.5 / (spread * (1 + offset)))
    batch.check(run(gpu, batch, q), q, 1 / np.sqrt(128), "spread %g offset %g" % (spread, offset))


@pytest.mark.parametrize("i4", [True, False])
@pytest.mark.parametrize("d", [128, 64])
def test_scores_beyond_the_steps_of_fp32(gpu, i4, d):
    """Scores up to 2^39, whose neighbouring fp32 numbers are 2^16 apart, every two of them further than that: all weight is on
    the largest.  Off by the weight's and the output's rounding (2^-11 each) and those of the fp32 sums (2^-20 of their terms)."""
    rng = np.random.default_rng(d)
    lens = [300, 1, 1500]
    batch = Batch(lens, 2, d, 16, i4, seed=d, spread=0.01)
    q = np.full((3, 4, d), 30000, np.float16)
    K, V, Kp, Vp = (None if t is None else t.cpu() for t in batch.cache)
    best = np.zeros((3, 2), int)
    for b, n in enumerate(lens):
        for h in range(2):
            size = rng.permutation(np.arange(500, 500 + n)).astype(np.float32)
            best[b, h] = size.argmax()
            for t in range(n):
                page, at = batch.table[b, t // 16], t % 16
                if i4:
                    K[page, h, at], Kp[page, h, at] = 0x11, torch.tensor([float(size[t]), 0.0])
                else:
                    K[page, h, at] = float(size[t])
    batch.cache = tuple(None if t is None else t.cuda() for t in (K, V, Kp, Vp))
    got = run(gpu, batch, q, 64.0).astype(np.float64)
    for b in range(3):
        for head in range(4):
            v, size = batch.v[b][best[b, head // 2], head // 2], batch.v_size[b][best[b, head // 2], head // 2]
            assert (np.abs(got[b, head] - v) <= 2.0 ** -10 * np.abs(v) + 2.0 ** -20 * size + 2.0 ** -25).all(), (b, head)


@pytest.mark.parametrize("i4", [True, False])
@pytest.mark.parametrize("scale", [1e-4, 0.5, 3.0])
def test_scales_from_flat_to_one_token(gpu, i4, scale):
    batch = Batch([300, 16], 1, 64, 16, i4)
    q = queries(2, 4, 64)
    batch.check(run(gpu, batch, q, scale), q, np.float32(scale).astype(np.float64))


def test_steps_that_differ_by_far_between_tokens(gpu):
    """4-bit values whose steps span the range of fp16 inside one sequence."""
    batch = Batch([256], 1, 128, 16, True)
    K, V, Kp, Vp = batch.cache
    rng = np.random.default_rng(3)
    factor = 2.0 ** rng.integers(-20, 10, 256)
    slots = (batch.table[0, :, None] * 16 + np.arange(16)).reshape(-1)
    p = Vp.cpu().numpy()
    p[slots // 16, 0, slots % 16, 0] *= factor.astype(np.float32)
    batch.cache = (K, V, Kp, dev(p))
    batch.v[0], batch.v_size[0] = batch.v[0] * factor[:, None, None], batch.v_size[0] * factor[:, None, None]
    q = queries(1, 4, 128)
    batch.check(run(gpu, batch, q), q, 1 / np.sqrt(128))


def test_strided_rows_and_untouched_memory(gpu):
    batch = Batch([77, 500], 2, 128, 16, True)
    q = queries(2, 6, 128)
    wide = torch.full((2, 6 * 128 + 40), float("nan"), dtype=torch.float16, device="cuda")
    wide[:, 16:16 + 768] = dev(q.reshape(2, -1))
    out = torch.full((2, 6 * 128 + 24), 7.0, dtype=torch.float16, device="cuda")
    table = torch.full((2, batch.table.shape[1] + 5), -1, dtype=torch.int32, device="cuda")
    table[:, :batch.table.shape[1]] = batch.table_dev
    need = gpu.sr_attn_decode_workspace_bytes(2, 6, 2, 128, batch.table.shape[1], 16)
    work = torch.full((need + 512,), 0xFF, dtype=torch.uint8, device="cuda")
    got = gpu.sr_attn_decode(wide[:, 16:16 + 768], batch.cache, table[:, :batch.table.shape[1]], batch.lens_dev, O=out[:, 8:8 + 768], workspace=work[:need])
    torch.cuda.synchronize()
    batch.check(got.cpu().numpy().reshape(2, 6, 128), q, 1 / np.sqrt(128))
    assert (out[:, :8] == 7).all() and (out[:, 776:] == 7).all() and (work[need:] == 0xFF).all()
    again = run(gpu, batch, q)
    np.testing.assert_array_equal(got.cpu().numpy().reshape(2, 6, 128), again)


def test_pages_beyond_32_bit_offsets(gpu):
    """The same sequence in the first and in the last pages of a cache of 5 GB a side."""
    KV, d, page = 8, 128, 256
    pages = (5 << 30) // (KV * page * d * 2)
    batch = Batch([600], KV, d, page, False)
    K = torch.empty((pages, KV, page, d), dtype=torch.float16, device="cuda")
    V = torch.empty_like(K)
    far = np.array([pages - 1, pages // 2 + 1, pages - 7])
    for i, p in enumerate(far):
        K[p], V[p] = batch.cache[0][batch.table[0, i]], batch.cache[1][batch.table[0, i]]
    q = queries(1, 16, d)
    near = run(gpu, batch, q)
    batch.cache, batch.table_dev = (K, V, None, None), dev(far[None].astype(np.int32))
    np.testing.assert_array_equal(run(gpu, batch, q), near)
    batch.check(near, q, 1 / np.sqrt(d))


def test_more_sequences_than_workgroups_at_once(gpu):
    rng = np.random.default_rng(8)
    lens = [int(n) for n in rng.integers(0, 90, 400)]
    batch = Batch(lens, 4, 64, 32, True)
    q = queries(400, 8, 64)
    batch.check(run(gpu, batch, q), q, 1 / 8)
