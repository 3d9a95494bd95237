"""sr_attn_prefill against 64-bit attention."""
import numpy as np
import pytest
import torch

from attention_bounds import attention_bound, check_attention
from oracle import attention_oracle as ao

pytestmark = pytest.mark.gpu


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def ends(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)


def make(nq, nk, H, KV, d, seed=0, spread=1.5):
    rng = np.random.default_rng(seed)
    q = (spread * rng.standard_normal((sum(nq), H, d))).astype(np.float16)
    k, v = (rng.standard_normal((sum(nk), KV, d)).astype(np.float16) for _ in range(2))
    return q, k, v


def check(got, q, k, v, nq, nk, causal, scale, what=""):
    """got [T, H, d] against every sequence and head."""
    H, KV, d = q.shape[1], k.shape[1], q.shape[2]
    i = j = 0
    worst = 0.0
    for s, (n, m) in enumerate(zip(nq, nk)):
        seen = ao.causal(n, m) if causal else np.ones((n, m), bool)
        for h in range(H if n else 0):
            qq, kk, vv = q[i:i + n, h].astype(np.float64), k[j:j + m, h * KV // H].astype(np.float64), v[j:j + m, h * KV // H].astype(np.float64)
            o, p, sc = ao.attend(qq, kk, vv, scale, seen)
            bound = attention_bound(qq, np.abs(kk), vv, np.abs(vv), o, p, sc, scale, rounded_total=True)
            worst = max(worst, check_attention(got[i:i + n, h], o, bound, "%s sequence %d (%d queries, %d keys) head %d" % (what, s, n, m, h)))
        i, j = i + n, j + m
    return worst


def run(sr, q, k, v, nq, nk, causal=True, scale=None, **more):
    T, H, d = q.shape
    got = sr.sr_attn_prefill(dev(q.reshape(T, -1)), dev(k.reshape(len(k), k.shape[1] * d)), dev(v.reshape(len(v), v.shape[1] * d)), dev(ends(nq)), dev(ends(nk)), d, causal, scale, **more)
    torch.cuda.synchronize()
    return got.cpu().numpy().reshape(T, H, d)


LENS = [1, 2, 31, 32, 33, 63, 64, 65, 0, 127, 128, 129, 200, 300]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H,KV", [(8, 2), (3, 3), (5, 1)])
@pytest.mark.parametrize("causal", [True, False])
def test_packed_lengths(gpu, d, H, KV, causal):
    print("case prefill", d, H, KV, causal, flush=True)
    q, k, v = make(LENS, LENS, H, KV, d, seed=d + H)
    check(run(gpu, q, k, v, LENS, LENS, causal), q, k, v, LENS, LENS, causal, 1 / np.sqrt(d))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
def test_other_numbers_of_keys(gpu, d, causal):
    """Chunks behind a cached prefix, more queries than keys (rows that see nothing), no keys, no queries."""
    nq = [1, 1, 40, 130, 7, 150, 33, 0, 64, 5]
    nk = [1, 500, 40, 700, 0, 20, 97, 50, 63, 129]
    q, k, v = make(nq, nk, 4, 2, d, seed=d)
    got = run(gpu, q, k, v, nq, nk, causal)
    check(got, q, k, v, nq, nk, causal, 1 / np.sqrt(d))
    at = np.cumsum([0] + nq)
    assert (got[at[4]:at[5]] == 0).all()
    if causal:
        assert (got[at[5]:at[5] + 130] == 0).all()


def test_no_keys_at_all_and_output_over_the_queries(gpu):
    q, k, v = make([5, 40], [5, 40], 4, 2, 128)
    assert (run(gpu, q, k[:0], v[:0], [5, 40], [0, 0]) == 0).all() and (run(gpu, q, k[:0], v[:0], [5, 40], [0, 0], False) == 0).all()
    Q, cu = dev(q.reshape(45, -1)), dev(ends([5, 40]))
    want = run(gpu, q, k, v, [5, 40], [5, 40])
    assert gpu.sr_attn_prefill(Q, dev(k.reshape(45, -1)), dev(v.reshape(45, -1)), cu, cu, 128, O=Q).data_ptr() == Q.data_ptr()
    torch.cuda.synchronize()
    np.testing.assert_array_equal(Q.cpu().numpy().reshape(45, 4, 128), want)


@pytest.mark.parametrize("T,H,KV,d", [(1, 32, 8, 128), (1000, 4, 1, 128), (777, 2, 2, 64)])
def test_one_prompt(gpu, T, H, KV, d):
    q, k, v = make([T], [T], H, KV, d, seed=T)
    check(run(gpu, q, k, v, [T], [T]), q, k, v, [T], [T], True, 1 / np.sqrt(d))


@pytest.mark.parametrize("nq,nk,H,KV,d", [([300], [300], 12, 3, 128), ([700, 650, 900, 80], [700, 1400, 900, 33], 24, 6, 128), ([2500], [2500], 56, 1, 128),
                                          ([1100, 1500], [1100, 1700], 60, 2, 128), ([700, 10, 650], [800, 10, 650], 40, 4, 64), ([140] * 70, [150] * 70, 8, 8, 128),
                                          ([1400], [1400], 18, 2, 128), ([5, 64, 1, 130, 0], [2050, 3000, 2200, 2500, 2300], 6, 2, 128), ([200, 77], [1200, 1111], 4, 2, 64),
                                          ([10, 40, 3], [0, 6200, 5], 5, 5, 128), ([33, 300], [20, 2100], 3, 1, 64),
                                          ([2200], [2200], 60, 4, 128), ([2200, 2300], [2200, 2300], 30, 5, 128), ([40] * 9, [45] * 9, 32, 8, 128),
                                          ([300, 20, 150], [300, 20, 150], 24, 2, 64), ([7] * 100, [9] * 100, 16, 4, 64)])
@pytest.mark.parametrize("causal", [True, False])
def test_every_shape_of_workgroup(gpu, nq, nk, H, KV, d, causal):
    """Few rows (two or four sets of waves over the keys), more of them (128 rows a workgroup, with and without all of them at once, and
    more sequences than a wave looks at), and long sequences (256)."""
    print("case prefill", len(nq), sum(nq), H, KV, d, causal, flush=True)
    q, k, v = make(nq, nk, H, KV, d, seed=sum(nq))
    got = run(gpu, q, k, v, nq, nk, causal)
    few = [0, H // 2, H - 1]                             # of the heads
    at = [h * KV // H for h in few]
    check(got[:, few], q[:, few], k[:, at], v[:, at], nq, nk, causal, 1 / np.sqrt(d))


@pytest.mark.parametrize("scale", [1e-4, 0.7, 4.0])
def test_scales_from_flat_to_one_token(gpu, scale):
    q, k, v = make([150, 90], [150, 90], 2, 1, 128)
    check(run(gpu, q, k, v, [150, 90], [150, 90], scale=scale), q, k, v, [150, 90], [150, 90], True, float(np.float32(scale)))


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("H,T", [(2, 300), (2, 1500), (26, 2048), (48, 1024)])
def test_scores_beyond_the_steps_of_fp32(gpu, d, H, T):
    """Scores up to 2^39, whose neighbouring fp32 numbers are 2^16 apart, every two of them further than that: all weight is on
    the largest so far, a power of two that comes out again."""
    q, k, v = make([T], [T], H, 1, d, seed=T)
    size = np.random.default_rng(d).permutation(np.arange(T) % 1500 + 500 + np.arange(T) // 1500 * 0.5).astype(np.float16)
    size = np.unique(size)                               # (fp16 holds the halves up to 1023.5)
    T = len(size)
    q, v = q[:T], v[:T]
    np.random.default_rng(d).shuffle(size)
    q[:], k = 30000, np.broadcast_to(size[:, None, None], (T, 1, d)).copy()
    best = np.array([size[:i + 1].argmax() for i in range(T)])
    got = run(gpu, q, k, v, [T], [T], True, 64.0)
    for h in range(H):
        np.testing.assert_array_equal(got[:, h], v[best, 0])


def test_scores_that_grow_and_fall_along_the_keys(gpu):
    """The running maximum is replaced at every tile, and never."""
    T, d = 400, 128
    q, k, v = make([T], [T], 2, 2, d)
    for sign in (1, -1):
        kk = k.copy()
        q[:, :, 0], kk[:, :, 0] = 8, (sign * np.linspace(-30, 30, T)[:, None]).astype(np.float16)
        check(run(gpu, q, kk, v, [T], [T], False), q, kk, v, [T], [T], False, 1 / np.sqrt(d))


def test_rows_of_no_sequence_and_other_columns_stay(gpu):
    d, H, KV = 64, 3, 1
    nq, nk = [50, 20], [50, 20]
    q, k, v = make(nq, nk, H, KV, d)
    pad = 13
    fused = torch.full((70 + pad, (H + 2 * KV) * d + 16), float("nan"), dtype=torch.float16, device="cuda")
    fused[:70, :H * d], fused[:70, H * d:H * d + d], fused[:70, H * d + d:H * d + 2 * d] = dev(q.reshape(70, -1)), dev(k.reshape(70, -1)), dev(v.reshape(70, -1))
    out = torch.full((70 + pad, H * d + 16), 7.0, dtype=torch.float16, device="cuda")
    gpu.sr_attn_prefill(fused[:, :H * d], fused[:, H * d:H * d + d], fused[:, H * d + d:H * d + 2 * d], dev(ends(nq)), dev(ends(nk)), d, O=out[:, 8:8 + H * d])
    torch.cuda.synchronize()
    check(out[:70, 8:8 + H * d].cpu().numpy().reshape(70, H, d), q, k, v, nq, nk, True, 1 / 8)
    assert (out[70:] == 7).all() and (out[:, :8] == 7).all() and (out[:, 8 + H * d:] == 7).all()


def test_neighbours_do_not_leak(gpu):
    """A sequence of NaN and infinities between two others."""
    nq = [70, 33, 90]
    q, k, v = make(nq, nq, 2, 1, 128)
    bad = slice(70, 103)
    k[bad], v[bad], q[bad] = np.nan, np.inf, np.nan
    got = run(gpu, q, k, v, nq, nq)
    for part, n in ((slice(0, 70), 70), (slice(103, 193), 90)):
        check(got[part], q[part], k[part], v[part], [n], [n], True, 1 / np.sqrt(128))


def test_ends_that_do_not_fit_are_cut(gpu):
    q, k, v = make([100], [100], 2, 1, 64)
    want = run(gpu, q, k, v, [60, 40], [60, 40])
    Q, K, V = dev(q.reshape(100, -1)), dev(k.reshape(100, -1)), dev(v.reshape(100, -1))
    cu = dev(np.array([0, 60, 1000], np.int32))
    got = gpu.sr_attn_prefill(Q, K, V, cu, cu, 64)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(got.cpu().numpy().reshape(want.shape), want)
    # descending and negative ends: no rows
    out = torch.full((100, 128), 7.0, dtype=torch.float16, device="cuda")
    cu = dev(np.array([-5, -2, -9], np.int32))
    gpu.sr_attn_prefill(Q, K, V, cu, cu, 64, O=out)
    torch.cuda.synchronize()
    assert (out == 7).all()


def test_more_sequences_than_lanes(gpu):
    rng = np.random.default_rng(6)
    lens = [int(n) for n in rng.integers(0, 12, 300)]
    lens[170] = 200
    q, k, v = make(lens, lens, 2, 2, 64)
    check(run(gpu, q, k, v, lens, lens), q, k, v, lens, lens, True, 1 / 8)
