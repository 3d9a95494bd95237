"""The cache and attention kernels that only larger batches, or other combinations of types and heads, reach."""
import numpy as np
import pytest
import torch

import test_gpu_attn_decode as decode
import test_gpu_attn_prefill as prefill
from test_gpu_kv_cache import check_append

pytestmark = pytest.mark.gpu


def lengths(n, longest, some, seed):
    """n lengths: the longest, a few of `some` and more, the others short, one of them none."""
    rng = np.random.default_rng(seed)
    lens = [longest] + [int(x) for x in rng.integers(some, longest, 3)] + [int(x) for x in rng.integers(0, 40, n - 5)] + [0]
    return [lens[i] for i in rng.permutation(n)]


def check_decode(sr, lens, H, KV, d, i4, shares, page=16):
    print("case decode", len(lens), max(lens), H, KV, d, i4, shares, flush=True)
    batch = decode.Batch(lens, KV, d, page, i4, seed=H + d)
    assert (sr.sr_attn_decode_workspace_bytes(len(lens), H, KV, d, batch.table.shape[1], page, int(i4)) > 0) == shares
    q = decode.queries(len(lens), H, d)
    batch.check(decode.run(sr, batch, q), q, 1 / np.sqrt(d))


# Heads of a key/value head: up to 4, 8, 16 and more (the copies in the matrix columns, 4 bits)
GROUPS = [3, 8, 12, 20]


@pytest.mark.parametrize("i4", [True, False])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("group", GROUPS)
def test_short_tables(gpu, i4, d, group):
    """A workgroup of four waves per sequence: a table of 256 tokens, and more pairs of sequence and head than compute units."""
    check_decode(gpu, [0, 1, 31, 64, 129, 200, 256], 2 * group, 2, d, i4, False)
    check_decode(gpu, lengths(90, 350, 200, group), 4 * group, 4, d, i4, False)


@pytest.mark.parametrize("i4", [True, False])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("group", GROUPS)
def test_pieces_of_few_sequences(gpu, i4, d, group):
    """Shares, joined by several parts of a workgroup (more than four shares for a sequence)."""
    check_decode(gpu, [2900, 0, 1700], 2 * group, 2, d, i4, True)


@pytest.mark.parametrize("i4", [True, False])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("group", GROUPS)
def test_pieces_of_many_sequences(gpu, i4, d, group):
    """Shares, joined by one (up to four shares for a sequence)."""
    check_decode(gpu, lengths(36, 3200, 1500, group), 4 * group, 4, d, i4, True)


def test_pieces_of_sequences_with_heads_of_their_own(gpu):
    check_decode(gpu, lengths(24, 2000, 1500, 1), 32, 32, 64, False, True, page=32)


@pytest.mark.parametrize("n,KV", [(1030, 1), (260, 8)])
def test_a_long_sequence_among_very_many(gpu, n, KV):
    """Beyond 1024 sequences, or eight pairs of sequence and head on a compute unit, nothing is shared."""
    check_decode(gpu, lengths(n, 4000, 2100, n), 2 * KV, KV, 64, True, False)


@pytest.mark.parametrize("T,H,KV,d,i4,pairs", [(5501, 40, 4, 128, True, True), (5601, 42, 4, 64, True, False), (5601, 41, 3, 128, False, False),
                                               (8200, 30, 4, 64, False, True), (5901, 31, 7, 64, True, True)])
def test_append_of_many_rows(gpu, T, H, KV, d, i4, pairs):
    check_append(gpu, T, H, KV, d, 64, i4, pairs, False, seed=5)


@pytest.mark.parametrize("nq,nk,H,KV,d", [([300], [300], 12, 3, 128), ([5, 64, 1, 130, 0], [2050, 3000, 2200, 2500, 2300], 6, 2, 128), ([200, 77], [1200, 1111], 4, 2, 64),
                                          ([300, 20, 150], [300, 20, 150], 24, 2, 64), ([140] * 70, [150] * 70, 8, 8, 128), ([7] * 100, [9] * 100, 16, 4, 64),
                                          ([2200], [2200], 60, 4, 128)])
@pytest.mark.parametrize("causal", [True, False])
def test_output_over_the_queries(gpu, nq, nk, H, KV, d, causal):
    """In every shape of workgroup: bit for bit what an output of its own gets, where the queries are columns of a wider matrix."""
    print("case prefill in place", len(nq), sum(nq), H, KV, d, causal, flush=True)
    q, k, v = prefill.make(nq, nk, H, KV, d, seed=sum(nk))
    want = prefill.run(gpu, q, k, v, nq, nk, causal)
    few = [0, H - 1]
    at = [h * KV // H for h in few]
    prefill.check(want[:, few], q[:, few], k[:, at], v[:, at], nq, nk, causal, 1 / np.sqrt(d))
    wide = torch.full((sum(nq), H * d + 24), 7.0, dtype=torch.float16, device="cuda")
    Q = wide[:, 16:16 + H * d]
    Q.copy_(prefill.dev(q.reshape(len(q), -1)))
    K, V = (prefill.dev(x.reshape(len(x), -1)) for x in (k, v))
    gpu.sr_attn_prefill(Q, K, V, prefill.dev(prefill.ends(nq)), prefill.dev(prefill.ends(nk)), d, causal, O=Q)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(Q.cpu().numpy().reshape(want.shape), want)
    assert (wide[:, :16] == 7).all() and (wide[:, 16 + H * d:] == 7).all()
