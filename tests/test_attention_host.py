"""The cache and attention calls without a GPU: exported symbols, what is refused before a device is touched, the sizes of
workspaces, and the oracle that the GPU tests compare with."""
import ctypes
import os
import re

import numpy as np
import pytest

import paper_2506_05413_amd as sr
from oracle import attention_oracle as ao

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A, WS = 0x1000, 0x10000       # fake addresses, aligned to 16 and to 256 bytes; never followed on the host


def test_library_exports_what_the_header_declares():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "smoothrot_attention.h")).read(), flags=re.S)
    names = re.findall(r"SR_API\s+[\w\s\*]+?\b(sr_\w+)\s*\(", text)
    assert set(names) == set(sr.binding._ATTENTION_SIGNATURES) and len(names) == 5
    lib = ctypes.CDLL(sr.LIB_PATH)
    for n in names:
        assert hasattr(lib, n) and hasattr(sr, n), n


def cache(**changed):
    c = sr.sr_kv_cache(K=A, V=A, K_params=A, V_params=A, n_pages=4, page_size=16, n_kv_heads=2, head_dim=128, type=sr.SR_KV_I4)
    for k, v in changed.items():
        setattr(c, k, v)
    return c


BAD_CACHES = [(dict(type=2), sr.SR_ERR_ARG), (dict(type=-1), sr.SR_ERR_ARG), (dict(head_dim=96), sr.SR_ERR_ARG), (dict(head_dim=0), sr.SR_ERR_ARG),
              (dict(page_size=8), sr.SR_ERR_ARG), (dict(page_size=24), sr.SR_ERR_ARG), (dict(page_size=0), sr.SR_ERR_ARG), (dict(page_size=-16), sr.SR_ERR_ARG),
              (dict(page_size=1 << 21), sr.SR_ERR_ARG), (dict(n_pages=0), sr.SR_ERR_SHAPE), (dict(n_pages=1 << 31), sr.SR_ERR_SHAPE),
              (dict(n_pages=1 << 30, page_size=1 << 20), sr.SR_ERR_SHAPE), (dict(n_kv_heads=0), sr.SR_ERR_SHAPE), (dict(n_kv_heads=-2), sr.SR_ERR_SHAPE), (dict(n_kv_heads=1 << 16), sr.SR_ERR_SHAPE),
              (dict(K=None), sr.SR_ERR_NULL), (dict(V=None), sr.SR_ERR_NULL), (dict(K_params=None), sr.SR_ERR_NULL), (dict(V_params=None), sr.SR_ERR_NULL),
              (dict(K=A + 8), sr.SR_ERR_ALIGN), (dict(V=A + 4), sr.SR_ERR_ALIGN), (dict(K_params=A + 8), sr.SR_ERR_ALIGN), (dict(V_params=A + 4), sr.SR_ERR_ALIGN)]


def append(c=None, **changed):
    a = dict(Q=A, ldq=1024, K=A, ldk=256, V=A, ldv=256, T=3, H=8, positions=A, slots=A, table=A, max_pos=100, flags=0, clip=0.95, Qo=A, ldqo=1024, Ko=None, ldko=0)
    a.update(changed)
    c = cache() if c is None else c
    return sr.raw().sr_rope_kv_append(a["Q"], a["ldq"], a["K"], a["ldk"], a["V"], a["ldv"], a["T"], a["H"], a["positions"], a["slots"], a["table"], a["max_pos"],
                                      a["flags"], a["clip"], ctypes.byref(c) if c else None, a["Qo"], a["ldqo"], a["Ko"], a["ldko"], None)


def gather(c=None, **changed):
    a = dict(slots=A, T=3, Ko=A, ldko=256, Vo=A, ldvo=256)
    a.update(changed)
    c = cache() if c is None else c
    return sr.raw().sr_kv_gather(a["slots"], a["T"], ctypes.byref(c) if c else None, a["Ko"], a["ldko"], a["Vo"], a["ldvo"], None)


def decode(c=None, **changed):
    a = dict(Q=A, ldq=1024, B=3, H=8, table=A, pages=4, ld_table=4, lens=A, scale=0.1, O=A, ldo=1024, ws=WS, ws_bytes=1 << 30)
    a.update(changed)
    c = cache() if c is None else c
    return sr.raw().sr_attn_decode(a["Q"], a["ldq"], a["B"], a["H"], ctypes.byref(c) if c else None, a["table"], a["pages"], a["ld_table"], a["lens"], a["scale"],
                                   a["O"], a["ldo"], a["ws"], a["ws_bytes"], None)


def prefill(**changed):
    a = dict(Q=A, ldq=1024, K=A, ldk=256, V=A, ldv=256, cu_q=A, cu_k=A, n=2, Tq=10, Tk=10, H=8, KV=2, d=128, causal=1, scale=0.1, O=A, ldo=1024)
    a.update(changed)
    return sr.raw().sr_attn_prefill(a["Q"], a["ldq"], a["K"], a["ldk"], a["V"], a["ldv"], a["cu_q"], a["cu_k"], a["n"], a["Tq"], a["Tk"], a["H"], a["KV"], a["d"],
                                    a["causal"], a["scale"], a["O"], a["ldo"], None)


@pytest.mark.parametrize("call", [append, gather, decode])
def test_caches_that_are_refused(call):
    for changed, status in BAD_CACHES:
        assert call(cache(**changed)) == status, changed
    assert call(False) == sr.SR_ERR_NULL
    nothing = {"T": 0} if call is not decode else {"B": 0}
    assert call(cache(type=sr.SR_KV_F16, K_params=None, V_params=None), **nothing) == sr.SR_OK


NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("changed,status", [
    (dict(T=-1), sr.SR_ERR_SHAPE), (dict(H=-1), sr.SR_ERR_SHAPE), (dict(H=1 << 16, ldq=1 << 24, ldqo=1 << 24), sr.SR_ERR_SHAPE), (dict(ldq=1016), sr.SR_ERR_SHAPE), (dict(ldqo=1016), sr.SR_ERR_SHAPE),
    (dict(ldk=248), sr.SR_ERR_SHAPE), (dict(ldv=248), sr.SR_ERR_SHAPE), (dict(Ko=A, ldko=248), sr.SR_ERR_SHAPE), (dict(T=1 << 27), sr.SR_ERR_SHAPE),
    (dict(T=1 << 24), sr.SR_ERR_SHAPE), (dict(flags=4), sr.SR_ERR_ARG), (dict(clip=0.0), sr.SR_ERR_ARG), (dict(clip=1.01), sr.SR_ERR_ARG), (dict(clip=NAN), sr.SR_ERR_ARG),
    (dict(max_pos=0), sr.SR_ERR_SHAPE), (dict(max_pos=1 << 31), sr.SR_ERR_SHAPE), (dict(K=None), sr.SR_ERR_NULL), (dict(V=None), sr.SR_ERR_NULL),
    (dict(slots=None), sr.SR_ERR_NULL), (dict(positions=None), sr.SR_ERR_NULL), (dict(Q=None), sr.SR_ERR_NULL), (dict(Qo=None), sr.SR_ERR_NULL),
    (dict(ldq=1028), sr.SR_ERR_ALIGN), (dict(ldk=260), sr.SR_ERR_ALIGN), (dict(ldv=260), sr.SR_ERR_ALIGN), (dict(ldqo=1028), sr.SR_ERR_ALIGN), (dict(Ko=A, ldko=260), sr.SR_ERR_ALIGN),
    (dict(Q=A + 2), sr.SR_ERR_ALIGN), (dict(K=A + 8), sr.SR_ERR_ALIGN), (dict(V=A + 8), sr.SR_ERR_ALIGN), (dict(Qo=A + 8), sr.SR_ERR_ALIGN), (dict(Ko=A + 8, ldko=256), sr.SR_ERR_ALIGN),
    (dict(table=A + 4), sr.SR_ERR_ALIGN), (dict(T=0, Q=None, K=None, V=None, slots=None), sr.SR_OK)])
def test_append_refusals(changed, status):
    assert append(**changed) == status


@pytest.mark.parametrize("changed,status", [
    (dict(T=-1), sr.SR_ERR_SHAPE), (dict(T=1 << 27), sr.SR_ERR_SHAPE), (dict(T=1 << 25), sr.SR_ERR_SHAPE), (dict(ldko=248), sr.SR_ERR_SHAPE), (dict(ldvo=248), sr.SR_ERR_SHAPE),
    (dict(slots=None), sr.SR_ERR_NULL), (dict(Ko=None), sr.SR_ERR_NULL), (dict(Vo=None), sr.SR_ERR_NULL), (dict(ldko=260), sr.SR_ERR_ALIGN), (dict(ldvo=260), sr.SR_ERR_ALIGN),
    (dict(Ko=A + 2), sr.SR_ERR_ALIGN), (dict(Vo=A + 2), sr.SR_ERR_ALIGN), (dict(T=0, slots=None, Ko=None, Vo=None), sr.SR_OK)])
def test_gather_refusals(changed, status):
    assert gather(**changed) == status


@pytest.mark.parametrize("changed,status", [
    (dict(B=-1), sr.SR_ERR_SHAPE), (dict(B=1 << 20), sr.SR_ERR_SHAPE), (dict(H=0), sr.SR_ERR_SHAPE), (dict(H=7), sr.SR_ERR_SHAPE), (dict(H=1), sr.SR_ERR_SHAPE),
    (dict(pages=0), sr.SR_ERR_SHAPE), (dict(pages=(1 << 26) + 1, ld_table=1 << 27), sr.SR_ERR_SHAPE), (dict(ld_table=3), sr.SR_ERR_SHAPE), (dict(ldq=1016), sr.SR_ERR_SHAPE),
    (dict(ldo=1016), sr.SR_ERR_SHAPE), (dict(scale=0.0), sr.SR_ERR_ARG), (dict(scale=-1.0), sr.SR_ERR_ARG), (dict(scale=NAN), sr.SR_ERR_ARG), (dict(scale=INF), sr.SR_ERR_ARG), (dict(scale=2e19), sr.SR_ERR_ARG),
    (dict(Q=None), sr.SR_ERR_NULL), (dict(table=None), sr.SR_ERR_NULL), (dict(lens=None), sr.SR_ERR_NULL), (dict(O=None), sr.SR_ERR_NULL),
    (dict(ldq=1028), sr.SR_ERR_ALIGN), (dict(ldo=1028), sr.SR_ERR_ALIGN), (dict(Q=A + 8), sr.SR_ERR_ALIGN), (dict(O=A + 8), sr.SR_ERR_ALIGN),
    (dict(B=0, Q=None, table=None, lens=None, O=None, ws=None, ws_bytes=0), sr.SR_OK)])
def test_decode_refusals(changed, status):
    assert decode(**changed) == status


def test_decode_workspace():
    f = sr.sr_attn_decode_workspace_bytes
    need = f(1, 32, 8, 128, 512, 64)
    assert need > 0 and need % 4 == 0
    c, wide = cache(page_size=64, n_kv_heads=8), dict(B=1, H=32, ldq=4096, ldo=4096, pages=512, ld_table=512)
    assert decode(c, **wide, ws=None) == sr.SR_ERR_WORKSPACE
    assert decode(c, **wide, ws_bytes=need - 1) == sr.SR_ERR_WORKSPACE
    assert decode(c, **wide, ws=WS + 16) == sr.SR_ERR_WORKSPACE
    assert f(0, 32, 8, 128, 512, 64) == f(1, 32, 8, 96, 512, 64) == f(1, 30, 8, 128, 512, 64) == f(1, 32, 8, 128, 0, 64) == f(1, 32, 8, 128, 1 << 30, 64) == 0
    assert f(1, 32, 8, 128, 1, 16) == f(1, 32, 8, 128, 512, 64, 2) == f(1, 32, 8, 128, 512, 64, -1) == 0
    assert f(1, 32, 8, 128, 512, 64, sr.SR_KV_F16) > 0


@pytest.mark.parametrize("changed,status", [
    (dict(d=96), sr.SR_ERR_ARG), (dict(d=0), sr.SR_ERR_ARG), (dict(scale=0.0), sr.SR_ERR_ARG), (dict(scale=-0.5), sr.SR_ERR_ARG), (dict(scale=NAN), sr.SR_ERR_ARG), (dict(scale=INF), sr.SR_ERR_ARG), (dict(scale=2e19), sr.SR_ERR_ARG),
    (dict(n=-1), sr.SR_ERR_SHAPE), (dict(Tq=-1), sr.SR_ERR_SHAPE), (dict(Tk=-1), sr.SR_ERR_SHAPE), (dict(Tq=1 << 31), sr.SR_ERR_SHAPE), (dict(Tk=1 << 31), sr.SR_ERR_SHAPE),
    (dict(H=1 << 16, ldq=1 << 22, ldo=1 << 22), sr.SR_ERR_SHAPE), (dict(H=0), sr.SR_ERR_SHAPE), (dict(H=7), sr.SR_ERR_SHAPE), (dict(KV=0), sr.SR_ERR_SHAPE), (dict(KV=16), sr.SR_ERR_SHAPE),
    (dict(ldq=1016), sr.SR_ERR_SHAPE), (dict(ldo=1016), sr.SR_ERR_SHAPE), (dict(ldk=248), sr.SR_ERR_SHAPE), (dict(ldv=248), sr.SR_ERR_SHAPE),
    (dict(ldq=1 << 23), sr.SR_ERR_SHAPE), (dict(ldk=1 << 23), sr.SR_ERR_SHAPE), (dict(ldv=1 << 23), sr.SR_ERR_SHAPE), (dict(ldo=1 << 23), sr.SR_ERR_SHAPE),
    (dict(n=1 << 30, Tq=(1 << 31) - 1), sr.SR_ERR_SHAPE), (dict(Q=None), sr.SR_ERR_NULL), (dict(K=None), sr.SR_ERR_NULL), (dict(V=None), sr.SR_ERR_NULL), (dict(O=None), sr.SR_ERR_NULL),
    (dict(cu_q=None), sr.SR_ERR_NULL), (dict(cu_k=None), sr.SR_ERR_NULL), (dict(ldq=1028), sr.SR_ERR_ALIGN), (dict(ldk=260), sr.SR_ERR_ALIGN), (dict(ldv=260), sr.SR_ERR_ALIGN),
    (dict(ldo=1028), sr.SR_ERR_ALIGN), (dict(Q=A + 8), sr.SR_ERR_ALIGN), (dict(K=A + 8), sr.SR_ERR_ALIGN), (dict(V=A + 8), sr.SR_ERR_ALIGN), (dict(O=A + 8), sr.SR_ERR_ALIGN),
    (dict(Tq=0, Q=None, O=None, K=None, V=None, cu_q=None, cu_k=None), sr.SR_OK), (dict(n=0, Q=None), sr.SR_OK)])
def test_prefill_refusals(changed, status):
    assert prefill(**changed) == status


# ---- the oracle ------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("hadamard", [False, True])
def test_rotation_in_fp32_is_the_rotation(d, pairs, hadamard):
    rng = np.random.default_rng(d)
    x = rng.standard_normal((50, 3, d)).astype(np.float16)
    table, pos = ao.angles(100, d), rng.integers(0, 100, 50)
    exact = ao.rotate_heads_by_position(x, pos, table, pairs, hadamard)
    got = ao.rotate_heads_by_position(x, pos, table, pairs, hadamard, np.float32)
    # two products and a sum, half a step each: 3 u of the row's size at most; each of log2(d) sums adds as much of what it
    # sums, whose size a row's norm bounds
    size = np.linalg.norm(x.astype(np.float64), axis=-1, keepdims=True)
    assert got.dtype == np.float32 and (np.abs(got - exact) <= (3 + (np.log2(d) + 2 if hadamard else 0)) * 2.0 ** -24 * size).all()
    # lengths of rows and products of rows are kept
    np.testing.assert_allclose(np.linalg.norm(exact, axis=-1), size[..., 0], rtol=1e-6)
    # by hand: position 0 turns nothing, and a pair turns as a complex number
    still = ao.rotate_heads_by_position(x, np.zeros(50, int), table, pairs, False)
    np.testing.assert_array_equal(still, x.astype(np.float64))
    if not hadamard:
        a, b = (x[7, 0, 0], x[7, 0, 1]) if pairs else (x[7, 0, 0], x[7, 0, d // 2])
        z = complex(a, b) * np.exp(1j * pos[7])
        got = (exact[7, 0, 0], exact[7, 0, 1]) if pairs else (exact[7, 0, 0], exact[7, 0, d // 2])
        np.testing.assert_allclose(got, (z.real, z.imag), atol=1e-6)


def test_hadamard_of_heads_is_the_matrix():
    from oracle.smoothrot_oracle import sylvester
    x = np.random.default_rng(0).standard_normal((4, 128))
    np.testing.assert_allclose(ao.hadamard_heads(x), x @ sylvester(128) / np.sqrt(128), atol=1e-12)


def test_quantiser_is_the_group_quantiser():
    from oracle import smoothrot_oracle as o
    x = np.random.default_rng(1).standard_normal((30, 128)).astype(np.float16)
    codes, scale, zero = ao.quantise_heads(x, 0.95)
    c, s, z, _, _ = o.quant_asym_int4_groups(x, 128, float(np.float32(0.95)))
    np.testing.assert_array_equal(codes, c)
    np.testing.assert_allclose(scale, s[:, 0], rtol=1e-12)
    np.testing.assert_array_equal(zero, z[:, 0])
    np.testing.assert_array_equal(ao.unpack_uint4(o.pack_uint4(codes)), codes)
    np.testing.assert_allclose(ao.values_of(codes, scale, zero), o.dequant_asym(c, s, z, 128), rtol=1e-12)


def test_attention_by_hand():
    q, k, v = np.array([[1.0, 0.0], [0.0, 2.0]]), np.array([[1.0, 1.0], [2.0, 0.0], [5.0, 5.0]]), np.array([[1.0, 0.0], [0.0, 1.0], [9.0, 9.0]])
    o, p, s = ao.attend(q, k, v, 0.5, ao.causal(2, 3))
    np.testing.assert_array_equal(ao.causal(2, 3), [[True, True, False], [True, True, True]])
    np.testing.assert_array_equal(ao.causal(3, 1), [[False], [False], [True]])
    e = np.exp([0.5, 1.0])
    np.testing.assert_allclose(o[0], [e[0] / e.sum(), e[1] / e.sum()])
    assert (ao.attend(q, k, v, 1.0, np.zeros((2, 3), bool))[0] == 0).all()
