"""Pins of the serving oracle on the CPU, and the C ABI's checks of the serving entry points."""

import ctypes

import numpy as np
import pytest

import paper_2606_12487_amd as dptq
from oracle.serving import (PAGE, e4m3_encode, e4m3_values, kv8_append_ref, kv8_attention_ref, kv8_scale,
                            rms_norm_quant_ref, token_logprobs_ref)

OK, INVALID, UNSUPPORTED = 0, 1, 2
FAKE = ctypes.c_void_p(0x10000)           # aligned, never dereferenced
MISALIGNED = ctypes.c_void_p(0x10001)
NULL = ctypes.c_void_p(0)


def test_norm_codes_stand_for_the_normalised_row():
    rng = np.random.default_rng(0)
    x, res = (rng.standard_normal((6, 64)).astype(np.float16) for _ in range(2))
    w = rng.standard_normal(64).astype(np.float16)
    codes, scales, h = rms_norm_quant_ref(x, w, 1e-5, res)
    h64 = h.astype(np.float64)
    y = h64 / np.sqrt((h64 ** 2).mean(1, keepdims=True) + 1e-5) * w.astype(np.float64)
    assert np.abs(h64 - (x.astype(np.float64) + res.astype(np.float64))).max() <= 2.0 ** -9
    assert np.all(np.abs(codes * scales[:, None] - y) <= scales[:, None] * (0.5 + 1e-4))
    assert np.abs(codes).max(1).min() == 127


def test_e4m3():
    v = e4m3_values()
    assert v[0x7E] == 448 and v[1] == 2.0 ** -9 and v[8] == 2.0 ** -6 and np.isnan(v[0x7F])
    fine = ~np.isnan(v)
    assert np.array_equal(e4m3_encode(v[fine]), np.arange(256)[fine])
    assert e4m3_encode(np.array([17.0]))[0] == e4m3_encode(np.array([16.0]))[0]     # tie to even
    assert e4m3_encode(np.array([19.0]))[0] == e4m3_encode(np.array([20.0]))[0]
    for a in (0.0, 1.0, 448.0, 448.1, 65504.0, 6e-8):
        s = float(kv8_scale(a))
        assert a <= 448 * s and (s == 2.0 ** -32 or a > 224 * s)


def test_cache_and_attention_definitions():
    rng = np.random.default_rng(1)
    H, Hkv, D, n = 4, 2, 64, 90
    k, v = (rng.standard_normal((n, Hkv, D)).astype(np.float16) for _ in range(2))
    cache = [np.zeros((3, Hkv, PAGE, D), np.uint8), np.zeros((3, Hkv, D, PAGE), np.uint8),
             np.ones((3, Hkv), np.float32), np.ones((3, Hkv), np.float32)]
    table = np.array([[2, 0]], np.int32)
    got = kv8_append_ref(k, v, [0, n], [n], table, cache)
    q = rng.standard_normal((3, H, D)).astype(np.float16)
    out, lse, tol, _ = kv8_attention_ref(q, [0, 3], [n], table, got, 0.125, window=20, sinks=2)
    for i in range(3):
        p = n - 3 + i
        see = [j for j in range(p + 1) if j > p - 20 or j < 2]
        for h in range(H):
            s = 0.125 * (k[see, h // 2].astype(np.float64) @ q[i, h].astype(np.float64))
            w = np.exp(s) / np.exp(s).sum()
            # e4m3 keeps four significant bits: values are off by a sixteenth at most, scores by their sum
            assert np.abs(out[i, h] - w @ v[see, h // 2].astype(np.float64)).max() < 0.3
            assert abs(lse[i, h] - np.log(np.exp(s).sum())) < 0.2
    assert np.all(tol > 0)


def test_logprobs_definition():
    lp, ent, tops, ids = token_logprobs_ref(np.array([[0, 0, -np.inf, 0]]), [1], 2)
    assert np.allclose([lp[0], ent[0], tops[0, 0]], [-np.log(3), np.log(3), -np.log(3)])
    assert ids.tolist() == [[0, 1]]


@pytest.fixture(scope="module")
def L():
    import os
    if not os.path.exists(dptq.library_path()):
        import __graft_entry__
        __graft_entry__.build()
    return dptq.lib()


def test_norm_validation(L):
    def f(x=FAKE, res=FAKE, w=FAKE, M=4, K=256, eps=1e-5, s=FAKE, c=FAKE, sc=FAKE):
        return L.dptq_rms_norm_quant(x, res, w, M, K, eps, s, c, sc, NULL)
    assert f(M=-1) == INVALID and f(K=0) == INVALID and f(K=252) == INVALID
    assert f(K=65544) == UNSUPPORTED and f(M=1 << 31) == UNSUPPORTED
    for eps in (-1.0, float("nan"), float("inf")):
        assert f(eps=eps) == INVALID
    for name in ("x", "w", "c", "sc"):
        assert f(**{name: NULL}) == INVALID, name
        assert f(**{name: MISALIGNED}) == INVALID, name
    assert f(res=MISALIGNED) == INVALID and f(s=MISALIGNED) == INVALID
    assert f(res=NULL) == INVALID and f(s=NULL) == INVALID      # a sum without a residual, and the reverse
    assert f(M=0, x=NULL, w=NULL) == OK


def append(L, k=FAKE, ldk=256, v=FAKE, ldv=256, T=4, cu=FAKE, n=FAKE, B=2, t=FAKE, mp=4, P=8, H=2, D=128, kp=FAKE,
           vp=FAKE, ks=FAKE, vs=FAKE, mx=0):
    return L.dptq_kv8_append(k, ldk, v, ldv, T, cu, n, B, t, mp, P, H, D, kp, vp, ks, vs, mx, NULL)


def attend(L, q=FAKE, ld=512, T=4, cu=FAKE, n=FAKE, B=2, t=FAKE, mp=4, P=8, H=4, Hkv=2, D=128, kp=FAKE, vp=FAKE,
           ks=FAKE, vs=FAKE, scale=0.1, window=0, sinks=0, mq=0, ml=0, out=FAKE, lse=FAKE, w=FAKE, wb=1 << 40):
    return L.dptq_kv8_attention(q, ld, T, cu, n, B, t, mp, P, H, Hkv, D, kp, vp, ks, vs, scale, window, sinks, mq, ml,
                                out, lse, w, wb, NULL)


def test_kv8_validation(L):
    for f in (lambda **kw: append(L, **kw), lambda **kw: attend(L, **kw)):
        assert f(T=-1) == INVALID and f(B=-1) == INVALID and f(mp=-1) == INVALID and f(P=-1) == INVALID
        assert f(D=96) == UNSUPPORTED and f(D=0) == INVALID
        assert f(T=1 << 30) == UNSUPPORTED and f(B=65536) == UNSUPPORTED and f(mp=1 << 25) == UNSUPPORTED
        for name in ("cu", "n", "t", "kp", "vp", "ks", "vs"):
            assert f(**{name: NULL}) == INVALID, name
            assert f(**{name: MISALIGNED}) == INVALID, name
        assert f(T=0, cu=NULL, kp=NULL) == OK and f(B=0, cu=NULL, kp=NULL) == OK
    assert append(L, H=0) == INVALID and append(L, H=1025) == UNSUPPORTED and append(L, mx=-1) == INVALID
    for name in ("k", "v"):
        assert append(L, **{name: NULL}) == INVALID and append(L, **{name: MISALIGNED}) == INVALID
    for name in ("ldk", "ldv"):
        assert append(L, **{name: 248}) == INVALID and append(L, **{name: 260}) == INVALID
    assert append(L, mp=0) == OK and append(L, P=0) == OK
    assert attend(L, H=3) == INVALID and attend(L, H=0) == INVALID and attend(L, H=1 << 17) == UNSUPPORTED
    assert attend(L, ld=504) == INVALID and attend(L, ld=516) == INVALID
    assert attend(L, window=-1) == INVALID and attend(L, sinks=-1) == INVALID
    assert attend(L, window=1 << 30) == UNSUPPORTED and attend(L, sinks=1 << 30) == UNSUPPORTED
    assert attend(L, mq=-1) == INVALID and attend(L, ml=-1) == INVALID
    for scale in (float("nan"), float("inf"), -float("inf")):
        assert attend(L, scale=scale) == INVALID
    for name in ("q", "out", "lse"):
        assert attend(L, **{name: NULL}) == INVALID and attend(L, **{name: MISALIGNED}) == INVALID
    assert L.dptq_kv8_attention_workspace(4, 2, 4, 3, 2, 128, 0, 0, 0, 0) == -1
    assert L.dptq_kv8_attention_workspace(0, 2, 4, 4, 2, 128, 0, 0, 0, 0) == 0


def test_logprobs_validation(L):
    def f(x=FAKE, dt=1, ld=100, M=4, V=100, t=FAKE, top=5, lp=FAKE, e=FAKE, tl=FAKE, ti=FAKE, w=FAKE, wb=1 << 40):
        return L.dptq_token_logprobs(x, dt, ld, M, V, t, top, lp, e, tl, ti, w, wb, NULL)
    assert f(M=-1) == INVALID and f(V=0) == INVALID and f(ld=99) == INVALID and f(dt=2) == INVALID
    assert f(top=-1) == INVALID and f(top=65) == UNSUPPORTED and f(V=3, top=4) == INVALID
    assert f(V=1 << 30, ld=1 << 30) == UNSUPPORTED and f(M=1 << 31) == UNSUPPORTED
    for name in ("x", "t", "lp", "e", "tl", "ti"):
        assert f(**{name: NULL}) == INVALID, name
        assert f(**{name: MISALIGNED}) == INVALID, name
    assert f(M=0, x=NULL, t=NULL) == OK
    assert L.dptq_token_logprobs_workspace(4, 100, 101, 0) == -1
