"""What the serving operators refuse, before anything is enqueued (no GPU needed): the C ABI with pointers that are
never read, and the binding's own checks."""

import ctypes
import math

import pytest

torch = pytest.importorskip("torch")
dptq = pytest.importorskip("paper_2606_12487_amd")

OK, INVALID, UNSUPPORTED = 0, 1, 2
P = 0x1000   # an aligned address that nothing reads


@pytest.fixture(scope="module")
def L():
    return dptq.lib()


def _call(f, names, good, **changes):
    assert set(changes) <= set(names), changes
    return f(*[{**good, **changes}[n] for n in names])


ROTARY = ["q", "ld_q", "heads", "k", "ld_k", "kv_heads", "T", "D", "positions", "inv_freq", "r", "interleaved", "scale",
          "q_out", "ld_q_out", "k_out", "ld_k_out", "stream"]
ROTARY_GOOD = dict(q=P, ld_q=512, heads=4, k=P, ld_k=256, kv_heads=2, T=3, D=128, positions=P, inv_freq=P, r=128,
                   interleaved=0, scale=1.0, q_out=2 * P, ld_q_out=512, k_out=2 * P, ld_k_out=256, stream=None)


@pytest.mark.parametrize("status,changes", [
    (INVALID, dict(T=-1)), (INVALID, dict(heads=0)), (INVALID, dict(kv_heads=-1)), (INVALID, dict(D=0)),
    (INVALID, dict(D=132, r=128)), (INVALID, dict(r=0)), (INVALID, dict(r=63)), (INVALID, dict(r=130)),
    (INVALID, dict(r=-2)), (INVALID, dict(scale=math.nan)), (INVALID, dict(scale=math.inf)),
    (UNSUPPORTED, dict(T=1 << 30)), (UNSUPPORTED, dict(D=520)), (UNSUPPORTED, dict(heads=8191)),
    (UNSUPPORTED, dict(heads=2 ** 31 - 1, kv_heads=2 ** 31 - 1)),
    (INVALID, dict(q=None)), (INVALID, dict(k=None)), (INVALID, dict(positions=None)), (INVALID, dict(inv_freq=None)),
    (INVALID, dict(q_out=None)), (INVALID, dict(k_out=None)), (INVALID, dict(q=P + 8)), (INVALID, dict(k_out=P + 2)),
    (INVALID, dict(ld_q=504)), (INVALID, dict(ld_k=260)), (INVALID, dict(ld_q_out=511)), (INVALID, dict(ld_k_out=0)),
    (INVALID, dict(positions=P + 2)), (INVALID, dict(inv_freq=P + 4)),
    (INVALID, dict(q_out=P, ld_q_out=1024)), (INVALID, dict(k_out=P, ld_k_out=512)),
    (OK, dict(T=0)), (OK, dict(T=0, q=None, k=None, positions=None, inv_freq=None)),
])
def test_rotary(L, status, changes):
    assert _call(L.dptq_rotary, ROTARY, ROTARY_GOOD, **changes) == status


APPEND = ["q", "ld_q", "heads", "k", "ld_k", "v", "ld_v", "T", "cu", "lengths", "B", "table", "max_pages", "num_pages",
          "kv_heads", "D", "k_pages", "v_pages", "k_scales", "v_scales", "inv_freq", "r", "interleaved", "scale",
          "q_out", "ld_q_out", "max_new", "stream"]
APPEND_GOOD = dict(q=P, ld_q=512, heads=4, k=P, ld_k=256, v=P, ld_v=256, T=3, cu=P, lengths=P, B=1, table=P, max_pages=4,
                   num_pages=4, kv_heads=2, D=128, k_pages=P, v_pages=P, k_scales=P, v_scales=P, inv_freq=P, r=128,
                   interleaved=0, scale=1.0, q_out=2 * P, ld_q_out=512, max_new=0, stream=None)


@pytest.mark.parametrize("status,changes", [
    (INVALID, dict(T=-1)), (INVALID, dict(B=-1)), (INVALID, dict(heads=0)), (INVALID, dict(kv_heads=0)),
    (UNSUPPORTED, dict(D=96, r=96)), (UNSUPPORTED, dict(kv_heads=1025)), (UNSUPPORTED, dict(heads=8191)),
    (UNSUPPORTED, dict(B=65536)), (INVALID, dict(r=130)), (INVALID, dict(r=5)), (INVALID, dict(scale=-math.inf)),
    (INVALID, dict(max_new=-1)), (INVALID, dict(q=None)), (INVALID, dict(k=None)), (INVALID, dict(v=P + 4)),
    (INVALID, dict(cu=None)), (INVALID, dict(k_pages=None)), (INVALID, dict(table=None)), (INVALID, dict(inv_freq=None)),
    (INVALID, dict(inv_freq=P + 4)), (INVALID, dict(q_out=None)), (INVALID, dict(q_out=P, ld_q_out=520)),
    (INVALID, dict(ld_v=248)), (OK, dict(T=0)), (OK, dict(B=0)),
])
def test_rotary_kv8_append(L, status, changes):
    assert _call(L.dptq_rotary_kv8_append, APPEND, APPEND_GOOD, **changes) == status


GATED = ["codes", "a_scales", "M", "K", "bits", "w", "weights", "w_scales", "F", "act", "y", "stream"]
GATED_GOOD = dict(codes=P, a_scales=P, M=4, K=256, bits=8, w=P, weights=0, w_scales=P, F=32, act=0, y=P, stream=None)


@pytest.mark.parametrize("status,changes", [
    (INVALID, dict(M=-1)), (INVALID, dict(F=0)), (INVALID, dict(F=12)), (INVALID, dict(F=-8)), (INVALID, dict(bits=5)),
    (UNSUPPORTED, dict(K=200)), (UNSUPPORTED, dict(K=1 << 17)), (UNSUPPORTED, dict(F=1 << 30)), (INVALID, dict(act=2)),
    (INVALID, dict(act=-1)), (INVALID, dict(weights=1)), (INVALID, dict(weights=4)), (INVALID, dict(weights=2, bits=4)),
    (UNSUPPORTED, dict(weights=3, M=17)), (INVALID, dict(codes=None)), (INVALID, dict(a_scales=None)),
    (INVALID, dict(w=None)), (INVALID, dict(w_scales=None)), (INVALID, dict(y=None)), (INVALID, dict(codes=P + 8)),
    (INVALID, dict(a_scales=P + 4)), (INVALID, dict(w_scales=P + 4)), (INVALID, dict(y=P + 2)), (INVALID, dict(w=P + 1)),
    (OK, dict(M=0, codes=None, y=None)),
])
def test_gated(L, status, changes):
    assert _call(L.dptq_qlinear_gated, GATED, GATED_GOOD, **changes) == status


FP6 = ["a6", "a_scales", "M", "K", "w6", "w_scales", "F", "act", "y", "stream"]
FP6_GOOD = dict(a6=P, a_scales=P, M=40, K=256, w6=P, w_scales=P, F=32, act=1, y=P, stream=None)


@pytest.mark.parametrize("status,changes", [
    (INVALID, dict(M=-1)), (INVALID, dict(F=4)), (UNSUPPORTED, dict(K=64)), (INVALID, dict(act=7)),
    (INVALID, dict(a6=None)), (INVALID, dict(a_scales=P + 2)), (INVALID, dict(w6=P + 4)), (INVALID, dict(w_scales=None)),
    (INVALID, dict(y=P + 8)), (OK, dict(M=0, a6=None)),
])
def test_gated_fp6(L, status, changes):
    assert _call(L.dptq_qlinear_gated_fp6, FP6, FP6_GOOD, **changes) == status


SAMPLE = ["logits", "dtype", "ld", "M", "V", "uniform", "temperature", "t", "top_k", "k", "top_p", "p", "min_p", "m",
          "tokens", "probs", "workspace", "bytes", "stream"]
SAMPLE_GOOD = dict(logits=P, dtype=0, ld=1000, M=600, V=1000, uniform=P, temperature=P, t=1.0, top_k=P, k=0, top_p=P,
                   p=1.0, min_p=P, m=0.0, tokens=P, probs=P, workspace=None, bytes=0, stream=None)


@pytest.mark.parametrize("status,changes", [
    (INVALID, dict(M=-1)), (INVALID, dict(V=0)), (INVALID, dict(ld=999)), (INVALID, dict(dtype=2)),
    (UNSUPPORTED, dict(M=1 << 31)), (UNSUPPORTED, dict(V=1 << 30, ld=1 << 30)), (INVALID, dict(logits=None)),
    (INVALID, dict(uniform=None)), (INVALID, dict(tokens=None)), (INVALID, dict(probs=None)), (INVALID, dict(logits=P + 1)),
    (INVALID, dict(dtype=1, logits=P + 2)), (INVALID, dict(uniform=P + 2)), (INVALID, dict(temperature=P + 1)),
    (INVALID, dict(top_k=P + 2)), (INVALID, dict(top_p=P + 2)), (INVALID, dict(min_p=P + 2)),
    (INVALID, dict(tokens=P + 4)), (INVALID, dict(probs=P + 2)),
    (INVALID, dict(M=1, V=100000, ld=100000)), (INVALID, dict(M=1, V=100000, ld=100000, workspace=P, bytes=1000)),
    (INVALID, dict(M=1, V=100000, ld=100000, workspace=P + 8, bytes=1 << 30)), (OK, dict(M=0, logits=None)),
])
def test_sample_tokens(L, status, changes):
    assert _call(L.dptq_sample_tokens, SAMPLE, SAMPLE_GOOD, **changes) == status


def test_sample_tokens_workspace(L):
    assert L.dptq_sample_tokens_workspace(0, 100, 0) == 0 and L.dptq_sample_tokens_workspace(1, 0, 0) == -1
    assert L.dptq_sample_tokens_workspace(1, 100, 5) == -1 and L.dptq_sample_tokens_workspace(-1, 100, 0) == -1
    assert L.dptq_sample_tokens_workspace(1, 100, 0) == 0 and L.dptq_sample_tokens_workspace(1, 1 << 17, 1) > 0


def test_gate_up_rows():
    gate, up = torch.arange(48).view(24, 2), torch.arange(100, 148).view(24, 2)
    w = dptq.gate_up_rows(gate, up)
    assert w.shape == (48, 2) and w.is_contiguous()
    for f in range(24):
        row = f // 8 * 16 + f % 8
        assert torch.equal(w[row], gate[f]) and torch.equal(w[row + 8], up[f])
    for a, b in ((gate[:20], up[:20]), (gate, up[:16]), (gate, up.float()), (gate[:0], up[:0])):
        with pytest.raises(ValueError):
            dptq.gate_up_rows(a, b)


def test_frequencies():
    f = dptq.rotary_inv_freq(64, device="cpu")
    assert f.dtype == torch.float64 and f.tolist() == [10000.0 ** (-i / 32) for i in range(32)]
    assert dptq.rotary_inv_freq(64, factor=4.0, device="cpu").tolist() == [x / 4 for x in f.tolist()]
    for ramp in ("turns", "index"):
        g = dptq.rotary_inv_freq(64, factor=8.0, original_length=8192, low_turns=1, high_turns=32, ramp=ramp,
                                 device="cpu").tolist()
        turns = [8192 * x / (2 * math.pi) for x in f.tolist()]
        for x, y, t in zip(f.tolist(), g, turns):
            assert x / 8 * (1 - 1e-15) <= y <= x
            if t >= 64:
                assert y == x
            if t <= 0.5:
                assert y == pytest.approx(x / 8, rel=1e-15)
        assert g == sorted(g, reverse=True)
    for bad in (dict(rotary_dim=3), dict(rotary_dim=0), dict(base=1.0), dict(factor=0.0), dict(ramp="x"),
                dict(original_length=0), dict(original_length=10, low_turns=4.0, high_turns=4.0)):
        with pytest.raises(ValueError):
            dptq.rotary_inv_freq(**{"rotary_dim": 8, "device": "cpu", **bad})


def test_binding_refuses_cpu_tensors():
    x = torch.zeros((1, 4, 64), dtype=torch.float16)
    p, f = torch.zeros(1, dtype=torch.int32), dptq.rotary_inv_freq(64, device="cpu")
    with pytest.raises(ValueError, match="GPU"):
        dptq.rotary(x, None, p, f)
    with pytest.raises(TypeError, match="float16"):
        dptq.rotary(x.float(), None, p, f)
