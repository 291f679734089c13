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
