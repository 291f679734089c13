"""GPU parity of rms_norm_quant: codes and sums bit for bit, scales in float64."""

import numpy as np
import pytest

from oracle.serving import rms_norm_quant_ref

torch = pytest.importorskip("torch")
dptq = pytest.importorskip("paper_2606_12487_amd")

pytestmark = pytest.mark.gpu

# At most 64 squares a thread in turn, then a tree of ten levels, halved by the
# square root; the root, the quotients and the products add six roundings.
SCALE_TOL = (74 / 2 + 6) * 2.0 ** -24


def _d(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _check(x, w, eps, res):
    got = dptq.rms_norm_quant(_d(x), _d(w), eps, None if res is None else _d(res))
    codes, scales, h = (t.cpu().numpy() for t in got)
    rc, rs, rh = rms_norm_quant_ref(x, w, eps, res)
    assert np.array_equal(h.view(np.uint16), rh.view(np.uint16))
    assert np.array_equal(codes, rc)
    assert np.all(np.abs(scales - rs) <= SCALE_TOL * rs)


@pytest.mark.parametrize("M,K", [(1, 8), (3, 16), (1, 4096), (5, 2048), (2, 2056), (7, 5120), (33, 8192), (2, 8200),
                                 (3, 32768), (2, 32776), (2, 65536), (513, 1032), (1030, 4096),
                                 (2 ** 20 + 3, 8)])
@pytest.mark.parametrize("add", [True, False])
def test_norm_matches_oracle(M, K, add):
    rng = np.random.default_rng(M * 31 + K)
    x = rng.standard_normal((M, K)).astype(np.float16)
    res = rng.standard_normal((M, K)).astype(np.float32)
    res[:, rng.choice(K, 2, replace=False)] *= 100
    w = (1 + 0.2 * rng.standard_normal(K)).astype(np.float16)
    _check(x, w, 1e-5, res.astype(np.float16) if add else None)


def test_norm_special_rows():
    rng = np.random.default_rng(5)
    K = 256
    x = rng.standard_normal((8, K)).astype(np.float16)
    res = np.zeros((8, K), np.float16)
    w = rng.standard_normal(K).astype(np.float16)
    w[:7] = 0
    x[0] = 0                                    # a row of zeros
    x[1] = np.float16(6e-8)                     # subnormals
    x[2] = 60000                                # large values
    x[3, 1:] = 0                                # one value, whose weight is 0
    x[4] = -x[4]
    res[5] = -x[5]                              # cancels exactly
    x[6, :] = rng.choice([-1.0, 1.0], K)        # ties of the codes
    res[7] = np.float16(1e-3)
    for eps in (0.0, 1e-6, 1.0):
        _check(x, w, eps, res)
        _check(x, np.ones(K, np.float16), eps, res)


def test_norm_codes_at_ties():
    # t / s on and beside halves: a row whose largest value is 127 has s = 1.
    K = 1024
    t = (np.arange(K) % 254 - 126.5).astype(np.float16)
    x = np.stack([t, np.nextafter(t, np.float16(1000)), np.nextafter(t, np.float16(-1000))])
    x[:, 0] = 127
    _check(x, np.ones(K, np.float16), 1e-5, None)


def test_norm_in_place_and_streams():
    rng = np.random.default_rng(6)
    x, res = (rng.standard_normal((9, 4096)).astype(np.float16) for _ in range(2))
    w = rng.standard_normal(4096).astype(np.float16)
    rc, _, rh = rms_norm_quant_ref(x, w, 1e-5, res)
    for into in ("residual", "x"):
        xd, rd = _d(x), _d(res)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            buf = rd if into == "residual" else xd
            codes, scales, h = dptq.rms_norm_quant(xd, _d(w), 1e-5, rd, sum=buf)
        side.synchronize()
        assert h is buf
        assert np.array_equal(h.cpu().numpy(), rh) and np.array_equal(codes.cpu().numpy(), rc)


def test_norm_feeds_the_linear():
    # The codes are qlinear's 8-bit activations on weights without a rotation.
    from oracle import prepare_weights_ref, qlinear_ref
    rng = np.random.default_rng(7)
    x = rng.standard_normal((5, 512)).astype(np.float16)
    w = np.ones(512, np.float16)
    wp, ws = prepare_weights_ref((0.02 * rng.standard_normal((64, 512))).astype(np.float32), 1)
    codes, scales, _ = dptq.rms_norm_quant(_d(x), _d(w), 1e-5)
    y = dptq.qlinear(codes, scales, 8, _d(wp), _d(ws)).cpu().numpy()
    ref = qlinear_ref(codes.cpu().numpy(), scales.cpu().numpy(), 8, wp, ws)
    assert np.array_equal(y.view(np.uint16), ref.view(np.uint16))


def test_norm_refusals():
    x = torch.zeros((2, 64), dtype=torch.float16, device="cuda")
    w = torch.ones(64, dtype=torch.float16, device="cuda")
    with pytest.raises(TypeError, match="weight must have dtype torch.float16"):
        dptq.rms_norm_quant(x, w.float(), 1e-5)
    with pytest.raises(ValueError, match="weight must have shape"):
        dptq.rms_norm_quant(x, w[:8], 1e-5)
    with pytest.raises(ValueError, match="residual must have shape"):
        dptq.rms_norm_quant(x, w, 1e-5, x[:1])
    with pytest.raises(ValueError, match="sum is given without a residual"):
        dptq.rms_norm_quant(x, w, 1e-5, sum=x)
    with pytest.raises(ValueError, match="must be contiguous"):
        dptq.rms_norm_quant(torch.zeros((64, 4), dtype=torch.float16, device="cuda").t(), w, 1e-5)
    for call in (lambda: dptq.rms_norm_quant(x[:, :12].contiguous(), w[:12], 1e-5),
                 lambda: dptq.rms_norm_quant(x, w, -1.0), lambda: dptq.rms_norm_quant(x, w, float("nan"))):
        with pytest.raises(dptq.DptqError) as e:
            call()
        assert e.value.status == 1
    codes, scales, h = dptq.rms_norm_quant(x[:0], w, 1e-5, x[:0])
    assert codes.shape == (0, 64) and scales.shape == (0,) and h.shape == (0, 64)
