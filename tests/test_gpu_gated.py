"""The gated feed-forward block on every kernel of the GEMMs: the shapes at which the dispatch picks each of them, ragged
ones among them, against the activation and the product in 64 bits of the exact accumulators; each weight layout bit
for bit the same.  The accumulators themselves are checked in the GEMMs' own tests."""

import numpy as np
import pytest

import workloads
from oracle.gated import gate_up_order, gated_ref
from test_gpu_fp6_ksplit import CASES as FP6_CASES
from test_gpu_ksplit import CASES as KSPLIT_CASES

torch = pytest.importorskip("torch")
dptq = pytest.importorskip("paper_2606_12487_amd")

pytestmark = pytest.mark.gpu

ACTS = ["silu", "gelu_tanh"]


def _operands(M, K, N, bits, size=3.0):
    """Codes, weights and scales on the GPU; g and u of about `size`."""
    rng = np.random.default_rng([M, K, N, bits])
    a = torch.from_numpy(workloads.random_code_bytes(rng, M, K, bits)).cuda()
    w = torch.from_numpy(workloads.random_weight_bytes(rng, N, K)).cuda()
    a_s = torch.from_numpy(rng.uniform(0.5, 2.0, M).astype(np.float32)).cuda()
    spread = (4.6 if bits == 4 else 74.0) * 4.6 * K ** 0.5
    w_s = torch.from_numpy((rng.uniform(0.5, 2.0, N) * size / spread).astype(np.float32)).cuda()
    return a, a_s, w, w_s


def _close(y, acc, a_s, w_s, act, what=""):
    """In units of 2^-24: g and u have three roundings each, and the argument of the sigmoid, t (of which a relative
    error counts |t| times, three times over in the cube of the GELU), at most twelve; exp and the reciprocal one each
    and the products two.  Then the rounding to fp16: 2^-11, or 2^-25 below its normal range."""
    z = acc.double() * a_s.double()[:, None] * w_s.double()
    z = z.view(z.shape[0], -1, 2, 8)
    g, u = z[:, :, 0].flatten(1), z[:, :, 1].flatten(1)
    t = g if act == "silu" else (8 / torch.pi) ** 0.5 * (g + 0.044715 * g ** 3)
    want = g * u * torch.sigmoid(t)
    error = (y.double() - want).abs()
    tolerance = want.abs() * (2.0 ** -11 + 2.0 ** -24 * (16 + 16 * t.abs())) + 2.0 ** -25
    inside = want.abs() <= 65000
    assert bool((error <= tolerance)[inside].all()), (what, float((error / tolerance)[inside].max()))
    assert bool(inside.float().mean() > 0.99)


@pytest.mark.parametrize("M,K,N,bits", KSPLIT_CASES)
def test_each_int8_kernel(M, K, N, bits):
    a, a_s, w, w_s = _operands(M, K, N, bits)
    act = ACTS[(M + N // 16) % 2]
    acc = dptq.qlinear_acc(a, bits, w)
    y = dptq.qlinear_gated(a, a_s, bits, w, w_s, activation=act)
    _close(y, acc, a_s, w_s, act, (M, K, N, bits))
    if bits == 8:
        assert torch.equal(dptq.qlinear_gated_a8(a, a_s, dptq.pack_w4_a8(w), w_s, activation=act), y)
    else:
        y6 = dptq.qlinear_gated_fp6(dptq.pack_fp6(a), a_s, dptq.pack_fp6(w), w_s, M, K, N // 2, activation=act)
        assert torch.equal(y6, y)
    if M <= 16:
        wd = dptq.prepack_weights(w, dptq.WEIGHTS_DECODE)
        assert torch.equal(dptq.qlinear_gated_decode_native(a, a_s, bits, wd, w_s, activation=act), y)


# The two tile kernels: fewer rows or k than the wide one takes, ragged ones, its shifted edge tiles.
TILE_CASES = [(640, 256, 11008, 4), (1100, 256, 8208, 8), (300, 4096, 28672, 8), (1033, 1024, 8224, 4),
              (2049, 640, 12304, 8), (2100, 512, 16400, 4), (4001, 1152, 6160, 8)]


@pytest.mark.parametrize("M,K,N,bits", TILE_CASES)
def test_each_tile_kernel(M, K, N, bits):
    test_each_int8_kernel(M, K, N, bits)


# The gated products' own tiles: ragged rows and channels, a last stage of 128 k, one to three rounds.
# test_gated_rules.py keeps each on the tile named at 256 compute units.
SMALL_CASES = [(211, 384, 10960, 4), (211, 384, 10960, 8), (100, 1152, 28688, 4), (300, 1152, 8208, 8),
               (129, 128, 12304, 8), (65536, 128, 64, 8)]
TALL_CASES = [(339, 1152, 30256, 4), (339, 1152, 30256, 8), (190, 128, 54096, 4), (190, 640, 54096, 8),
              (2100, 512, 16400, 4), (1100, 256, 8208, 8)]


@pytest.mark.parametrize("M,K,N,bits", SMALL_CASES + TALL_CASES)
def test_each_gated_tile(M, K, N, bits):
    test_each_int8_kernel(M, K, N, bits)


@pytest.mark.parametrize("M,N,K", FP6_CASES)
def test_each_fp6_kernel(M, N, K):
    a, a_s, w, w_s = _operands(M, K, N, 4)
    for act in ACTS:
        y = dptq.qlinear_gated_fp6(dptq.pack_fp6(a), a_s, dptq.pack_fp6(w), w_s, M, K, N // 2, activation=act)
        _close(y, dptq.qlinear_acc(a, 4, w), a_s, w_s, act, (M, N, K))
        assert torch.equal(y, dptq.qlinear_gated(a, a_s, 4, w, w_s, activation=act))


@pytest.mark.parametrize("M,K,F,bits", [(1, 256, 8, 4), (5, 128, 24, 8), (40, 256, 48, 4), (300, 640, 104, 8)])
@pytest.mark.parametrize("act", ACTS)
def test_matches_the_oracle(M, K, F, bits, act):
    """From fp32 weights: the order of the rows, and values from the oracle's own product."""
    rng = np.random.default_rng([M, K, F])
    x = workloads.gauss_massive(rng, M, K)
    gate, up = workloads.weights(rng, F, K), workloads.weights(rng, F, K)
    w = dptq.gate_up_rows(*(torch.from_numpy(v).cuda() for v in (gate, up)))
    assert np.array_equal(w.cpu().numpy(), np.concatenate([gate, up])[gate_up_order(F)])
    wp, ws = dptq.prepare_weights(w, K & -K)
    codes, scales = dptq.rotate_quant(torch.from_numpy(x).cuda(), K & -K, bits)
    y = dptq.qlinear_gated(codes, scales, bits, wp, ws, activation=act)
    c, s, p, q = (v.cpu().numpy() for v in (codes, scales, wp, ws))
    want, g, _ = gated_ref(c, s, bits, p, q, act)
    t = np.abs(g) if act == "silu" else np.abs((8 / np.pi) ** 0.5 * (g + 0.044715 * g ** 3))
    error = np.abs(y.cpu().numpy().astype(np.float64) - want)
    assert (error <= np.abs(want) * (2.0 ** -11 + 2.0 ** -24 * (16 + 16 * t)) + 2.0 ** -25).all()
    # Packed rows and scales take the order as well.
    half = [dptq.prepare_weights(torch.from_numpy(v).cuda(), K & -K) for v in (gate, up)]
    assert torch.equal(dptq.gate_up_rows(half[0][0], half[1][0]), wp)
    assert torch.equal(dptq.gate_up_rows(half[0][1], half[1][1]), ws)


@pytest.mark.parametrize("act", ACTS)
def test_far_arguments(act):
    """Gates so far out that exp overflows or the sigmoid is 1, and zeros."""
    M, K, F, bits = 17, 128, 64, 8
    a, a_s, w, w_s = _operands(M, K, 2 * F, bits)
    a[3] = 0
    acc = dptq.qlinear_acc(a, bits, w)
    a_s[:] = torch.logspace(-8, 8, M, device="cuda")
    w_s.view(-1, 2, 8)[:, 1] *= 1e-8                       # up channels, so that products stay within fp16
    y = dptq.qlinear_gated(a, a_s, bits, w, w_s, activation=act)
    assert bool(torch.isfinite(y[:-4]).all()) and not bool(torch.isnan(y).any()) and bool((y[3] == 0).all())
    z = (acc.double() * a_s.double()[:, None] * w_s.double()).view(M, -1, 2, 8)
    g, u = z[:, :, 0].flatten(1), z[:, :, 1].flatten(1)
    want = torch.where(g > 100, g * u, 0.0).clamp(-1e300, 1e300)
    far = (g.abs() > 100) & (want.abs() < 65000)
    assert bool(far.any()) and bool(((y.double() - want).abs() <= want.abs() * 2.0 ** -10 + 2.0 ** -25)[far].all())


def test_given_outputs_and_no_rows():
    a, a_s, w, w_s = _operands(20, 256, 64, 4)
    y = torch.empty((20, 32), dtype=torch.float16, device="cuda")
    assert dptq.qlinear_gated(a, a_s, 4, w, w_s, y=y) is y
    assert torch.equal(y, dptq.qlinear_gated(a, a_s, 4, w, w_s))
    assert dptq.qlinear_gated(a[:0], a_s[:0], 4, w, w_s).shape == (0, 32)
    with pytest.raises(ValueError):
        dptq.qlinear_gated(a, a_s, 4, w, w_s, y=torch.empty((20, 64), dtype=torch.float16, device="cuda"))
    with pytest.raises(ValueError, match="activation"):
        dptq.qlinear_gated(a, a_s, 4, w, w_s, activation="relu")
    with pytest.raises(ValueError):
        dptq.qlinear_gated(a, a_s, 4, w[:40], w_s[:40])
    with pytest.raises(dptq.DptqError):
        dptq.qlinear_gated_decode_native(a, a_s, 4, dptq.prepack_weights(w, dptq.WEIGHTS_DECODE), w_s)
