"""Drawn tokens where the borders lie in crowded bins of the value: around zero, beside zeros of both signs."""

import numpy as np
import pytest

from test_gpu_sampling import _check

torch = pytest.importorskip("torch")
dptq = pytest.importorskip("paper_2606_12487_amd")

pytestmark = pytest.mark.gpu

NEAR = 2.0 ** -6    # values of a smaller magnitude are in the two bins at zero


def _asked(x, kind, at, t, rng):
    """What puts the border of `kind` behind the token at place `at` of the row's order, and a uniform number."""
    order = np.sort(x.astype(np.float64))[::-1]
    w = np.exp((order - order[0]) / t)
    sums = np.cumsum(w)
    middle = np.float32((sums[at] - w[at] / 2) / sums[-1])       # in the middle of the token
    u = np.float32(rng.random())
    if kind == "token":
        return dict(temperature=t), middle
    if kind == "top_k":
        return dict(temperature=t, top_k=at + 1), u
    if kind == "top_p":
        return dict(temperature=t, top_p=float(middle)), u
    if kind == "min_p":
        return dict(temperature=t, min_p=float(w[at] * (1 - 3e-7))), u
    k = (at + len(x)) // 2
    return dict(temperature=t, top_k=k, top_p=float(np.float32((sums[at] - w[at] / 2) / sums[k - 1]))), u


def _around_zero(rng, V, zeros, near, half):
    """Zeros of both signs, `near` values in each of the bins at zero, and others on both sides of these."""
    rest = V - zeros - 2 * near
    above = rest // 3
    x = np.concatenate([np.where(rng.random(zeros) < 0.5, -0.0, 0.0), NEAR * 0.99 * rng.random(near),
                        -NEAR * 0.99 * rng.random(near), 0.02 + 2 * rng.random(above), -0.02 - 3 * rng.random(rest - above)])
    x = x.astype(np.float16 if half else np.float32)
    return x[rng.permutation(V)]


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("zeros", [1, 50, 100, 3000])
@pytest.mark.parametrize("near", [60, 1500])
@pytest.mark.parametrize("V", [7000, 40000])
def test_borders_beside_zeros(V, near, zeros, half):
    rng = np.random.default_rng([V, near, zeros, half])
    rows, asked, u = [], [], []
    for kind in ("token", "top_k", "top_p", "top_k and top_p", "min_p"):
        x = _around_zero(rng, V, zeros, near, half)
        first = int((x > 0).sum())         # of the zeros
        # In the bin below zero, at its first and its last token, among the zeros, in the bin above.
        for at in (first + zeros, first + zeros + near - 1, first + zeros + int(rng.integers(near)),
                   first + zeros + int(rng.integers(near)), first + int(rng.integers(zeros)), first - 1 - int(rng.integers(near))):
            a, v = _asked(x, kind, at, float(np.float32(rng.choice([0.5, 1.0, 2.0]))), rng)
            rows.append(x)
            asked.append(a)
            u.append(v)
    _check(np.stack(rows), asked, np.array(u, np.float32), (V, near, zeros))


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("V", [5000, 30000])
def test_largest_logits_are_zeros(V, half):
    """Zeros alone pass a min-p of 1, at any temperature; 0 and -0 are equal, drawn by index."""
    rng = np.random.default_rng(V)
    x = -0.001 - rng.random((4, V))
    places = np.sort(np.stack([rng.permutation(V)[:3000] for _ in range(4)]), axis=1)
    np.put_along_axis(x, places, np.where(rng.random((4, 3000)) < 0.5, -0.0, 0.0), axis=1)
    x = torch.from_numpy(x.astype(np.float16 if half else np.float32)).cuda()
    u = np.array([0.0, 0.3, 0.7, 1 - 2.0 ** -24], np.float32)
    for t in (1.0, 2e-38):
        tokens, probs = dptq.sample_tokens(x, torch.from_numpy(u).cuda(), temperature=t, min_p=1.0)
        # Sums are whole numbers here: exact.
        assert tokens.tolist() == [int(places[i][int(np.floor(float(u[i]) * 3000))]) for i in range(4)], t
        assert probs.tolist() == [float(np.float32(1 / 3000))] * 4


@pytest.mark.parametrize("half", [True, False])
@pytest.mark.parametrize("mean,deviation,t", [(6, 0.7, 1.0), (10, 0.7, 1.0), (12, 1.0, 1.0), (20, 2.0, 3.0), (-9, 1.0, 0.8)])
def test_min_p_in_a_crowded_bin(mean, deviation, t, half):
    """Logits far from zero, whose bins of a 1/32 octave hold thousands: the bin of min-p's smallest weight is cut, in
    fp16 mostly into stretches between two numbers."""
    rng = np.random.default_rng([mean + 100, half])
    M = 24
    x = (mean + deviation * rng.standard_normal((M, 131072))).astype(np.float16 if half else np.float32)
    shares = np.exp(-deviation * rng.uniform(1.0, 4.5, M) / t)
    asked = [dict(temperature=t, min_p=float(p)) for p in shares]
    for i in range(0, M, 4):
        asked[i].update(top_p=0.9)
        asked[i + 1].update(top_k=5000)
    _check(x, asked, rng.random(M).astype(np.float32), (mean, deviation))


@pytest.mark.parametrize("half", [True, False])
def test_min_p_where_no_token_is(half):
    """Between two clusters, in an empty bin and in an empty part of a crowded one; and behind the last token."""
    rng = np.random.default_rng(7)
    x = np.concatenate([8 + 0.004 * rng.integers(0, 8, (8, 3000)), 7.9 - 0.04 * rng.random((8, 4000)),
                        5 + 0.5 * rng.random((8, 1000))], axis=1)
    x = np.stack([row[rng.permutation(8000)] for row in x]).astype(np.float16 if half else np.float32)
    top = x.max(axis=1).astype(np.float64)
    at = np.array([6.5, 7.0, 7.95, 7.915, 7.905, 4.0, 5.6, 7.88])
    asked = [dict(min_p=float(np.exp(a - m))) for a, m in zip(at, top)]
    _check(x, asked, rng.random(8).astype(np.float32))
    for a in asked:
        a["top_p"] = 0.999
    _check(x, asked, rng.random(8).astype(np.float32))
