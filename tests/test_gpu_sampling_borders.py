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
    return dict(temperature=t, top_k=(at + len(x)) // 2, top_p=float(np.float32((sums[at] - w[at] / 2) /
                                                                              sums[(at + len(x)) // 2 - 1]))), u


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
    kinds = ["token", "top_k", "top_p", "top_k and top_p"] + ([] if half else ["min_p"])
    rows, asked, u = [], [], []
    for kind in kinds:
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
