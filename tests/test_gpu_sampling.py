"""Tokens drawn from rows of logits: equal to the definition's in 64 bits wherever the uniform number does not stand
within 2^-31 of a border between two tokens, and their probabilities to fp32's rounding."""

import numpy as np
import pytest

from oracle.sampling import sample_row_ref

torch = pytest.importorskip("torch")
dptq = pytest.importorskip("paper_2606_12487_amd")

pytestmark = pytest.mark.gpu

# Weights are off by 1.2e-10 < 2^-32.9 of themselves and by 2^-46 (2^-45 for 131072 logits) of the largest, which for
# 2^17 of them sums up to 2^-28 of it if all are off to one side, and to 2^-36.5 at random: a sum of weights, and with
# it a border, is within 2^-32.9 + 2^-36.5 of its place, and the total as well: 2^-31 covers both.
SLACK = 2.0 ** -31

ASKED = [dict(), dict(temperature=0.0), dict(top_k=1), dict(top_k=40), dict(top_p=0.9), dict(top_p=0.0),
         dict(min_p=0.05), dict(min_p=1.0), dict(min_p=2.0), dict(temperature=0.7, top_k=50, top_p=0.9),
         dict(temperature=1.3, top_k=1000, top_p=0.99, min_p=0.001), dict(top_p=0.5, min_p=0.3),
         dict(temperature=100.0, top_p=0.999), dict(temperature=0.05), dict(top_k=10 ** 9), dict(top_k=3000, top_p=0.7),
         dict(temperature=30.0, top_k=9000, min_p=0.9), dict(temperature=5.0, min_p=0.2)]


def _check(x, asked, u, what="", **kw):
    """x a numpy array [M, V]; asked: a dict for each row."""
    dev = torch.from_numpy(x).cuda() if isinstance(x, np.ndarray) else x
    host = dev.float().cpu().numpy()
    M = len(host)
    defaults = dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0)
    rows = {n: torch.tensor([{**defaults, **r}[n] for r in asked], device="cuda",
                            dtype=torch.int32 if n == "top_k" else torch.float32) for n in defaults}
    tokens, probs = dptq.sample_tokens(dev, torch.tensor(u, dtype=torch.float32, device="cuda"), **rows, **kw)
    assert tokens.dtype == torch.int64 and probs.dtype == torch.float32 and tokens.shape == probs.shape == (M,)
    again = dptq.sample_tokens(dev, torch.tensor(u, dtype=torch.float32, device="cuda"), **rows)
    assert torch.equal(tokens, again[0]) and torch.equal(probs, again[1])
    checked = 0
    for i in range(M):
        mine = {n: float(v[i]) if n != "top_k" else int(v[i]) for n, v in rows.items()}
        token, prob, slack = sample_row_ref(host[i], np.float32(u[i]), **mine)
        if slack < SLACK:
            continue
        checked += 1
        assert int(tokens[i]) == token, (what, i, mine, u[i], int(tokens[i]), token, slack)
        # A weight and a sum, 2^-32 each, and the rounding to fp32.
        assert abs(float(probs[i]) - prob) <= prob * (2.0 ** -24 + 2.0 ** -31) + 2.0 ** -149, (what, i, mine)
    assert checked >= 0.9 * M, what


def _logits(rng, M, V, half, kind="usual"):
    x = 3 * rng.standard_normal((M, V))
    if kind == "peaked":
        x[np.arange(M), rng.integers(0, V, M)] += 20
    elif kind == "flat":
        x *= 1e-3
    elif kind == "far":
        x = x * 300 + 5000
    elif kind == "ties":
        x = np.round(x)
    elif kind == "masked":
        x[:, rng.random(V) < 0.9] = -np.inf
        x[::3] = -np.inf
        x[::3, rng.integers(0, V)] = -3.0
    return x.astype(np.float16 if half else np.float32)


SIZES = [(1, 1), (3, 2), (5, 7), (18, 63), (18, 1000), (18, 2048), (18, 2049), (18, 4097), (36, 32000), (18, 100003),
         (300, 5000), (2, 131072)]


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("kind", ["usual", "peaked", "flat", "far", "ties", "masked"])
@pytest.mark.parametrize("M,V", SIZES)
def test_matches_the_definition(M, V, kind, half):
    rng = np.random.default_rng([M, V, half])
    x = _logits(rng, M, V, half, kind)
    shift = rng.integers(0, len(ASKED))
    _check(x, [ASKED[(i + shift) % len(ASKED)] for i in range(M)], rng.random(M).astype(np.float32), (M, V, kind))


@pytest.mark.parametrize("half", [False, True])
def test_equal_logits(half):
    """Every value the same: borders and tokens by index alone, below and above what is sorted at once."""
    for V in (5, 2048, 2049, 50000):
        x = np.full((6, V), -7.25, np.float16 if half else np.float32)
        u = np.array([0.0, 0.25, 0.5, 0.75, 0.999, 1 - 2.0 ** -24], np.float32)
        for asked in (dict(), dict(top_p=0.5), dict(top_k=V // 2 + 1), dict(min_p=1.0), dict(top_k=7, top_p=0.25)):
            tokens, probs = dptq.sample_tokens(torch.from_numpy(x).cuda(), torch.from_numpy(u).cuda(), **asked)
            n = V
            if "top_k" in asked:
                n = min(asked["top_k"], V)
            if "top_p" in asked:
                n = int(np.ceil(asked["top_p"] * n))
            # Sums are whole numbers here: exact.
            assert tokens.tolist() == [int(np.floor(float(v) * n)) for v in u], (V, asked)
            assert probs.tolist() == [float(np.float32(1 / n))] * 6


def test_ends_of_the_uniform_number():
    rng = np.random.default_rng(3)
    x = _logits(rng, 4, 3000, False)
    order = np.argsort(-x, axis=1, kind="stable")
    tokens, _ = dptq.sample_tokens(torch.from_numpy(x).cuda(), torch.zeros(4, device="cuda"))
    assert tokens.tolist() == order[:, 0].tolist()
    tokens, _ = dptq.sample_tokens(torch.from_numpy(x).cuda(), torch.ones(4, device="cuda"), top_k=10)
    assert tokens.tolist() == order[:, 9].tolist()           # 1 is beyond all: the last one kept
    tokens, probs = dptq.sample_tokens(torch.from_numpy(x).cuda(), torch.rand(4, device="cuda"), temperature=0)
    assert tokens.tolist() == order[:, 0].tolist() and probs.tolist() == [1.0] * 4


@pytest.mark.parametrize("half", [False, True])
def test_rows_without_anything(half):
    x = torch.full((5, 70000), -torch.inf, dtype=torch.float16 if half else torch.float32, device="cuda")
    x[1, 69999] = -60000.0
    x[3, 5] = torch.nan
    tokens, probs = dptq.sample_tokens(x, torch.full((5,), 0.7, device="cuda"), top_p=0.9)
    assert tokens.tolist()[:3] == [-1, 69999, -1] and tokens.tolist()[4] == -1
    assert probs.tolist()[:3] == [0.0, 1.0, 0.0] and -1 <= int(tokens[3]) < 70000


def test_odd_values_stay_in_range():
    """+inf, NaN and parameters out of range: any token of the row, and no harm to its neighbours."""
    rng = np.random.default_rng(4)
    x = _logits(rng, 12, 9001, False)
    x[1, 77] = x[1, 78] = np.inf
    x[3, ::2] = np.nan
    x[5] = np.nan
    x[7] = np.inf
    asked = [dict()] * 12
    asked[9] = dict(temperature=np.inf)
    asked[11] = dict(temperature=np.nan, top_p=np.nan, min_p=np.nan, top_k=-5)
    u = rng.random(12).astype(np.float32)
    u[8], u[10] = np.nan, -3.0
    d = dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0)
    rows = {n: torch.tensor([{**d, **r}[n] for r in asked], device="cuda",
                            dtype=torch.int32 if n == "top_k" else torch.float32) for n in d}
    for extra in (dict(), dict(top_p=0.9), dict(min_p=0.1), dict(top_k=2500), dict(top_k=2500, top_p=0.8, min_p=0.5)):
        tokens, _ = dptq.sample_tokens(torch.from_numpy(x).cuda(), torch.from_numpy(u).cuda(), **{**rows, **extra})
        assert all(-1 <= t < 9001 for t in tokens.tolist())
        for i in (0, 2, 4, 6):
            mine = {**d, **extra}
            token, _, slack = sample_row_ref(x[i], u[i], mine["temperature"], mine["top_k"],
                                             float(np.float32(mine["top_p"])), float(np.float32(mine["min_p"])))
            assert slack < SLACK or int(tokens[i]) == token


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("first,V,ld", [(1, 5001, 5003), (3, 40000, 40011), (0, 777, 777), (5, 100, 4096)])
def test_rows_of_a_wider_matrix(first, V, ld, half):
    rng = np.random.default_rng(V)
    wide = torch.from_numpy(_logits(rng, 7, ld, half)).cuda()
    x = wide[:, first:first + V] if first + V <= ld else wide[:, :V]
    u = rng.random(7).astype(np.float32)
    _check(x, [ASKED[i * 2 % len(ASKED)] for i in range(7)], u, (first, V, ld))


def test_numbers_for_all_rows_and_given_outputs():
    rng = np.random.default_rng(9)
    x = torch.from_numpy(_logits(rng, 9, 20000, True)).cuda()
    u = torch.rand(9, device="cuda")
    rows = dict(temperature=torch.full((9,), 0.8, device="cuda"), top_p=torch.full((9,), 0.9, device="cuda"),
                top_k=torch.full((9,), 300, dtype=torch.int32, device="cuda"), min_p=torch.full((9,), 0.01, device="cuda"))
    tokens = torch.empty(9, dtype=torch.int64, device="cuda")
    probs = torch.empty(9, device="cuda")
    got = dptq.sample_tokens(x, u, temperature=0.8, top_k=300, top_p=0.9, min_p=0.01, tokens=tokens, probs=probs)
    assert got[0] is tokens and got[1] is probs
    want = dptq.sample_tokens(x, u, **rows)
    assert torch.equal(tokens, want[0]) and torch.equal(probs, want[1])
    assert dptq.sample_tokens(x[:0], u[:0])[0].shape == (0,)
    for bad in (dict(temperature=-1.0), dict(top_k=-1), dict(top_p=-0.5), dict(min_p=float("nan")),
                dict(top_k=rows["top_p"]), dict(temperature=rows["top_k"]), dict(top_p=rows["top_p"][:5])):
        with pytest.raises((ValueError, TypeError)):
            dptq.sample_tokens(x, u, **bad)


def test_frequencies_of_drawn_tokens():
    """Many uniform numbers over one distribution: counts are n p +- 1 a border, since numbers are evenly spaced."""
    x = torch.tensor([[0.0, 2.0, -1.0, 1.0, 1.0]], device="cuda")
    n = 4096
    u = (torch.arange(n, device="cuda") + 0.5) / n
    tokens, _ = dptq.sample_tokens(x.expand(n, 5).contiguous(), u.float())
    p = torch.softmax(x[0].double(), 0).tolist()
    for t, count in enumerate(torch.bincount(tokens, minlength=5).tolist()):
        assert abs(count - n * p[t]) <= 2


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("V", [50304, 131072])
def test_top_p_of_long_rows(V, half):
    """Top-p alone, whose border and the token's are in bins of hundreds of tokens, far apart and next to each other."""
    rng = np.random.default_rng([V, half])
    u = np.repeat(np.float32([0.01, 0.3, 0.6, 0.9, 0.97, 0.999]), 5)
    x = np.concatenate([_logits(rng, len(u) // 2, V, half, "usual"),
                        (2 * rng.standard_normal((len(u) - len(u) // 2, V))).astype(np.float16 if half else np.float32)])
    _check(x, [dict(top_p=p, temperature=t) for p, t in ((0.5, 1.0), (0.8, 0.7), (0.9, 1.0), (0.95, 1.5), (0.99, 0.5))] * 6,
           u, V)


def test_more_rows_than_a_launch_holds():
    M = (2 ** 32 - 1) // 1024 + 5
    x = torch.zeros((M, 2), dtype=torch.float16, device="cuda")
    x[-7:, 1] = torch.tensor([3.0, -3.0, 3.0, -3.0, 3.0, 3.0, -3.0], device="cuda").half()
    tokens, probs = dptq.sample_tokens(x, torch.zeros(M, device="cuda"), top_k=1)
    assert tokens[-7:].tolist() == [1, 0, 1, 0, 1, 1, 0] and int(tokens[:-7].sum()) == 0
    assert bool((probs == 1).all())
