"""Rotary positions: against the definition in 64 bits, in each layout of rows, and with the cache's append in one
launch, bit for bit what the two calls give."""

import numpy as np
import pytest

from oracle.rotary import rotary_ref
from oracle.serving import kv8_append_ref
from test_gpu_kv8 import APPENDS, _cache, _cu, _d, _garbage, _pages, _rows, _same, _table

torch = pytest.importorskip("torch")
dptq = pytest.importorskip("paper_2606_12487_amd")

pytestmark = pytest.mark.gpu


def _close(got, x, positions, f, interleaved, scale, what=""):
    """The rounding to fp16 (half a step: 2^-11 of the value, 2^-25 below its normal range), and of fp32: the angle
    within the quarter turn, the series, scale, and two products, under eight roundings of 2^-24 of |x1| + |x2|, twice
    that allowed.  Angles in 64 bits: three roundings of 2^-53."""
    want, size = rotary_ref(x, positions, f, interleaved, scale)
    angle = np.abs(np.asarray(positions, np.float64)).max(initial=0) * f.max()
    tolerance = 2.0 ** -11 * np.abs(want) + 2.0 ** -25 + size * (2.0 ** -20 + angle * 2.0 ** -50)
    got = got.cpu().numpy().astype(np.float64)
    wrong = ~(np.abs(got - want) <= tolerance)
    turned = 2 * len(f)
    assert not wrong.any(), (what, np.argwhere(wrong)[:3], got[wrong][:3], want[wrong][:3])
    assert np.array_equal(got[..., turned:], want[..., turned:]), what


SHAPES = [
    # (tokens, heads, kv_heads, head_dim, rotary_dim)
    (1, 1, 1, 8, 2), (1, 32, 8, 128, 128), (3, 5, 2, 64, 64), (17, 8, 1, 80, 80), (2, 3, 3, 96, 48), (5, 7, 2, 256, 64),
    (9, 2, 1, 512, 512), (4, 6, 0, 128, 34), (33, 4, 4, 40, 22), (7, 3, 1, 8, 8), (6, 1, 1, 16, 16), (1, 71, 2, 24, 16),
    (300, 64, 8, 128, 128), (301, 40, 8, 128, 32), (299, 32, 32, 112, 56), (1300, 33, 7, 72, 70),
]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T,H,Hkv,D,r", SHAPES)
def test_matches_the_definition(T, H, Hkv, D, r, interleaved):
    rng = np.random.default_rng(T + H + D + r)
    q, k = _rows(rng, T, H, D), _rows(rng, T, Hkv, D) if Hkv else None
    positions = rng.integers(0, 1 << 20, T).astype(np.int32)
    f = dptq.rotary_inv_freq(r)
    scale = 1.0 if T % 2 else 1.25
    got_q, got_k = dptq.rotary(_d(q), None if k is None else _d(k), _d(positions), f, interleaved, scale)
    _close(got_q, q, positions, f.cpu().numpy(), interleaved, scale, "q")
    if k is None:
        assert got_k is None
    else:
        _close(got_k, k, positions, f.cpu().numpy(), interleaved, scale, "k")


def test_any_position():
    rng = np.random.default_rng(1)
    positions = np.array([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 2 ** 24 + 1, -777777], np.int32)
    f = np.array([1.0, np.pi / 2, np.pi, 0.25, 1e-4, 0.0, -0.3, 3.0])
    x = _rows(rng, len(positions), 2, 16)
    for interleaved in (False, True):
        got, _ = dptq.rotary(_d(x), None, _d(positions), _d(f), interleaved, -2.0)
        _close(got, x, positions, f, interleaved, -2.0)
    got, _ = dptq.rotary(_d(x[:1]), None, _d(positions[:1]), _d(f))
    assert torch.equal(got, _d(x[:1]))                       # position 0 turns nothing


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,r", [(128, 128), (64, 32), (96, 22), (16, 8)])
def test_rows_of_a_wider_matrix_in_and_out_of_place(D, r, interleaved):
    rng = np.random.default_rng(D + r)
    T, H, Hkv = 37, 6, 2
    x = _rows(rng, T, H + 2 * Hkv, D)
    positions, f = rng.integers(0, 5000, T).astype(np.int32), dptq.rotary_inv_freq(r)
    rows = _d(x)
    q, k, v = rows.split([H, Hkv, Hkv], dim=1)
    out_q, out_k = dptq.rotary(q, k, _d(positions), f, interleaved)
    _close(out_q, x[:, :H], positions, f.cpu().numpy(), interleaved, 1.0)
    _close(out_k, x[:, H:H + Hkv], positions, f.cpu().numpy(), interleaved, 1.0)
    assert torch.equal(rows, _d(x))
    wide = torch.full((T, H + 5, D), 9.0, dtype=torch.float16, device="cuda")
    got = dptq.rotary(q, k, _d(positions), f, interleaved, q_out=wide[:, 1:1 + H], k_out=wide[:, 2 + H:2 + H + Hkv])
    assert torch.equal(got[0], out_q) and torch.equal(got[1], out_k) and got[0].data_ptr() == wide[:, 1:].data_ptr()
    assert bool((wide[:, 0] == 9).all() and (wide[:, 1 + H] == 9).all() and (wide[:, 2 + H + Hkv:] == 9).all())
    dptq.rotary(q, k, _d(positions), f, interleaved, q_out=q, k_out=k)      # in place
    assert torch.equal(rows[:, :H], out_q) and torch.equal(rows[:, H:H + Hkv], out_k)
    assert torch.equal(rows[:, H + Hkv:], _d(x)[:, H + Hkv:])


def test_nothing_to_do():
    f = dptq.rotary_inv_freq(16)
    x = torch.empty((0, 4, 16), dtype=torch.float16, device="cuda")
    q, k = dptq.rotary(x, x[:, :2].contiguous(), torch.empty(0, dtype=torch.int32, device="cuda"), f)
    assert q.shape == (0, 4, 16) and k.shape == (0, 2, 16)


@pytest.mark.parametrize("before,new,Hkv,D", APPENDS)
@pytest.mark.parametrize("interleaved", [False, True])
def test_append_in_one_launch(before, new, Hkv, D, interleaved):
    rng = np.random.default_rng(sum(new) + D)
    lengths = [a + b for a, b in zip(before, new)]
    P = _pages(lengths)
    arrays, table = _garbage(rng, P, Hkv, D), _table(rng, lengths, P)
    for x in arrays[2:]:
        x[~np.isfinite(x) | (x == 0)] = 1.0      # pages that hold tokens have scales
    T, H = sum(new), 3 * Hkv
    rows = _rows(rng, T, H + 2 * Hkv, D)
    cu, n = _cu(new), np.array(lengths, np.int32)
    positions = np.concatenate([np.arange(a, b) for a, b in zip(before, lengths)]).astype(np.int32)
    for r in (D, D // 2, 22):
        f = dptq.rotary_inv_freq(r, factor=4.0, original_length=2048)
        q, k, v = _d(rows).split([H, Hkv, Hkv], dim=1)
        for hint in (None, max(new), 1):
            cache = _cache(arrays)
            got = dptq.rotary_kv8_append(q, k, v, _d(cu), _d(n), _d(table), cache, f, interleaved, 1.1, max_new=hint)
            want_q, want_k = dptq.rotary(q, k, _d(positions), f, interleaved, 1.1)
            assert torch.equal(got, want_q)
            _close(got, rows[:, :H], positions, f.cpu().numpy(), interleaved, 1.1)
            want = kv8_append_ref(want_k.cpu().numpy(), rows[:, H + Hkv:], cu, lengths, table, arrays)
            _same(cache, want)
    same = q.clone()
    dptq.rotary_kv8_append(same, k, v, _d(cu), _d(n), _d(table), _cache(arrays), f, interleaved, 1.1, q_out=same)
    assert torch.equal(same, want_q)


def test_append_odd_batches():
    """Rows of no sequence, a sequence without new tokens, pages that are not there, lengths below the new tokens."""
    rng = np.random.default_rng(5)
    Hkv, H, D = 2, 6, 128
    cu, n = np.array([0, 3, 3, 73, 80], np.int32), np.array([70, 5, 70, 4], np.int32)
    table = np.array([[0, 1], [2, -1], [3, 10 ** 6], [5, 4]], np.int32)
    rows = _rows(rng, 90, H + 2 * Hkv, D)
    arrays = _garbage(rng, 6, Hkv, D)
    for x in arrays[2:]:
        x[:] = 2.0 ** -3
    f = dptq.rotary_inv_freq(D)
    q, k, v = _d(rows).split([H, Hkv, Hkv], dim=1)
    start = np.array([67, 0, 0, -3])
    positions = np.concatenate([start[b] + np.arange(cu[b + 1] - cu[b]) for b in range(4)]).astype(np.int32)
    cache, apart = _cache(arrays), _cache(arrays)
    out = torch.full((90, H, D), 9.0, dtype=torch.float16, device="cuda")
    dptq.rotary_kv8_append(q, k, v, _d(cu), _d(n), _d(table), cache, f, q_out=out)
    want_q, want_k = dptq.rotary(q[:80], k[:80], _d(positions), f)
    assert torch.equal(out[:80], want_q) and bool((out[80:] == 9).all())
    whole = torch.cat((want_k, k[80:]))
    dptq.kv8_append(whole, v, _d(cu), _d(n), _d(table), apart)
    for a, b in zip(cache, apart):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    # Without pages, in the cache or in the table, the queries turn all the same.
    none = dptq.kv8_cache(0, Hkv, D)
    for cache, t in ((none, _d(table)), (_cache(arrays), _d(table[:, :0]))):
        out.fill_(9.0)
        dptq.rotary_kv8_append(q, k, v, _d(cu), _d(n), t, cache, f, q_out=out)
        assert torch.equal(out[:80], want_q) and bool((out[80:] == 9).all())


@pytest.mark.parametrize("new,interleaved", [((850,), True), ((600, 0, 660), True), ((600, 1, 660), False)])
def test_append_of_many_query_heads(new, interleaved):
    """More than 64 angles a token, which a wave turns several parts of the heads by."""
    rng = np.random.default_rng(sum(new))
    H, Hkv, D = 64, 1, 256
    T, P = sum(new), _pages(new)
    arrays, table = _garbage(rng, P, Hkv, D), _table(rng, list(new), P)
    rows = torch.randn((T, H + 2 * Hkv, D), device="cuda", generator=torch.Generator("cuda").manual_seed(T)).half()
    q, k, v = rows.split([H, Hkv, Hkv], dim=1)
    n, positions = _d(np.array(new, np.int32)), _d(np.concatenate([np.arange(b) for b in new]).astype(np.int32))
    for r in (D, 200):
        f = dptq.rotary_inv_freq(r)
        one, two = _cache(arrays), _cache(arrays)
        got = dptq.rotary_kv8_append(q, k, v, _d(_cu(new)), n, _d(table), one, f, interleaved)
        want_q, want_k = dptq.rotary(q, k, positions, f, interleaved)
        assert torch.equal(got, want_q)
        dptq.kv8_append(want_k, v, _d(_cu(new)), n, _d(table), two)
        for a, b in zip(one, two):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


@pytest.mark.parametrize("D", [64, 128, 256])
def test_append_in_pieces_of_growing_size(D):
    """Pages filled by calls of 1 to 70 tokens whose values grow now and then, so that older codes are scaled again from
    every slot on."""
    rng = np.random.default_rng(D)
    B, H, Hkv, P = 2, 4, 2, 12
    one, two = dptq.kv8_cache(P, Hkv, D), dptq.kv8_cache(P, Hkv, D)
    for pages in (*one[:2], *two[:2]):
        pages.view(torch.uint8).fill_(0x7F)      # a new cache's pages hold anything
    table = _d(np.arange(P, dtype=np.int32)[rng.permutation(P)].reshape(B, P // B))
    f = dptq.rotary_inv_freq(D // 2)
    size, start = 2.0 ** -9, np.zeros(B, np.int64)
    for step, new in enumerate([(1, 5), (1, 1), (3, 0), (6, 2), (8, 1), (1, 9), (20, 16), (24, 31), (1, 64), (70, 1), (5, 3),
                                (1, 1), (17, 70), (40, 8)]):
        size *= (1.0, 1.5, 16.0, 0.25)[step % 4]
        cu, start = _cu(new), start + np.array(new)
        rows = (size * torch.randn((sum(new), H + 2 * Hkv, D), device="cuda",
                                   generator=torch.Generator("cuda").manual_seed(step))).half()
        q, k, v = rows.split([H, Hkv, Hkv], dim=1)
        n = _d(start.astype(np.int32))
        positions = _d(np.concatenate([np.arange(e - c, e) for e, c in zip(start, new)]).astype(np.int32))
        got = dptq.rotary_kv8_append(q, k, v, _d(cu), n, table, one, f, max_new=max(new))
        want_q, want_k = dptq.rotary(q, k, positions, f)
        dptq.kv8_append(want_k, v, _d(cu), n, table, two, max_new=max(new))
        assert torch.equal(got, want_q)
        for a, b, what in zip(one, two, ("K", "V", "K's scales", "V's scales")):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), (step, what)
