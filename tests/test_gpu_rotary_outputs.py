"""Outputs of rotary positions in the matrix of their inputs: beside them, behind them, and over them, which is refused
where they are not the same rows."""

import numpy as np
import pytest

from test_gpu_kv8 import _cache, _cu, _d, _garbage, _rows, _table

torch = pytest.importorskip("torch")
dptq = pytest.importorskip("paper_2606_12487_amd")

pytestmark = pytest.mark.gpu

H, HKV, D = 4, 2, 64


@pytest.mark.parametrize("T", [1, 2, 77])
def test_beside_and_behind_the_inputs(T):
    rng = np.random.default_rng(T)
    x, positions = _d(_rows(rng, 2 * T, 2 * (H + HKV), D)), _d(rng.integers(0, 4000, T).astype(np.int32))
    f, before = dptq.rotary_inv_freq(D), x.clone()
    q, k = x[:T, :H], x[:T, H:H + HKV]
    want = dptq.rotary(q, k, positions, f)
    for q_out, k_out in ((x[:T, H + HKV:2 * H + HKV], x[:T, 2 * H + HKV:]), (x[T:, :H], x[T:, H:H + HKV]),
                         (x[T:, H + HKV:2 * H + HKV], x[:T, 2 * H + HKV:]), (q, x[T:, :HKV]), (q, k)):
        x.copy_(before)
        dptq.rotary(q, k, positions, f, q_out=q_out, k_out=k_out)
        assert torch.equal(q_out, want[0]) and torch.equal(k_out, want[1])


@pytest.mark.parametrize("T", [1, 77])
def test_over_the_inputs(T):
    rng = np.random.default_rng(T)
    x, positions = _d(_rows(rng, T, H + 2 * HKV, D)), _d(rng.integers(0, 4000, T).astype(np.int32))
    f, before = dptq.rotary_inv_freq(D), x.clone()
    q, k, v = x.split([H, HKV, HKV], dim=1)
    for q_out, k_out in ((x[:, 1:1 + H], None), (x[:, HKV:HKV + H], k), (None, x[:, 1:1 + HKV]), (q, x[:, :HKV]),
                         (x.view(-1)[8:8 + T * H * D].view(T, H, D), None)):
        with pytest.raises(dptq.DptqError):
            dptq.rotary(q, k, positions, f, q_out=q_out, k_out=k_out)
    lengths, P = [T], 3
    cache, table = _cache(_garbage(rng, P, HKV, D)), _table(rng, lengths, P)
    args = _d(_cu([T])), _d(np.array(lengths, np.int32)), _d(table), cache, f
    for q_out in (x[:, HKV:HKV + H], x[:, 1:1 + H], x[:, 2 * HKV:]):
        with pytest.raises(dptq.DptqError):
            dptq.rotary_kv8_append(q, k, v, *args, q_out=q_out)
    assert torch.equal(x, before)
    want, _ = dptq.rotary(q, None, torch.arange(T, dtype=torch.int32, device="cuda"), f)
    dptq.rotary_kv8_append(q, k, v, *args, q_out=q)
    assert torch.equal(q, want) and torch.equal(x[:, H:], before[:, H:])
