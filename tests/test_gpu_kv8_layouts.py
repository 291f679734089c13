"""Attention over the 8-bit cache in each of the ways that a call is laid out: prompts in tiles of 128 rows, decode
with several pages a wave, and the join of hundreds of parts.  A few heads of each call are checked."""

import numpy as np
import pytest

from oracle.serving import PAGE, kv8_attention_ref
from test_gpu_kv8 import _append, _cache, _cu, _d, _garbage, _host, _matches, _pages, _rows, _table

torch = pytest.importorskip("torch")
dptq = pytest.importorskip("paper_2606_12487_amd")

pytestmark = pytest.mark.gpu


def _cus():
    return torch.cuda.get_device_properties(0).multi_processor_count


def _sequences(rng, lengths, Hkv, D, spread):
    """A cache and its table: V of neighbouring pages up to 10^spread apart, and NaN past each sequence's end."""
    k, v = _rows(rng, sum(lengths), Hkv, D), _rows(rng, sum(lengths), Hkv, D).astype(np.float64)
    at = 0
    for n in lengths:
        for first in range(0, n, PAGE):
            v[at + first:at + min(first + PAGE, n)] *= 10.0 ** (rng.integers(0, spread + 1) - spread // 2 - 1)
        at += n
    v = np.clip(v, -60000, 60000).astype(np.float16)
    P = _pages(lengths)
    table = _table(rng, lengths, P)
    cache = _append(_cache(_garbage(rng, P, Hkv, D)), k, v, _cu(lengths), lengths, table)
    for b, n in enumerate(lengths):
        if n % PAGE:
            last = int(table[b, n // PAGE])
            cache[0].view(torch.uint8)[last, :, n % PAGE:] = 0x7F
            cache[1].view(torch.uint8)[last, :, :, n % PAGE:] = 0xFF
    return cache, table


def _check(args, hints, arrays, q, cu, lengths, table, heads, Hkv, window, sinks):
    """The call against the definition, on the key heads `heads`."""
    out, lse = dptq.kv8_attention(*args, window=window, sinks=sinks, **hints)
    group = q.shape[1] // Hkv
    mine = [h * group + g for h in heads for g in range(group)]
    want = kv8_attention_ref(q[:, mine], cu, lengths, table, [a[:, heads] for a in arrays], q.shape[2] ** -0.5, window,
                             sinks)
    _matches((out[:, mine], lse[:, mine]), want)


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 4), (70, 130)])
def test_prompts_in_tiles_of_128_rows(D, window, sinks):
    rng = np.random.default_rng(D + window)
    Hkv, group = 32, 4
    before, new = [200, 0, 77, 311], [130, 33, 125, 1]
    lengths = [a + b for a, b in zip(before, new)]
    cache, table = _sequences(rng, lengths, Hkv, D, 6)
    table[0, 2], table[3, 0] = -1, 10 ** 6                # pages that are not there
    q = (1.5 * rng.standard_normal((sum(new), Hkv * group, D))).astype(np.float16)
    cu, arrays = _cu(new), _host(cache)
    args = (_d(q), _d(cu), _d(np.array(lengths, np.int32)), _d(table), cache)
    # With max_q 100 a workgroup has more tiles than one; 128 rows where there are two tiles a compute unit.
    for hints in ({}, dict(max_q=130, max_len=400), dict(max_q=100)):
        assert -(-hints.get("max_q", sum(new)) * group // 128) * Hkv * len(new) >= 2 * _cus()
        _check(args, hints, arrays, q, cu, lengths, table, [0, 19], Hkv, window, sinks)


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("window,sinks", [(0, 0), (700, 130)])
def test_decode_with_several_pages_a_wave(D, window, sinks):
    # As many sequences and heads as give one part each: up to 24 pages, six of a wave.
    rng = np.random.default_rng(D + window + 1)
    Hkv, group, B = 32, 2, 32
    lengths = [1500, 64, 1, 1473] + [int(n) for n in rng.integers(1, 1500, B - 4)]
    cache, table = _sequences(rng, lengths, Hkv, D, 6)
    table[3, 5], table[5, 0] = -1, -1
    q = (1.5 * rng.standard_normal((B, Hkv * group, D))).astype(np.float16)
    cu, arrays = _cu([1] * B), _host(cache)
    assert B * Hkv >= 256 // D * _cus()
    args = (_d(q), _d(cu), _d(np.array(lengths, np.int32)), _d(table), cache)
    _check(args, dict(max_q=1, max_len=1500), arrays, q, cu, lengths, table, [3, 30], Hkv, window, sinks)


@pytest.mark.parametrize("lengths,width", [([70400, 100], 1101), ([70400], 2200)])
def test_decode_in_hundreds_of_parts(lengths, width):
    # 276 parts of four pages, a short sequence beside a long one; then parts of five, as 512 of four do not reach.
    rng = np.random.default_rng(width)
    Hkv, group, D, B = 1, 4, 64, len(lengths)
    cache, table = _sequences(rng, lengths, Hkv, D, 2)
    wide = np.full((B, width), -1, np.int32)
    wide[:, :table.shape[1]] = table[:, :width]
    q = rng.standard_normal((B, Hkv * group, D)).astype(np.float16)
    cu, arrays = _cu([1] * B), _host(cache)
    args = (_d(q), _d(cu), _d(np.array(lengths, np.int32)), _d(wide), cache)
    _check(args, dict(max_q=1), arrays, q, cu, lengths, wide, [0], Hkv, 0, 0)


@pytest.mark.parametrize("D", [64, 128, 256])
def test_prompts_in_a_graph(D):
    # Replays give what the eager call gives on the same buffers, with eager work between them.
    rng = np.random.default_rng(D + 7)
    Hkv, group = 2, 4
    lengths, new = [300, 90], [100, 37]
    cache, table = _sequences(rng, lengths, Hkv, D, 2)
    q = torch.zeros((sum(new), Hkv * group, D), dtype=torch.float16, device="cuda")
    n, cu, tab = _d(np.array(lengths, np.int32)), _d(_cu(new)), _d(table)
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        dptq.kv8_attention(q, cu, n, tab, cache, window=150, sinks=3, max_q=100, out=out, lse=lse)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dptq.kv8_attention(q, cu, n, tab, cache, window=150, sinks=3, max_q=100, out=out, lse=lse)
    for i in range(4):
        q.copy_(_d(rng.standard_normal(tuple(q.shape)).astype(np.float16)))
        n.copy_(_d(np.array([300 - 60 * i, 90 - 11 * i], np.int32)))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), lse.clone()
        want = dptq.kv8_attention(q, cu, n, tab, cache, window=150, sinks=3, max_q=100)
        assert torch.equal(got[0].view(torch.int16), want[0].view(torch.int16))
        assert torch.equal(got[1].view(torch.int32), want[1].view(torch.int32))
