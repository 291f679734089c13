"""The 8-bit paged cache and its attention where sizes and lengths end: lengths beyond any page table, and caches and
tables without pages."""

import numpy as np
import pytest

from oracle.serving import kv8_attention_ref
from test_gpu_kv8 import _cu, _d, _filled, _matches

torch = pytest.importorskip("torch")
dptq = pytest.importorskip("paper_2606_12487_amd")

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("new", [1, 100])
@pytest.mark.parametrize("window,sinks", [(0, 0), (2 ** 30 - 1, 130)])
def test_lengths_beyond_2_to_the_30_see_no_missing_page(new, window, sinks):
    # Every position of the table is visible; pages that are not there give nothing, page 0 least of all.
    rng = np.random.default_rng(31)
    H, Hkv, D = 4, 2, 128
    cache, ref, table = _filled(rng, [500], Hkv, D)
    table = np.repeat(table, 3, 0)
    table[0] = -1
    table[1, 1:3] = [2 ** 30, -5]
    lengths = np.array([2 ** 30 + 200, 2 ** 30 + 100, 2 ** 31 - 1], np.int32)
    q = rng.standard_normal((3 * new, H, D)).astype(np.float16)
    cu = _cu([new] * 3)
    want = kv8_attention_ref(q, cu, lengths, table, ref, 0.1, window, sinks)
    assert np.isneginf(want[1][:new]).all()
    for hints in ({}, dict(max_q=new, max_len=500)):
        _matches(dptq.kv8_attention(_d(q), _d(cu), _d(lengths), _d(table), cache, 0.1, window, sinks, **hints), want)


@pytest.mark.parametrize("counts", [[1, 1], [40, 3]])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_caches_and_tables_without_pages(counts, D):
    # Nothing is written and nothing is seen.
    T, H, Hkv = sum(counts), 4, 2
    q = torch.ones((T, H, D), dtype=torch.float16, device="cuda")
    k = torch.ones((T, Hkv, D), dtype=torch.float16, device="cuda")
    cu, n = _d(_cu(counts)), _d(np.array(counts, np.int32))
    for pages, width in ((0, 3), (2, 0), (0, 0)):
        cache = dptq.kv8_cache(pages, Hkv, D)
        table = torch.zeros((2, width), dtype=torch.int32, device="cuda")
        assert dptq.kv8_append(k, k, cu, n, table, cache) is cache
        out, lse = torch.full_like(q, 7), torch.full((T, H), 7.0, device="cuda")
        dptq.kv8_attention(q, cu, n, table, cache, out=out, lse=lse)
        assert bool((out == 0).all()) and bool(torch.isneginf(lse).all())
