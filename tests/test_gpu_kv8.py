"""GPU parity of the 8-bit paged KV cache: appends bit for bit, attention within the rounding that its formula admits."""

import numpy as np
import pytest

from oracle.serving import PAGE, e4m3_values, kv8_append_ref, kv8_attention_ref

torch = pytest.importorskip("torch")
dptq = pytest.importorskip("paper_2606_12487_amd")

pytestmark = pytest.mark.gpu


def _d(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _cache(arrays):
    k, v, ks, vs = (_d(a) for a in arrays)
    return dptq.KV8Cache(k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn), ks, vs)


def _host(cache):
    return [cache[0].view(torch.uint8).cpu().numpy(), cache[1].view(torch.uint8).cpu().numpy(),
            cache[2].cpu().numpy(), cache[3].cpu().numpy()]


def _rows(rng, T, H, D):
    x = rng.standard_normal((T, H, D)) * rng.uniform(0.2, 2.0, (H, D))
    x[:, :, rng.integers(0, D)] *= 8
    return (x * rng.choice([1.0, 1.0, 1.0, 4.0], (T, 1, 1))).astype(np.float16)


def _garbage(rng, P, H, D):
    """A cache of freed pages: any bytes, NaN codes among them, and any scales."""
    return [rng.integers(0, 256, (P, H, PAGE, D)).astype(np.uint8), rng.integers(0, 256, (P, H, D, PAGE)).astype(np.uint8),
            rng.choice([np.nan, 0, 3, 1e30], (P, H)).astype(np.float32),
            rng.choice([np.nan, 0, 3, 1e30], (P, H)).astype(np.float32)]


def _table(rng, lengths, P, extra=1):
    width = max((max(lengths) + PAGE - 1) // PAGE, 0) + extra
    table = np.full((len(lengths), width), -1, np.int32)
    order = rng.permutation(P)
    at = 0
    for b, n in enumerate(lengths):
        k = (n + PAGE - 1) // PAGE
        table[b, :k] = order[at:at + k]
        at += k
    return table


def _pages(lengths):
    return sum((n + PAGE - 1) // PAGE for n in lengths) + 1


def _cu(counts):
    return np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)


def _append(cache, k, v, cu, lengths, table, **kw):
    return dptq.kv8_append(_d(k), _d(v), _d(cu), _d(np.array(lengths, np.int32)), _d(table), cache, **kw)


def _filled(rng, lengths, H, D):
    """A cache that holds sequences of these lengths, written by the library and checked against the oracle."""
    P = _pages(lengths)
    arrays, table = _garbage(rng, P, H, D), _table(rng, lengths, P)
    k, v, cu = _rows(rng, sum(lengths), H, D), _rows(rng, sum(lengths), H, D), _cu(lengths)
    cache = _append(_cache(arrays), k, v, cu, lengths, table)
    ref = kv8_append_ref(k, v, cu, lengths, table, arrays)
    _same(cache, ref)
    return cache, ref, table


def _same(cache, ref):
    for got, want, what in zip(_host(cache), ref, ("K codes", "V codes", "K scales", "V scales")):
        assert np.array_equal(got.view(np.uint8), want.view(np.uint8)), what


APPENDS = [
    # (lengths before, new tokens, heads, head_dim)
    ([0], [1], 1, 64), ([0, 63, 64, 65], [1, 1, 1, 1], 2, 128), ([5], [59], 3, 64), ([5], [60], 1, 128),
    ([0], [300], 2, 256), ([0, 17, 100, 0], [130, 0, 29, 64], 2, 128), ([127, 128, 1], [1, 2, 200], 8, 64),
    ([62], [3], 5, 256), ([0] * 9, [1, 2, 3, 63, 64, 65, 127, 128, 129], 1, 128),
]


@pytest.mark.parametrize("before,new,H,D", APPENDS)
def test_append_matches_oracle(before, new, H, D):
    rng = np.random.default_rng(len(before) * 1000 + sum(new) + D)
    lengths = [a + b for a, b in zip(before, new)]
    P = _pages(lengths)
    table, arrays = _table(rng, lengths, P), _garbage(rng, P, H, D)
    cache, ref = _cache(arrays), arrays
    if sum(before):
        k, v = _rows(rng, sum(before), H, D), _rows(rng, sum(before), H, D)
        _append(cache, k, v, _cu(before), before, table)
        ref = kv8_append_ref(k, v, _cu(before), before, table, ref)
        _same(cache, ref)
    k, v = 3 * _rows(rng, sum(new), H, D), 0.1 * _rows(rng, sum(new), H, D)
    k, v = k.astype(np.float16), v.astype(np.float16)
    ref = kv8_append_ref(k, v, _cu(new), lengths, table, ref)
    for _ in range(2):     # the same call again leaves the cache as it is
        _append(cache, k, v, _cu(new), lengths, table)
        _same(cache, ref)
    for hint in (1, 65):   # and no hint changes it
        _same(_append(cache, k, v, _cu(new), lengths, table, max_new=hint), ref)


def test_append_every_code_and_growth():
    # All fp16 magnitudes through one page, then a token that makes the scale grow by 2^20, 2^9 and 2^3.
    D = 128
    bits = np.arange(0x7C00, dtype=np.uint16)
    vals = bits.view(np.float16)
    rng = np.random.default_rng(9)
    for top in (448.0, 2.0 ** -15, 65504.0, 1.0):
        pool = vals[vals <= top]
        n = 40
        k = (rng.choice(pool, (n, 1, D)) * rng.choice([-1, 1], (n, 1, D))).astype(np.float16)
        k[0, 0, :4] = [top, -top, 0, -0.0]
        v = (rng.choice(pool, (n, 1, D)) * np.float16(0.25)).astype(np.float16)
        P, table = 2, np.array([[1, 0]], np.int32)
        arrays = _garbage(rng, P, 1, D)
        cache = _cache(arrays)
        ref = arrays
        at = 0
        for count, factor in ((n, 1), (1, 8), (1, 512), (1, 2 ** 20), (1, 1)):
            kk = np.clip(k[:count].astype(np.float64) * factor, -65504, 65504).astype(np.float16)
            vv = np.clip(v[:count].astype(np.float64) * factor, -65504, 65504).astype(np.float16)
            at += count
            _append(cache, kk, vv, _cu([count]), [at], table)
            ref = kv8_append_ref(kk, vv, _cu([count]), [at], table, ref)
            _same(cache, ref)


def test_append_rows_of_wider_ones_and_zeros():
    rng = np.random.default_rng(10)
    H, D, n = 2, 64, 70
    wide = _rows(rng, n, 3 * H, D).reshape(n, 3 * H * D)
    wide[:, H * D:2 * H * D] = 0                     # K all zeros: the lowest scale
    w = _d(wide)
    k, v = (w[:, i * H * D:(i + 1) * H * D].unflatten(1, (H, D)) for i in (1, 2))
    arrays, table = _garbage(rng, 2, H, D), np.array([[0, 1]], np.int32)
    cache = dptq.kv8_append(k, v, _d(_cu([n])), _d(np.array([n], np.int32)), _d(table), _cache(arrays))
    ref = kv8_append_ref(k.cpu().numpy(), v.cpu().numpy(), _cu([n]), [n], table, arrays)
    _same(cache, ref)
    assert np.all(ref[2] == np.float32(2.0 ** -32))


def test_append_leaves_out_pages_that_are_not_there():
    # Entries outside [0, P), tokens past the table, and tokens before position 0 are not written.
    rng = np.random.default_rng(11)
    H, D = 2, 64
    arrays = _garbage(rng, 4, H, D)
    table = np.array([[0, 4, 2], [-7, 1, 2 ** 31 - 1]], np.int32)
    counts, lengths = [192, 300], [192, 250]
    k, v = _rows(rng, 492, H, D), _rows(rng, 492, H, D)
    cache = _append(_cache(arrays), k, v, _cu(counts), lengths, table)
    _same(cache, kv8_append_ref(k, v, _cu(counts), lengths, table, arrays))


def _attend(rng, before, new, H, Hkv, D, window=0, sinks=0, scale=None, q_size=1.5, **kw):
    lengths = [a + b for a, b in zip(before, new)]
    cache, ref, table = _filled(rng, lengths, Hkv, D)
    T = sum(new)
    q = (q_size * rng.standard_normal((T, H, D))).astype(np.float16)
    cu, n = _cu(new), np.array(lengths, np.int32)
    args = (_d(q), _d(cu), _d(n), _d(table), cache, scale, window, sinks)
    want = kv8_attention_ref(q, cu, n, table, ref, D ** -0.5 if scale is None else scale, window, sinks)
    for hints in ((kw,) if kw else ({}, dict(max_q=max(new), max_len=max(lengths)))):
        _matches(dptq.kv8_attention(*args, **hints), want)
    return args, want


def _matches(got, want):
    out, lse = (t.cpu().numpy().astype(np.float64) for t in got)
    r_out, r_lse, tol_out, tol_lse = want
    empty = np.isneginf(r_lse)
    assert np.array_equal(np.isneginf(lse), empty) and not np.isnan(lse).any()
    assert np.all(np.abs(lse - np.where(empty, 0, r_lse))[~empty] <= tol_lse[~empty])
    bad = ~(np.abs(out - r_out) <= tol_out)
    assert not bad.any(), (bad.sum(), np.argwhere(bad)[:3], np.abs(out - r_out)[bad][:3], tol_out[bad][:3])
    assert np.all(out[empty] == 0)


DECODES = [
    # (lengths before, H, Hkv, D, window, sinks)
    ([0], 1, 1, 64, 0, 0), ([0], 8, 8, 128, 0, 0), ([62], 4, 2, 128, 0, 0), ([63], 4, 1, 128, 0, 0),
    ([64], 3, 3, 64, 0, 0), ([300, 5, 0, 1000], 8, 2, 128, 0, 0), ([776], 32, 8, 128, 0, 0),
    ([130], 17, 1, 128, 0, 0), ([200], 40, 1, 64, 0, 0), ([511], 14, 2, 256, 0, 0), ([2100], 5, 1, 256, 0, 0),
    ([1000], 8, 2, 128, 64, 0), ([1000], 8, 2, 128, 1, 0), ([1000], 8, 2, 128, 1, 1), ([1000], 4, 4, 64, 100, 4),
    ([1000, 30, 99], 8, 2, 128, 100, 65), ([500], 8, 2, 128, 100, 450), ([500], 8, 2, 128, 100, 1000),
    ([500], 8, 2, 128, 5000, 4), ([4999], 6, 2, 128, 130, 3),
]


@pytest.mark.parametrize("before,H,Hkv,D,window,sinks", DECODES)
def test_decode_matches_definition(before, H, Hkv, D, window, sinks):
    rng = np.random.default_rng(sum(before) + H * 7 + D + window)
    _attend(rng, before, [1] * len(before), H, Hkv, D, window, sinks)


PROMPTS = [
    # (lengths before, new tokens, H, Hkv, D, window, sinks)
    ([0], [2], 1, 1, 64, 0, 0), ([0], [64], 2, 1, 128, 0, 0), ([0], [65], 2, 2, 128, 0, 0),
    ([0, 0], [130, 77], 4, 2, 128, 0, 0), ([100, 3], [33, 150], 6, 2, 64, 0, 0), ([0], [200], 3, 1, 256, 0, 0),
    ([300], [9], 8, 1, 128, 0, 0), ([1], [129], 5, 1, 128, 0, 0), ([0], [260], 2, 1, 128, 64, 0),
    ([70], [300], 2, 2, 64, 100, 4), ([0], [333], 4, 4, 128, 1, 0), ([10], [257], 2, 1, 128, 130, 70),
    ([700, 0, 64], [190, 1, 64], 4, 2, 128, 200, 2), ([0, 0, 40], [0, 140, 1], 4, 1, 128, 0, 0),
    ([0], [150], 2, 1, 256, 50, 5),
]


@pytest.mark.parametrize("before,new,H,Hkv,D,window,sinks", PROMPTS)
def test_prompt_matches_definition(before, new, H, Hkv, D, window, sinks):
    rng = np.random.default_rng(sum(before) + sum(new) * 3 + H * 7 + D + window)
    _attend(rng, before, new, H, Hkv, D, window, sinks)


@pytest.mark.parametrize("new", [[1, 1, 1], [40, 1, 90]])
def test_hints_change_no_result(new):
    rng = np.random.default_rng(21)
    args, want = _attend(rng, [300, 0, 1900], new, 8, 2, 128)
    for max_q in (1, 3, 17, 1000):
        for max_len in (1, 64, 700, 10 ** 6):
            _matches(dptq.kv8_attention(*args, max_q=max_q, max_len=max_len), want)


@pytest.mark.parametrize("new", [1, 150])
def test_peaked_and_large_scores(new):
    rng = np.random.default_rng(22)
    _attend(rng, [400], [new], 4, 2, 128, q_size=30.0)               # scores of hundreds: nearly one key each
    _attend(rng, [400], [new], 4, 2, 128, scale=0.0)                 # all equal
    _attend(rng, [400], [new], 4, 2, 128, scale=-0.3)


@pytest.mark.parametrize("new", [1, 140])
def test_pages_of_very_different_sizes(new):
    # V scales of neighbouring pages far apart, both ways.
    rng = np.random.default_rng(23)
    H, Hkv, D, n = 4, 2, 128, 700
    k, v = _rows(rng, n, Hkv, D), _rows(rng, n, Hkv, D).astype(np.float64)
    for blk in range(11):
        v[blk * PAGE:(blk + 1) * PAGE] *= 10.0 ** rng.integers(-4, 3)
    v = np.clip(v, -60000, 60000).astype(np.float16)
    P = 11
    arrays, table = _garbage(rng, P, Hkv, D), _table(rng, [n], P)
    cache = _append(_cache(arrays), k, v, _cu([n]), [n], table)
    ref = kv8_append_ref(k, v, _cu([n]), [n], table, arrays)
    q = rng.standard_normal((new, H, D)).astype(np.float16)
    args = (_d(q), _d(_cu([new])), _d(np.array([n], np.int32)), _d(table), cache)
    _matches(dptq.kv8_attention(*args), kv8_attention_ref(q, _cu([new]), [n], table, ref, D ** -0.5))


@pytest.mark.parametrize("new", [1, 100])
def test_rows_that_see_nothing(new):
    # A page table without pages, more queries than tokens, and a length of zero.
    rng = np.random.default_rng(24)
    H, Hkv, D = 4, 2, 128
    cache, ref, table = _filled(rng, [500], Hkv, D)
    table = np.repeat(table, 4, 0)
    table[1] = -1
    table[2, 1:4] = [2 ** 30, -5, cache[0].shape[0]]
    lengths = np.array([500, 500, 500, 0], np.int32)
    lengths[0] = max(new // 2, 1) if new > 1 else 500
    q = rng.standard_normal((4 * new, H, D)).astype(np.float16)
    cu = _cu([new] * 4)
    want = kv8_attention_ref(q, cu, lengths, table, ref, 0.1)
    assert np.isneginf(want[1]).any()
    for hints in ({}, dict(max_q=new, max_len=500)):
        _matches(dptq.kv8_attention(_d(q), _d(cu), _d(lengths), _d(table), cache, 0.1, **hints), want)


@pytest.mark.parametrize("new", [1, 80])
def test_what_is_masked_does_not_matter(new):
    # NaN codes past the end, in other sequences' pages and in pages behind the window.
    rng = np.random.default_rng(25)
    H, Hkv, D, n = 4, 2, 128, 400 + new
    args, want = _attend(rng, [400], [new], H, Hkv, D, 70, 3)
    cache, table = args[4], args[3].cpu().numpy()
    nan = torch.tensor(0x7F, dtype=torch.uint8, device="cuda")
    k, v = cache[0].view(torch.uint8), cache[1].view(torch.uint8)
    last, at = int(table[0, (n - 1) // PAGE]), n % PAGE
    if at:
        k[last, :, at:] = nan
        v[last, :, :, at:] = nan
    first_seen = (n - new - 69) // PAGE
    for blk in range(1, first_seen):
        k[int(table[0, blk])] = nan
        v[int(table[0, blk])] = nan
        cache[2][int(table[0, blk])] = float("nan")
        cache[3][int(table[0, blk])] = float("inf")
    spare = sorted(set(range(k.shape[0])) - set(table[0, :(n + PAGE - 1) // PAGE].tolist()))
    k[spare] = nan
    v[spare] = nan
    _matches(dptq.kv8_attention(*args), want)


def test_a_prompt_equals_its_tokens_one_by_one():
    # Appended and attended token by token, against the definition on the same cache.
    rng = np.random.default_rng(26)
    H, Hkv, D, n = 4, 2, 64, 70
    k, v, q = _rows(rng, n, Hkv, D), _rows(rng, n, Hkv, D), rng.standard_normal((n, H, D)).astype(np.float16)
    arrays, table = _garbage(rng, 2, Hkv, D), np.array([[1, 0]], np.int32)
    cache, ref = _cache(arrays), arrays
    for i in range(n):
        _append(cache, k[i:i + 1], v[i:i + 1], _cu([1]), [i + 1], table)
        ref = kv8_append_ref(k[i:i + 1], v[i:i + 1], _cu([1]), [i + 1], table, ref)
        _same(cache, ref)
        got = dptq.kv8_attention(_d(q[i:i + 1]), _d(_cu([1])), _d(np.array([i + 1], np.int32)), _d(table), cache)
        _matches(got, kv8_attention_ref(q[i:i + 1], _cu([1]), [i + 1], table, ref, D ** -0.5))


def test_strided_queries_streams_and_buffers():
    rng = np.random.default_rng(27)
    args, want = _attend(rng, [90, 10], [5, 60], 4, 2, 128)
    q = args[0]
    wide = torch.full((q.shape[0], 8 * 128), float("nan"), dtype=torch.float16, device="cuda")
    part = wide[:, 256:768].unflatten(1, (4, 128)).copy_(q)
    out, lse = torch.empty_like(q), torch.empty((q.shape[0], 4), device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = dptq.kv8_attention(part, *args[1:], out=out, lse=lse)
    side.synchronize()
    assert got[0] is out and got[1] is lse
    _matches(got, want)


def test_graph_replays():
    # Decode steps in a graph: lengths and pages are read on the device at each replay.
    rng = np.random.default_rng(28)
    H, Hkv, D, B = 8, 2, 128, 3
    before = [100, 700, 5]
    lengths = [n + 5 for n in before]
    P = _pages(lengths)
    arrays, table = _garbage(rng, P, Hkv, D), _table(rng, lengths, P)
    rows = [_rows(rng, sum(before), Hkv, D) for _ in range(2)]
    cache = _append(_cache(arrays), *rows, _cu(before), before, table)
    ref = kv8_append_ref(*rows, _cu(before), before, table, arrays)
    k, v = (torch.zeros((B, Hkv, D), dtype=torch.float16, device="cuda") for _ in range(2))
    q = torch.zeros((B, H, D), dtype=torch.float16, device="cuda")
    n, cu, tab = _d(np.array(before, np.int32)), _d(_cu([1] * B)), _d(table)
    out, lse = torch.empty_like(q), torch.empty((B, H), device="cuda")

    def step():
        dptq.kv8_append(k, v, cu, n, tab, cache, max_new=1)
        dptq.kv8_attention(q, cu, n, tab, cache, max_q=1, out=out, lse=lse)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        n.zero_()            # nothing is written or seen
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(5):
        new = [_rows(rng, B, Hkv, D) for _ in range(2)]
        qh = rng.standard_normal((B, H, D)).astype(np.float16)
        now = [b + i + 1 for b in before]
        k.copy_(_d(new[0]))
        v.copy_(_d(new[1]))
        q.copy_(_d(qh))
        n.copy_(_d(np.array(now, np.int32)))
        graph.replay()
        torch.cuda.synchronize()
        ref = kv8_append_ref(*new, _cu([1] * B), now, table, ref)
        _same(cache, ref)
        _matches((out, lse), kv8_attention_ref(qh, _cu([1] * B), now, table, ref, D ** -0.5))


def test_offsets_past_32_bits():
    # A cache of more than 2^32 bytes each way: the last pages and the first.
    H, Hkv, D = 8, 8, 128
    P = 2 ** 32 // (Hkv * PAGE * D) + 5
    cache = dptq.kv8_cache(P, Hkv, D)
    rng = np.random.default_rng(29)
    table = np.array([[P - 1, 0, P - 2, 1]], np.int32)
    n = 200
    k, v = _rows(rng, n, Hkv, D), _rows(rng, n, Hkv, D)
    _append(cache, k, v, _cu([n]), [n], table)
    pages = table[0].tolist()
    small = [cache[0].view(torch.uint8)[pages].cpu().numpy(), cache[1].view(torch.uint8)[pages].cpu().numpy(),
             cache[2][pages].cpu().numpy(), cache[3][pages].cpu().numpy()]
    local = np.arange(4, dtype=np.int32)[None]
    ref = kv8_append_ref(k, v, _cu([n]), [n], local, _garbage(rng, 4, Hkv, D))
    for got, want in zip(small, ref):
        assert np.array_equal(got.view(np.uint8), want.view(np.uint8))
    q = rng.standard_normal((1, H, D)).astype(np.float16)
    got = dptq.kv8_attention(_d(q), _d(_cu([1])), _d(np.array([n], np.int32)), _d(table), cache)
    _matches(got, kv8_attention_ref(q, _cu([1]), [n], local, ref, D ** -0.5))


def test_kv8_refusals():
    c = dptq.kv8_cache(3, 2, 64)
    f16, i32 = dict(dtype=torch.float16, device="cuda"), dict(dtype=torch.int32, device="cuda")
    k, q = torch.zeros((4, 2, 64), **f16), torch.zeros((4, 4, 64), **f16)
    cu, n, t = torch.tensor([0, 4], **i32), torch.tensor([4], **i32), torch.zeros((1, 2), **i32)

    def append(k=k, v=k, cu=cu, n=n, t=t, c=c, **kw):
        return dptq.kv8_append(k, v, cu, n, t, c, **kw)

    def attend(q=q, cu=cu, n=n, t=t, c=c, **kw):
        return dptq.kv8_attention(q, cu, n, t, c, **kw)

    for call, error, text in [
        (lambda: append(k=k.float()), TypeError, "k must have dtype torch.float16"),
        (lambda: append(k=k[:, :1]), ValueError, "k must be 3-D"),
        (lambda: append(v=k[:2]), ValueError, "v must be 3-D"),
        (lambda: append(k=torch.zeros((2, 4, 64), **f16).transpose(0, 1)), ValueError, "dense heads"),
        (lambda: append(k=torch.zeros((4, 2 * 64 + 4), **f16)[:, :128].unflatten(1, (2, 64))), ValueError,
         "multiple of 8"),
        (lambda: append(cu=cu.long()), TypeError, "cu_seqlens must have dtype torch.int32"),
        (lambda: append(cu=cu[:1]), ValueError, "cu_seqlens must have shape"),
        (lambda: append(t=t[0]), ValueError, "page_table must be 2-D"),
        (lambda: append(t=torch.zeros((2, 2), **i32)), ValueError, "page_table must be 2-D"),
        (lambda: append(c=c._replace(k_pages=c[0].view(torch.uint8))), TypeError, "float8_e4m3fn"),
        (lambda: append(c=c._replace(v_pages=dptq.kv8_cache(3, 2, 128)[1])), ValueError, "v_pages must have shape"),
        (lambda: append(max_new=-1), ValueError, "max_new must not be negative"),
        (lambda: append(n=n.cpu()), ValueError, "lengths must be a GPU tensor"),
        (lambda: attend(q=q[:, :3]), ValueError, "multiple of the cache's kv_heads"),
        (lambda: attend(q=torch.zeros((4, 4, 128), **f16)), ValueError, "q must be 3-D"),
        (lambda: attend(window=-1), ValueError, "window must be in"),
        (lambda: attend(sinks=2 ** 31), ValueError, "sinks must be in"),
        (lambda: attend(max_q=1.5), TypeError, "max_q must be an integer"),
        (lambda: attend(out=q[:1]), ValueError, "out must have shape"),
    ]:
        with pytest.raises(error, match=text):
            call()
    for call, status in [
        (lambda: attend(scale=float("nan")), 1), (lambda: attend(scale=float("inf")), 1),
        (lambda: attend(window=2 ** 30), 2),
        (lambda: append(k=torch.zeros((4, 2, 96), **f16), v=torch.zeros((4, 2, 96), **f16),
                        c=dptq.kv8_cache(3, 2, 96)), 2),
    ]:
        with pytest.raises(dptq.DptqError) as e:
            call()
        assert e.value.status == status
    assert append(k=k[:0], v=k[:0]) is c
    out, lse = attend(q=q[:0])
    assert out.shape == (0, 4, 64) and lse.shape == (0, 4)


def test_e4m3_values_of_the_oracle_are_the_dtype_s():
    codes = torch.arange(256, dtype=torch.uint8)
    got = codes.view(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(got, e4m3_values().astype(np.float32), equal_nan=True)
