"""The operators of a serving step around the quantized linear, as they are measured.

Each case is one pass of one operator, through the functions of
``paper_2606_12487_amd`` where ``own`` is true, and as elementary torch
operations in 32 bits where it is false.

Kinds (``case["kind"]``):

* ``norm``      ``rms_norm_quant``: residual addition, RMS norm and 8-bit codes with a scale per row;
* ``append``    ``kv8_append``: new keys and values into the 8-bit paged cache;
* ``attention`` ``kv8_attention``: attention of new queries over that cache;
* ``logprobs``  ``token_logprobs``: log probabilities of given tokens, entropy, top alternatives.

The cache: pages of 64 tokens, K codes [pages, kv_heads, 64, D] and V codes
[pages, kv_heads, D, 64] in float8 e4m3, with one power-of-two fp32 scale per
page and head, for K and for V.
"""

import math
import random

import torch

own = False

PAGE = 64       # tokens of a cache page
TOP = 448.0     # largest e4m3 value
LOWEST = -32    # exponent of the smallest scale


def listed():
    return [
        # One token of one sequence before a projection: latency.
        dict(name="norm_token_k4096", kind="norm", M=1, K=4096),
        # A prompt of ragged length before a large model's 8-bit projection.
        dict(name="norm_prompt_m4001_k8192", kind="norm", M=4001, K=8192),
        # A decode step's keys and values: one token for each of 64 sequences.
        dict(name="append_decode_b64", kind="append", B=64, Hkv=8, D=128, q=1, len=1000),
        # Chunks of three prompts, ragged, that begin and end inside pages.
        dict(name="append_prompt_b3", kind="append", B=3, Hkv=8, D=128, q=2048, len=4000),
        # Decode of one short conversation: latency.
        dict(name="attn_decode_b1_len777", kind="attention", B=1, H=32, Hkv=8, D=128, q=1, len=777, window=0, sinks=0),
        # A large decode batch with lengths from short to long: the throughput of serving.
        dict(name="attn_decode_b64_len8192", kind="attention", B=64, H=64, Hkv=8, D=128, q=1, len=8192, window=0,
             sinks=0),
        # Two sequences with very long contexts.
        dict(name="attn_decode_b2_len131072", kind="attention", B=2, H=64, Hkv=8, D=128, q=1, len=131072, window=0,
             sinks=0),
        # Streaming decode: a window of the last tokens and four first ones, a head per key head.
        dict(name="attn_decode_window_b16", kind="attention", B=16, H=32, Hkv=32, D=128, q=1, len=16384, window=4096,
             sinks=4),
        # Prefill chunks of two prompts behind what their caches hold already.
        dict(name="attn_prompt_b2_q2048", kind="attention", B=2, H=64, Hkv=8, D=128, q=2048, len=4096, window=0,
             sinks=0),
        # A prompt through windowed layers with small heads, odd lengths.
        dict(name="attn_prompt_window_q1000", kind="attention", B=1, H=32, Hkv=8, D=64, q=1000, len=5003, window=1024,
             sinks=4),
        # Answers of a decode batch with their alternatives, part of the vocabulary masked off.
        dict(name="logprobs_b64_top20", kind="logprobs", M=64, V=131072, top=20, half=True, masked=True),
        # Scoring of a text: every position's token, an odd vocabulary, fp32 logits.
        dict(name="logprobs_m2047_v100003", kind="logprobs", M=2047, V=100003, top=0, half=False, masked=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "append", "attention", "attention", "attention", "logprobs"])
    if kind == "norm":
        K = rng.choice([2048, 2560, 3584, 4096, 5120, 8192, 8 * rng.randint(128, 1024)])
        return dict(kind=kind, M=_log_int(rng, 1, 4001), K=K)
    Hkv = rng.choice([1, 2, 4, 8, 8, 16])
    D = rng.choice([64, 128, 128, 128, 256])
    if kind == "append":
        q = rng.choice([1, _log_int(rng, 2, 2048)])
        B = _log_int(rng, 1, 64 if q == 1 else max(2, 4096 // q))
        return dict(kind=kind, B=min(B, 64), Hkv=min(Hkv, 8), D=D, q=q, len=q + _log_int(rng, 1, 1024))
    if kind == "attention":
        H = Hkv * rng.choice([g for g in (1, 2, 3, 4, 5, 7, 8, 16) if g * Hkv <= 64])
        window, sinks = rng.choice([(0, 0), (0, 0), (_log_int(rng, 16, 4096), rng.choice([0, 1, 4, 100]))])
        if rng.random() < 0.6:
            n = _log_int(rng, 1, 65536)
            B = _log_int(rng, 1, max(1, min(64, 2 ** 28 // (n * Hkv * D))))
            return dict(kind=kind, B=B, H=H, Hkv=Hkv, D=D, q=1, len=n, window=window, sinks=sinks)
        q = _log_int(rng, 2, 2048)
        n = q + _log_int(rng, 1, min(4096, 2 ** 29 // (H * q) - q))
        B = rng.randint(1, max(1, min(8, 2 ** 29 // (H * q * n))))
        return dict(kind=kind, B=B, H=H, Hkv=Hkv, D=D, q=q, len=n, window=window, sinks=sinks)
    V = rng.choice([1000, 32768, 65536, 131072, _log_int(rng, 2, 131072)])
    top = rng.choice([0, 0, 1, 5, 20])
    M = _log_int(rng, 1, min(2047, (64 if top else 1024) * 131072 // V))
    return dict(kind=kind, M=M, V=V, top=min(top, V), half=rng.random() < 0.5, masked=rng.random() < 0.3)


# ---------------------------------------------------------------------------
# Inputs, all from the seed
# ---------------------------------------------------------------------------
def _gen(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed(1_000_003 * int(seed) + stream)
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _norm_inputs(case, seed):
    # A residual stream with a few massive channels, and an update of its size.
    g = _gen(seed, 1)
    M, K = case["M"], case["K"]
    res = _randn(g, M, K)
    res[:, torch.randperm(K, generator=g, device="cuda")[:3]] *= 40
    x = _randn(g, M, K)
    w = 1 + 0.2 * _randn(g, K)
    return x.half(), res.half(), w.half()


def _scale_of(absmax):
    """2^e, the smallest with absmax <= 448 * 2^e and e >= LOWEST, of an fp32 absmax."""
    m, e = torch.frexp(absmax)                  # absmax = m * 2^e, 1/2 <= m < 1; 448 = 7/8 * 2^9
    e = torch.where(m <= TOP / 512, e - 9, e - 8)
    e = torch.where(absmax > 0, e, LOWEST).clamp(min=LOWEST)
    return ((e + 127) << 23).int().view(torch.float32)


def _rows(g, T, heads, D):
    """Keys or values: a spread over the channels, an outlier channel in each head, an offset for each token."""
    x = _randn(g, T, heads, D) * (0.2 + 1.8 * torch.rand((heads, D), generator=g, device="cuda"))
    x[:, :, int(torch.randint(0, D, (1,), generator=g, device="cuda"))] *= 8
    return x + 0.3 * _randn(g, T, heads, 1)


def _sizes(case):
    """New tokens and lengths (with them) of the case's sequences, ragged, the first as large as the case says."""
    r = random.Random("%(B)d %(q)d %(len)d" % case)
    q, n = case["q"], case["len"]
    counts = [q] + [r.randint((q + 2) // 3, q) for _ in range(case["B"] - 1)]
    return counts, [n] + [max(c, r.randint((n + 3) // 4, n)) for c in counts[1:]]


def _plan(case, seed):
    """Lengths, query counts, page table and page count of the case's sequences."""
    g = torch.Generator()
    g.manual_seed(int(seed) * 7 + 3)
    B, n = case["B"], case["len"]
    counts, lengths = (torch.tensor(x) for x in _sizes(case))
    cu = torch.zeros(B + 1, dtype=torch.int64)
    cu[1:] = counts.cumsum(0)
    width = (n + PAGE - 1) // PAGE
    pages = B * width
    table = torch.randperm(pages, generator=g).reshape(B, width)
    held = (lengths + PAGE - 1) // PAGE
    table = torch.where(torch.arange(width) < held[:, None], table, -1)
    return dict(T=int(cu[-1]), pages=pages, cu=cu.int().cuda(), lengths=lengths.int().cuda(), table=table.int().cuda())


def _cache(g, pages, Hkv, D):
    """Filled pages: codes and scales as K and V of ordinary tokens give them."""
    got = []
    for _ in range(2):
        x = _rows(g, pages * PAGE, Hkv, D).half().reshape(pages, PAGE, Hkv, D).transpose(1, 2)
        s = _scale_of(x.abs().amax((2, 3)).float())
        got += [(x / s[:, :, None, None]).to(torch.float8_e4m3fn), s]
        del x
    k, ks, v, vs = got
    return [k.contiguous(), v.view(torch.uint8).transpose(2, 3).contiguous().view(torch.float8_e4m3fn), ks, vs]


def _logits_inputs(case, seed):
    g = _gen(seed, 4)
    M, V = case["M"], case["V"]
    x = 3 * _randn(g, M, V)
    if case["masked"]:   # a grammar leaves a tenth of the tokens in every other row
        x[::2].masked_fill_(torch.rand((V,), generator=g, device="cuda") < 0.9, -math.inf)
    tokens = torch.randint(0, V, (M,), generator=g, device="cuda")
    tokens = torch.where(torch.arange(M, device="cuda") % 16 == 15, -1, tokens)   # padding: not scored
    return (x.half() if case["half"] else x), tokens


def prepare(case, seed):
    kind = case["kind"]
    if kind == "norm":
        x, res, w = _norm_inputs(case, seed)
        return dict(case=case, x=x, res=res, w=w, values=torch.empty_like(x))
    if kind == "logprobs":
        x, tokens = _logits_inputs(case, seed)
        return dict(case=case, x=x, tokens=tokens)
    plan = _plan(case, seed)
    g = _gen(seed, 2)
    Hkv, D = case["Hkv"], case["D"]
    whole = _cache(g, plan["pages"] + 1, Hkv, D)   # the last page is the plain form's, for what belongs to no sequence
    s = dict(case=case, whole=whole, cache=[x[:-1] for x in whole], **plan)
    if kind == "append":
        # K and V lie in the output of one fused projection: rows of a wider matrix.
        kv = torch.empty((s["T"], 3 * Hkv * D), dtype=torch.float16, device="cuda")
        s["k"] = kv[:, Hkv * D:2 * Hkv * D].unflatten(1, (Hkv, D)).copy_(_rows(g, s["T"], Hkv, D))
        s["v"] = kv[:, 2 * Hkv * D:].unflatten(1, (Hkv, D)).copy_(_rows(g, s["T"], Hkv, D))
    else:
        s["q"] = (1.5 * _randn(g, s["T"], case["H"], D)).half()
    return s


# ---------------------------------------------------------------------------
# The framework's calls
# ---------------------------------------------------------------------------
def _run_own(s):
    import paper_2606_12487_amd as dptq
    case = s["case"]
    kind = case["kind"]
    if kind == "norm":
        codes, scales, h = dptq.rms_norm_quant(s["x"], s["w"], 1e-5, residual=s["res"])
        # The 8-bit codes as the values that they stand for.
        return torch.mul(codes, scales[:, None], out=s["values"]), scales, h
    if kind == "logprobs":
        return dptq.token_logprobs(s["x"], s["tokens"], top=case["top"])
    cache = dptq.KV8Cache(*s["cache"])
    if kind == "append":
        return dptq.kv8_append(s["k"], s["v"], s["cu"], s["lengths"], s["table"], cache, max_new=case["q"])
    return dptq.kv8_attention(s["q"], s["cu"], s["lengths"], s["table"], cache, window=case["window"],
                              sinks=case["sinks"], max_q=case["q"], max_len=case["len"])


# ---------------------------------------------------------------------------
# The plain forms: elementary operations in 32 bits
# ---------------------------------------------------------------------------
def _plain_norm(s):
    h = (s["x"].float() + s["res"].float()).half()
    hf = h.float()
    t = hf * s["w"].float()
    step = t.abs().amax(1, keepdim=True) / 127
    codes = torch.where(step > 0, torch.round(t / step), torch.zeros_like(t)).clamp(-127, 127)
    scales = step * torch.rsqrt(hf.square().mean(1, keepdim=True) + 1e-5)
    return torch.mul(codes, scales, out=s["values"]), scales[:, 0], h


def _touched(s):
    """Pages that the new tokens touch [B, n] (the spare page where there is none), which of them there are, the
    positions of their slots [B, n, 64], each sequence's first new position [B, 1, 1], and which slots are new and
    from which token row."""
    case = s["case"]
    n = (case["q"] + PAGE - 2) // PAGE + 1
    lengths = s["lengths"].long()
    counts = (s["cu"][1:] - s["cu"][:-1]).long()
    start = lengths - counts
    block = start[:, None] // PAGE + torch.arange(n, device="cuda")
    there = block * PAGE < lengths[:, None]
    page = torch.gather(s["table"].long(), 1, block.clamp(max=s["table"].shape[1] - 1))
    page = torch.where(there, page, s["pages"])
    pos = block[:, :, None] * PAGE + torch.arange(PAGE, device="cuda")
    start = start[:, None, None]
    new = (pos >= start) & (pos < lengths[:, None, None]) & there[:, :, None]
    row = torch.where(new, s["cu"][:-1].long()[:, None, None] + pos - start, 0)
    return page, there, pos, start, new, row


def _plain_append(s):
    page, there, pos, start, new, row = _touched(s)
    B, n = page.shape
    flat = page.reshape(-1)
    fresh = pos[:, :, 0] >= start[:, :, 0]     # a page whose first slot is written now
    old = (pos < start)[:, :, None, :, None]
    k_pages, v_pages, k_scales, v_scales = s["whole"]
    for x, codes, scales, transposed in ((s["k"], k_pages, k_scales, False), (s["v"], v_pages, v_scales, True)):
        x = torch.where(new[:, :, :, None, None], x[row].float(), 0.0).transpose(2, 3)       # [B, n, Hkv, 64, D]
        had = torch.where(fresh[:, :, None], 0.0, scales[flat].reshape(B, n, -1))
        step = torch.maximum(_scale_of(x.abs().amax((3, 4))), had)
        c = codes.view(torch.uint8)[flat].view(torch.float8_e4m3fn).float()
        c = (c.transpose(2, 3) if transposed else c).reshape(x.shape)
        kept = torch.where(fresh[:, :, None, None, None], 0.0, c)     # a new page begins with zeros
        kept = torch.where(old, c * (had / step)[..., None, None], kept)
        c = torch.where(new[:, :, None, :, None], x / step[..., None, None], kept)
        c = torch.where(there[:, :, None, None, None], c, torch.zeros_like(c)).flatten(0, 1)
        c = (c.transpose(2, 3) if transposed else c).to(torch.float8_e4m3fn)
        codes.view(torch.uint8)[flat] = c.view(torch.uint8)
        scales[flat] = torch.where(there[:, :, None], step, torch.ones_like(step)).flatten(0, 1)
    return s["cache"]


def _visible(case, lengths, counts, device):
    """[B, q, len] whether a query sees a position."""
    j = torch.arange(case["len"], device=device)
    i = torch.arange(case["q"], device=device)
    p = ((lengths - counts)[:, None] + i)[:, :, None]
    seen = (j <= p) & (i < counts[:, None])[:, :, None]
    if case["window"]:
        seen &= (j > p - case["window"]) | (j < case["sinks"])
    return seen


def _token_places(s):
    """(sequence, index among its queries) of each query token."""
    t = torch.arange(s["T"], device="cuda")
    b = torch.searchsorted(s["cu"][1:].long(), t, right=True)
    return b, t - s["cu"][:-1].long()[b]


def _plain_attention(s):
    case = s["case"]
    B, H, Hkv, D, Q, n = (case[x] for x in ("B", "H", "Hkv", "D", "q", "len"))
    k_pages, v_pages, k_scales, v_scales = s["cache"]
    table = s["table"].long().clamp(min=0)
    k = k_pages.view(torch.uint8)[table].view(torch.float8_e4m3fn).float() * k_scales[table][..., None, None]
    v = v_pages.view(torch.uint8)[table].view(torch.float8_e4m3fn).float() * v_scales[table][..., None, None]
    k = k.transpose(1, 2).reshape(B, Hkv, -1, D)[:, :, :n]                        # [B, Hkv, len, D]
    v = v.permute(0, 2, 1, 4, 3).reshape(B, Hkv, -1, D)[:, :, :n]
    counts = (s["cu"][1:] - s["cu"][:-1]).long()
    rows = (s["cu"][:-1].long()[:, None] + torch.arange(Q, device="cuda")).clamp(max=s["T"] - 1)
    q = s["q"][rows].float().reshape(B, Q, Hkv, H // Hkv, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, -1, D)
    seen = _visible(case, s["lengths"].long(), counts, "cuda")[:, None, None]     # [B, 1, 1, Q, len]
    x = (q @ k.transpose(2, 3).contiguous()).mul_(D ** -0.5).reshape(B, Hkv, H // Hkv, Q, n)
    x = x.masked_fill_(~seen, -math.inf)
    m = x.amax(4, keepdim=True)
    x = x.sub_(torch.where(m > -math.inf, m, 0.0)).exp_()
    total = x.sum(4, keepdim=True)
    o = (x.reshape(B, Hkv, -1, n) @ v).reshape(B, Hkv, H // Hkv, Q, D) / torch.where(total > 0, total, 1.0)
    lse = m + torch.log(total)
    b, i = _token_places(s)
    o = o.permute(0, 3, 1, 2, 4).reshape(B, Q, H, D)[b, i]
    lse = lse[..., 0].permute(0, 3, 1, 2).reshape(B, Q, H)[b, i]
    return o.half(), lse


def _plain_logprobs(s):
    case = s["case"]
    x, tokens = s["x"].float(), s["tokens"]
    m = x.amax(1, keepdim=True)
    z = x - m
    e = torch.exp(z)
    total = e.sum(1, keepdim=True)
    lse = m + torch.log(total)
    picked = torch.gather(x, 1, tokens.clamp(min=0)[:, None])
    picked = torch.where(picked > -math.inf, picked - lse, -math.inf)[:, 0]
    logprobs = torch.where(tokens >= 0, picked, 0.0)
    entropy = torch.log(total) - torch.where(e > 0, e * z, 0.0).sum(1, keepdim=True) / total
    entropy = torch.where(m > -math.inf, entropy, 0.0)[:, 0]          # all masked: nothing to choose from
    if case["top"]:
        values, ids = torch.sort(x, dim=1, descending=True, stable=True)
        values, ids = values[:, :case["top"]], ids[:, :case["top"]]
        return logprobs, entropy, torch.where(values > -math.inf, values - lse, -math.inf), ids
    return logprobs, entropy, x[:, :0], tokens[:, None][:, :0]


def run(state):
    if own:
        return _run_own(state)
    kind = state["case"]["kind"]
    if kind == "norm":
        return _plain_norm(state)
    if kind == "append":
        return _plain_append(state)
    if kind == "attention":
        return _plain_attention(state)
    return _plain_logprobs(state)


# ---------------------------------------------------------------------------
# Work: each input read once, each output written once
# ---------------------------------------------------------------------------
def _seen(case):
    """Keys that each key head has to give, and pairs of a query and a key that it sees."""
    keys = pairs = 0
    for q, n in zip(*_sizes(case)):
        w, sinks = case["window"] or n, case["sinks"]
        for p in range(n - q, n):
            low = max(0, p + 1 - w)
            pairs += p + 1 - low + min(sinks, low)
        low = max(0, n - q + 1 - w)
        keys += n - low + min(sinks, low)
    return keys, pairs


def work(case):
    kind = case["kind"]
    if kind == "norm":
        M, K = case["M"], case["K"]
        return {"bytes": 7 * M * K + 2 * K + 4 * M, "flops": 6 * M * K}
    if kind == "logprobs":
        M, V = case["M"], case["V"]
        return {"bytes": M * (V * (2 if case["half"] else 4) + 8 + 8 + 12 * case["top"]), "flops": 4 * M * V}
    Hkv, D = case["Hkv"], case["D"]
    counts, lengths = _sizes(case)
    tokens = sum(counts)
    if kind == "append":
        blocks = sum((n - 1) // PAGE - (n - q) // PAGE + 1 for q, n in zip(counts, lengths))
        return {"bytes": tokens * 2 * Hkv * D * 3 + blocks * (4 + 16 * Hkv) + 8 * case["B"],
                "flops": 4 * tokens * Hkv * D}
    keys, pairs = _seen(case)
    H = case["H"]
    return {"bytes": keys * Hkv * (2 * D + 8 / PAGE) + tokens * H * (4 * D + 4), "flops": 4 * pairs * H * D}


# ---------------------------------------------------------------------------
# The same values in 64 bits
# ---------------------------------------------------------------------------
def _pow2(e):
    return ((e + 1023) << 52).view(torch.float64)


def _e4m3(x):
    """x in 64 bits, |x| <= 448, to the nearest e4m3 value, half to even: steps of 2^(e - 3), at least 2^-9."""
    step = _pow2(torch.frexp(x)[1].long().sub(4).clamp(min=-9))
    return torch.round(x / step) * step


def _exact_norm(case, seed):
    x, res, w = _norm_inputs(case, seed)
    h = (x.double() + res.double()).half().double()      # a sum of two fp16 values is exact in 64 bits
    t = h * w.double()
    a = t.abs().amax(1, keepdim=True)
    codes = torch.round(t * 127 / torch.where(a > 0, a, 1.0))
    scales = a / 127 / torch.sqrt((h * h).mean(1, keepdim=True) + 1e-5)
    return codes * scales, scales[:, 0], h


def _exact_append(case, seed):
    s = prepare(case, seed)
    cu, lengths, table = s["cu"].tolist(), s["lengths"].tolist(), s["table"].tolist()
    outs = [c.double() for c in s["cache"]]
    for c, scales, x, transposed in ((outs[0], outs[2], s["k"], False), (outs[1], outs[3], s["v"], True)):
        for b in range(case["B"]):
            start, t = lengths[b] - (cu[b + 1] - cu[b]), cu[b]
            while start < lengths[b]:
                page, first = table[b][start // PAGE], start % PAGE
                count = min(PAGE - first, lengths[b] - start)
                rows = x[t:t + count].double().transpose(0, 1)                       # [Hkv, count, D]
                view = c[page].transpose(1, 2) if transposed else c[page]            # [Hkv, 64, D]
                a = rows.abs().amax((1, 2)).clamp(min=TOP * 2.0 ** LOWEST)
                step = _pow2(torch.frexp(a)[1].long() - 9)
                step = torch.where(a > TOP * step, 2 * step, step)
                if first:
                    step = torch.maximum(step, scales[page])
                    view[:, :first] = _e4m3(view[:, :first] * (scales[page] / step)[:, None, None])
                else:
                    view[:, count:] = 0
                view[:, first:first + count] = _e4m3(rows / step[:, None, None])
                scales[page] = step
                start, t = start + count, t + count
    return outs


def _exact_attention(case, seed):
    s = prepare(case, seed)
    H, Hkv, D, window = case["H"], case["Hkv"], case["D"], case["window"]
    cu, lengths, table = s["cu"].tolist(), s["lengths"].tolist(), s["table"].tolist()
    out = torch.empty((s["T"], H, D), dtype=torch.float64, device="cuda")
    lse = torch.empty((s["T"], H), dtype=torch.float64, device="cuda")
    for b in range(case["B"]):
        n, t0, nq = lengths[b], cu[b], cu[b + 1] - cu[b]
        pages = torch.tensor(table[b][:(n + PAGE - 1) // PAGE], device="cuda")
        p = torch.arange(n - nq, n, device="cuda")[:, None]
        j = torch.arange(n, device="cuda")[None]
        hidden = j > p
        if window:
            hidden |= (j <= p - window) & (j >= case["sinks"])
        for h in range(Hkv):
            k = s["cache"][0].view(torch.uint8)[pages, h].view(torch.float8_e4m3fn).double()
            v = s["cache"][1].view(torch.uint8)[pages, h].view(torch.float8_e4m3fn).double()
            k = (k * s["cache"][2][pages, h].double()[:, None, None]).reshape(-1, D)[:n]
            v = (v * s["cache"][3][pages, h].double()[:, None, None]).transpose(1, 2).reshape(-1, D)[:n]
            for g in range(h * (H // Hkv), (h + 1) * (H // Hkv)):
                x = (s["q"][t0:t0 + nq, g].double() @ k.t()) / math.sqrt(D)
                x.masked_fill_(hidden, -math.inf)
                lse[t0:t0 + nq, g] = torch.logsumexp(x, 1)
                out[t0:t0 + nq, g] = torch.exp(x - lse[t0:t0 + nq, g, None]) @ v
    return out, lse


def _exact_logprobs(case, seed):
    x, tokens = _logits_inputs(case, seed)
    lp, H, top, ids = [], [], [], []
    for rows, ts in zip(x.split(64), tokens.split(64)):
        y = torch.log_softmax(rows.double(), 1)
        y = torch.where(rows > -math.inf, y, -math.inf)
        p = torch.exp(y)
        lp.append(torch.where(ts < 0, 0.0, y.gather(1, ts.clamp(min=0)[:, None])[:, 0]))
        H.append(-torch.where(p > 0, p * y, 0.0).sum(1))
        if case["top"]:
            best = torch.sort(y, dim=1, descending=True, stable=True)[0]
            top.append(best[:, :case["top"]])
        else:
            top.append(y[:, :0])
    return torch.cat(lp), torch.cat(H), torch.cat(top), None


def exact(case, seed):
    return {"norm": _exact_norm, "append": _exact_append, "attention": _exact_attention,
            "logprobs": _exact_logprobs}[case["kind"]](case, seed)
