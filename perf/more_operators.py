"""More operators of a serving step, as they are measured: positions, the gated
feed-forward, and the choice of the next token.

Each case is one pass of one operator, through the functions of
``paper_2606_12487_amd`` where ``own`` is true, and as elementary torch
operations in 32 bits (angles, long sums and their borders in 64) where it is
false.

Kinds (``case["kind"]``):

* ``rotary``  ``rotary``: rotary positions on queries and keys;
* ``append``  ``rotary_kv8_append``: the same, with the keys and the values written into the 8-bit paged cache;
* ``gated``   ``qlinear_gated`` and its forms for other weight layouts: both projections of a gated feed-forward
  block, the activation and the product;
* ``sample``  ``sample_tokens``: one token of each row of logits under temperature, top-k, top-p and min-p.

Rotary pairs: channels (i, i + r/2) of the first r of a head, or (2i, 2i + 1)
where ``interleaved``; angles position * inv_freq[i].  The cache: pages of 64
tokens, K codes [pages, kv_heads, 64, D] and V codes [pages, kv_heads, D, 64] in
float8 e4m3, one power-of-two fp32 scale per page and head, for K and for V.
Weights of the gated block: 4-bit codes [2F, K/2], rows 16 i .. 16 i + 7 those
of gate channels 8 i .. 8 i + 7, the next eight those of the same up channels.
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
        # One token of one sequence: latency.
        dict(name="rotary_token", kind="rotary", T=1, H=32, Hkv=8, D=128, r=128, interleaved=False, far=1000, scale=1.0),
        # A prompt's queries and keys, a large model with frequencies scaled for a long context, odd length.
        dict(name="rotary_prompt_t4099", kind="rotary", T=4099, H=64, Hkv=8, D=128, r=128, interleaved=False, far=131072,
             scale=1.2),
        # Interleaved pairs in a part of each head, a head per key head, positions of a very long context.
        dict(name="rotary_part_interleaved_t1000", kind="rotary", T=1000, H=32, Hkv=32, D=128, r=32, interleaved=True,
             far=1 << 20, scale=1.0),
        # A decode step: one token for each of 64 sequences.
        dict(name="append_decode_b64", kind="append", B=64, H=64, Hkv=8, D=128, r=128, interleaved=False, q=1, len=1000),
        # Chunks of three prompts, ragged, that begin and end inside pages.
        dict(name="append_prompt_b3", kind="append", B=3, H=64, Hkv=8, D=128, r=128, interleaved=False, q=2048, len=4000),
        # One token through an 8-bit layer: the weights' way from memory.
        dict(name="gated_token_a8", kind="gated", M=1, K=4096, F=14336, bits=8, layout="decode", act="silu"),
        # The largest decode batch of a large model's 4-bit layer.
        dict(name="gated_decode_m16_a4", kind="gated", M=16, K=8192, F=28672, bits=4, layout="decode", act="silu"),
        # A chunk of a prompt, ragged, through an 8-bit layer.
        dict(name="gated_chunk_m333_a8", kind="gated", M=333, K=4096, F=14336, bits=8, layout="a8", act="gelu_tanh"),
        # A prompt of a large model's 4-bit layer.
        dict(name="gated_prompt_m4001_a4", kind="gated", M=4001, K=8192, F=28672, bits=4, layout="fp6", act="silu"),
        # The next token of one conversation.
        dict(name="sample_token_v32000", kind="sample", M=1, V=32000, half=True, mode="usual", masked=False),
        # A decode batch whose requests ask for different things, every other row under a grammar.
        dict(name="sample_b64_v131072", kind="sample", M=64, V=131072, half=True, mode="mixed", masked=True),
        # Rollouts from the whole distribution, fp32 logits, odd vocabulary.
        dict(name="sample_m256_v100003", kind="sample", M=256, V=100003, half=False, mode="whole", masked=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotary", "append", "gated", "gated", "sample", "sample"])
    if kind in ("rotary", "append"):
        Hkv = rng.choice([1, 2, 4, 8, 8, 16, 32])
        H = Hkv * rng.choice([g for g in (1, 2, 3, 4, 5, 7, 8, 16) if g * Hkv <= 64])
        D = rng.choice([64, 128, 128, 256])
        r = rng.choice([D, D, D // 2, D // 4, 2 * rng.randint(1, D // 2)])
        interleaved = rng.random() < 0.4
        if kind == "rotary":
            D, r = rng.choice([(D, r), (80, 80), (96, 48), (8 * rng.randint(5, 40), 34)])
            T = _log_int(rng, 1, max(2, min(8192, 37_000_000 // ((H + Hkv) * D))))
            return dict(kind=kind, T=T, H=H, Hkv=Hkv, D=D, r=r, interleaved=interleaved, far=_log_int(rng, 2, 1 << 20),
                        scale=rng.choice([1.0, 1.0, 1.2, 0.9]))
        q = rng.choice([1, _log_int(rng, 2, 2048)])
        B = _log_int(rng, 1, max(2, min(64, 4096 * 72 * 128 // (q * (H + 2 * Hkv) * D))))
        return dict(kind=kind, B=B, H=H, Hkv=Hkv, D=D, r=r, interleaved=interleaved, q=q, len=q + _log_int(rng, 1, 1024))
    if kind == "gated":
        K = rng.choice([2048, 4096, 5120, 8192, 128 * rng.randint(2, 64)])
        F = rng.choice([5632, 11008, 14336, 13824, 8 * rng.randint(16, 1792)])
        M = rng.choice([1, rng.randint(2, 16), _log_int(rng, 17, 2048)])
        bits = rng.choice([4, 8])
        layout = rng.choice(["packed", "decode"] if M <= 16 else ["packed", "fp6" if bits == 4 else "a8"])
        return dict(kind=kind, M=M, K=K, F=F // 8 * 8, bits=bits, layout=layout, act=rng.choice(["silu", "gelu_tanh"]))
    V = rng.choice([32000, 65536, 131072, _log_int(rng, 2, 131072)])
    M = _log_int(rng, 1, min(1024, 256 * 100003 // V))
    return dict(kind=kind, M=M, V=V, half=rng.random() < 0.5, mode=rng.choice(["usual", "mixed", "mixed", "whole"]),
                masked=rng.random() < 0.3)


# ---------------------------------------------------------------------------
# Inputs, all from the seed
# ---------------------------------------------------------------------------
def _gen(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed(1_000_003 * int(seed) + stream)
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _inv_freq(r, scaled):
    """Frequencies of base 10000; scaled: by 1/8 where a turn is longer than 8192 positions, by none where it is
    shorter than 2048, and between the two in proportion to the turns."""
    f = [10000.0 ** (-2.0 * i / r) for i in range(r // 2)]
    if scaled:
        for i, x in enumerate(f):
            s = min(1.0, max(0.0, (8192 * x / (2 * math.pi) - 1) / 3))
            f[i] = x * (s + (1 - s) / 8)
    return torch.tensor(f, dtype=torch.float64, device="cuda")


def _heads(g, T, H, Hkv, D):
    """Queries, keys and values of T tokens: views of one projection's rows; channels of different spread, an
    outlier channel in each head of the keys and the values."""
    x = _randn(g, T, H + 2 * Hkv, D) * (0.2 + 1.8 * torch.rand((H + 2 * Hkv, D), generator=g, device="cuda"))
    x[:, H:, int(torch.randint(0, D, (1,), generator=g, device="cuda"))] *= 8
    return x.half().split([H, Hkv, Hkv], dim=1)


def _rotary_inputs(case, seed):
    g = _gen(seed, 1)
    q, k, _ = _heads(g, case["T"], case["H"], case["Hkv"], case["D"])
    # Positions that run on from one in the context, as a chunk's do.
    start = int(torch.randint(0, max(1, case["far"] - case["T"]), (1,), generator=g, device="cuda"))
    positions = torch.arange(start, start + case["T"], dtype=torch.int32, device="cuda")
    return q, k, positions, _inv_freq(case["r"], case["scale"] != 1.0)


def _sizes(case):
    """New tokens and lengths (with them) of the case's sequences, ragged, the first as large as the case says."""
    rng = random.Random("%(B)d %(q)d %(len)d" % case)
    q, n = case["q"], case["len"]
    counts = [q] + [rng.randint((q + 2) // 3, q) for _ in range(case["B"] - 1)]
    return counts, [n] + [max(c, rng.randint((n + 3) // 4, n)) for c in counts[1:]]


def _scale_of(absmax):
    """2^e, the smallest with absmax <= 448 * 2^e and e >= LOWEST, of an fp32 absmax."""
    m, e = torch.frexp(absmax)                  # absmax = m * 2^e, 1/2 <= m < 1; 448 = 7/8 * 2^9
    e = torch.where(m <= TOP / 512, e - 9, e - 8)
    e = torch.where(absmax > 0, e, LOWEST).clamp(min=LOWEST)
    return ((e + 127) << 23).int().view(torch.float32)


def _append_inputs(case, seed):
    """Plan, rows, and a cache that holds what stands before the new tokens (the last page is the plain form's)."""
    B, n, Hkv, D = case["B"], case["len"], case["Hkv"], case["D"]
    counts, lengths = (torch.tensor(x) for x in _sizes(case))
    cu = torch.zeros(B + 1, dtype=torch.int64)
    cu[1:] = counts.cumsum(0)
    width = (n + PAGE - 1) // PAGE
    pages = B * width
    order = torch.Generator()
    order.manual_seed(int(seed) * 7 + 3)
    table = torch.randperm(pages, generator=order).reshape(B, width)
    table = torch.where(torch.arange(width) < ((lengths + PAGE - 1) // PAGE)[:, None], table, -1)
    g = _gen(seed, 2)
    q, k, v = _heads(g, int(cu[-1]), case["H"], Hkv, D)
    whole = []
    for _ in range(2):
        x = _randn(g, pages + 1, Hkv, PAGE, D).half()
        s = _scale_of(x.abs().amax((2, 3)).float())
        whole += [(x / s[:, :, None, None]).to(torch.float8_e4m3fn), s]
    whole = [whole[0], whole[2].view(torch.uint8).transpose(2, 3).contiguous().view(torch.float8_e4m3fn), whole[1],
             whole[3]]
    return dict(q=q, k=k, v=v, cu=cu.int().cuda(), lengths=lengths.int().cuda(), table=table.int().cuda(), pages=pages,
                whole=whole, cache=[x[:-1] for x in whole], f=_inv_freq(case["r"], True))


def _gated_inputs(case, seed):
    """Activation codes of rotated rows, as bytes, their scales, weight codes packed two a byte, their scales."""
    g = _gen(seed, 3)
    M, K, F, bits = case["M"], case["K"], case["F"], case["bits"]
    top = 7 if bits == 4 else 127
    codes = torch.round(_randn(g, M, K) * (top / 3.5)).clamp(-top, top).to(torch.int8)
    a_scales = (3.5 / top) * (0.5 + torch.rand((M,), generator=g, device="cuda"))
    w = torch.empty((2 * F, K // 2), dtype=torch.uint8, device="cuda")
    for rows in w.split(4096):
        c = torch.round(_randn(g, rows.shape[0], K) * 2).clamp(-7, 7).to(torch.int8).view(torch.uint8) & 15
        rows.copy_(c[:, ::2] | c[:, 1::2] << 4)
    w_scales = (K ** -0.5 / 2) * (0.5 + torch.rand((2 * F,), generator=g, device="cuda"))
    return codes, a_scales, w, w_scales


# What the rows of a batch ask for: temperature, top_k, top_p, min_p.
ASKED = {
    "usual": [(0.7, 50, 0.9, 0.0)],
    "whole": [(1.0, 0, 1.0, 0.0)],
    "mixed": [(0.8, 0, 0.95, 0.0), (0.0, 0, 1.0, 0.0), (1.0, 40, 1.0, 0.0), (1.0, 0, 1.0, 0.05), (0.6, 1000, 0.9, 0.01),
              (1.0, 0, 1.0, 0.0), (1.3, 200, 0.99, 0.0), (1.0, 0, 0.5, 0.0)],
}


def _sample_inputs(case, seed):
    g = _gen(seed, 4)
    M, V = case["M"], case["V"]
    x = 3 * _randn(g, M, V)
    # A few tokens stand out in each row, in some rows by far.
    likely = torch.randint(0, V, (M, 8), generator=g, device="cuda")
    x.scatter_add_(1, likely, 14 * torch.rand((M, 8), generator=g, device="cuda"))
    if case["masked"]:   # a grammar leaves a tenth of the tokens in every other row, and nothing in every 16th
        x[::2].masked_fill_(torch.rand((V,), generator=g, device="cuda") < 0.9, -math.inf)
        x[15::16] = -math.inf
    asked = ASKED[case["mode"]]
    t, k, p, m = (torch.tensor([asked[i % len(asked)][j] for i in range(M)], device="cuda",
                               dtype=torch.int32 if j == 1 else torch.float32) for j in range(4))
    return (x.half() if case["half"] else x), torch.rand((M,), generator=g, device="cuda"), t, k, p, m


def prepare(case, seed):
    kind = case["kind"]
    if kind == "rotary":
        q, k, positions, f = _rotary_inputs(case, seed)
        return dict(case=case, q=q, k=k, positions=positions, f=f)
    if kind == "append":
        return dict(case=case, **_append_inputs(case, seed))
    if kind == "sample":
        x, u, t, k, p, m = _sample_inputs(case, seed)
        return dict(case=case, x=x, u=u, t=t, k=k, p=p, m=m)
    codes, a_scales, w, w_scales = _gated_inputs(case, seed)
    if case["bits"] == 4:
        c = codes.view(torch.uint8) & 15
        codes = c[:, ::2] | c[:, 1::2] << 4
    if own:   # the layout that a program keeps its weights in, and that the quantizer writes
        import paper_2606_12487_amd as dptq
        layout = case["layout"]
        if layout != "packed":
            w = dptq.prepack_weights(w, {"fp6": dptq.WEIGHTS_FP6, "a8": dptq.WEIGHTS_A8_ORDER,
                                         "decode": dptq.WEIGHTS_DECODE}[layout])
        if layout == "a8":
            w = w.view(2 * case["F"], -1)
        if layout == "fp6":
            codes = dptq.pack_fp6(codes)
    return dict(case=case, codes=codes, a_scales=a_scales, w=w, w_scales=w_scales)


# ---------------------------------------------------------------------------
# The framework's calls
# ---------------------------------------------------------------------------
def _run_own(s):
    import paper_2606_12487_amd as dptq
    case = s["case"]
    kind = case["kind"]
    if kind == "rotary":
        return dptq.rotary(s["q"], s["k"], s["positions"], s["f"], interleaved=case["interleaved"], scale=case["scale"])
    if kind == "append":
        cache = dptq.KV8Cache(*s["cache"])
        q = dptq.rotary_kv8_append(s["q"], s["k"], s["v"], s["cu"], s["lengths"], s["table"], cache, s["f"],
                                   interleaved=case["interleaved"], max_new=case["q"])
        return [q] + s["cache"]
    if kind == "sample":
        return dptq.sample_tokens(s["x"], s["u"], temperature=s["t"], top_k=s["k"], top_p=s["p"], min_p=s["m"])
    act, layout = case["act"], case["layout"]
    if layout == "fp6":
        return dptq.qlinear_gated_fp6(s["codes"], s["a_scales"], s["w"], s["w_scales"], case["M"], case["K"], case["F"],
                                      activation=act)
    if layout == "a8":
        return dptq.qlinear_gated_a8(s["codes"], s["a_scales"], s["w"], s["w_scales"], activation=act)
    if layout == "decode":
        return dptq.qlinear_gated_decode_native(s["codes"], s["a_scales"], case["bits"], s["w"], s["w_scales"],
                                                activation=act)
    return dptq.qlinear_gated(s["codes"], s["a_scales"], case["bits"], s["w"], s["w_scales"], activation=act)


# ---------------------------------------------------------------------------
# The plain forms: elementary operations
# ---------------------------------------------------------------------------
def _plain_rotate(x, cos, sin, r, interleaved):
    """x [T, heads, D] in 32 bits, cos and sin [T, r/2]."""
    cos, sin = cos[:, None], sin[:, None]
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if interleaved else (x[..., :r // 2], x[..., r // 2:r])
    y = x.clone()
    if interleaved:
        y[..., 0:r:2] = a * cos - b * sin
        y[..., 1:r:2] = a * sin + b * cos
    else:
        y[..., :r // 2] = a * cos - b * sin
        y[..., r // 2:r] = a * sin + b * cos
    return y.half()


def _plain_rotary(s):
    case = s["case"]
    angles = s["positions"].double()[:, None] * s["f"]
    cos, sin = ((f(angles) * case["scale"]).float() for f in (torch.cos, torch.sin))
    return tuple(_plain_rotate(s[x].float(), cos, sin, case["r"], case["interleaved"]) for x in "qk")


def _plain_append(s):
    case = s["case"]
    cu, lengths = s["cu"].long(), s["lengths"].long()
    T = s["q"].shape[0]
    t = torch.arange(T, device="cuda")
    b = torch.searchsorted(cu[1:].contiguous(), t, right=True)
    start = lengths - (cu[1:] - cu[:-1])
    angles = (start[b] + t - cu[:-1][b]).double()[:, None] * s["f"]
    cos, sin = torch.cos(angles).float(), torch.sin(angles).float()
    q, k = (_plain_rotate(s[x].float(), cos, sin, case["r"], case["interleaved"]) for x in "qk")
    # Pages that the new tokens touch, the spare one where there is none; their slots and the rows of new ones.
    n = (case["q"] + PAGE - 2) // PAGE + 1
    block = start[:, None] // PAGE + torch.arange(n, device="cuda")
    there = block * PAGE < lengths[:, None]
    flat = torch.where(there, torch.gather(s["table"].long(), 1, block.clamp(max=s["table"].shape[1] - 1)),
                       s["pages"]).reshape(-1)
    pos = block[:, :, None] * PAGE + torch.arange(PAGE, device="cuda")
    start = start[:, None, None]
    new = (pos >= start) & (pos < lengths[:, None, None]) & there[:, :, None]
    row = torch.where(new, cu[:-1][:, None, None] + pos - start, 0)
    fresh = pos[:, :, 0] >= start[:, :, 0]     # a page whose first slot is written now
    old = (pos < start)[:, :, None, :, None]
    k_pages, v_pages, k_scales, v_scales = s["whole"]
    for x, codes, scales, transposed in ((k, k_pages, k_scales, False), (s["v"], v_pages, v_scales, True)):
        x = torch.where(new[:, :, :, None, None], x[row].float(), 0.0).transpose(2, 3)       # [B, n, Hkv, 64, D]
        had = torch.where(fresh[:, :, None], 0.0, scales[flat].reshape(fresh.shape + (-1,)))
        step = torch.maximum(_scale_of(x.abs().amax((3, 4))), had)
        c = codes.view(torch.uint8)[flat].view(torch.float8_e4m3fn).float()
        c = (c.transpose(2, 3) if transposed else c).reshape(x.shape)
        kept = torch.where(fresh[:, :, None, None, None], 0.0, c)     # a new page begins with zeros
        kept = torch.where(old, c * (had / step)[..., None, None], kept)
        c = torch.where(new[:, :, None, :, None], x / step[..., None, None], kept)
        c = torch.where(there[:, :, None, None, None], c, 0.0).flatten(0, 1)
        c = (c.transpose(2, 3) if transposed else c).to(torch.float8_e4m3fn)
        codes.view(torch.uint8)[flat] = c.view(torch.uint8)
        scales[flat] = torch.where(there[:, :, None], step, 1.0).flatten(0, 1)
    return [q] + s["cache"]


def _unpack(c):
    """4-bit codes, two a byte, as signed bytes."""
    return torch.stack((c << 4, c & 0xF0), dim=-1).flatten(-2).view(torch.int8) >> 4


def _plain_gated(s):
    case = s["case"]
    F = case["F"]
    a = (_unpack(s["codes"]) if case["bits"] == 4 else s["codes"]).float()
    z = (a @ _unpack(s["w"]).float().t()) * s["a_scales"][:, None] * s["w_scales"]   # sums of integers below 2^24
    g, u = z.view(-1, F // 8, 2, 8).unbind(2)
    t = g if case["act"] == "silu" else (2 * math.sqrt(2 / math.pi)) * (g + 0.044715 * g * g * g)
    return (g / (1 + torch.exp(-t)) * u).reshape(-1, F).half()


def _plain_sample(s):
    greedy = s["t"] == 0
    t = torch.where(greedy, 1.0, s["t"]).double()[:, None]
    values, ids = torch.sort(s["x"], dim=1, descending=True, stable=True)
    top = values[:, :1].double()
    w = torch.exp((values.double() - torch.where(top > -math.inf, top, 0.0)) / t)
    V = w.shape[1]
    k = torch.where(greedy, 1, torch.where(s["k"] > 0, s["k"], V))[:, None]
    w = torch.where(torch.arange(V, device="cuda") < k, w, 0.0)
    before = torch.cumsum(w, 1) - w
    limit = torch.where(s["p"] < 1, s["p"], math.inf).double()[:, None] * w.sum(1, keepdim=True)
    w2 = torch.where((before < limit) & (w >= s["m"].double()[:, None]), w, 0.0)
    w2[:, :1] = w[:, :1]
    sums = torch.cumsum(w2, 1)
    total = sums[:, -1:]
    # The first token whose running sum is above u * total; of the kept ones where rounding leaves none.
    at = (sums <= s["u"].double()[:, None] * total).sum(1, keepdim=True)
    at = torch.minimum(at, (w2 > 0).sum(1, keepdim=True) - 1).clamp(min=0)
    none = top[:, 0] == -math.inf
    tokens = torch.where(none, -1, torch.gather(ids, 1, at)[:, 0])
    return tokens, torch.where(none, 0.0, torch.gather(w2, 1, at)[:, 0] / total[:, 0]).float()


def run(state):
    if own:
        return _run_own(state)
    kind = state["case"]["kind"]
    if kind == "rotary":
        return _plain_rotary(state)
    if kind == "append":
        return _plain_append(state)
    if kind == "gated":
        return _plain_gated(state)
    return _plain_sample(state)


# ---------------------------------------------------------------------------
# Work: each input read once, each output written once
# ---------------------------------------------------------------------------
def work(case):
    kind = case["kind"]
    if kind == "gated":
        M, K, F, bits = case["M"], case["K"], case["F"], case["bits"]
        return {"bytes": F * K + 8 * F + M * (K * bits // 8 + 4 + 2 * F), "flops": 4 * M * F * K}
    if kind == "sample":
        M, V = case["M"], case["V"]
        return {"bytes": M * (V * (2 if case["half"] else 4) + 32), "flops": 4 * M * V}
    H, Hkv, D, r = case["H"], case["Hkv"], case["D"], case["r"]
    if kind == "rotary":
        T = case["T"]
        return {"bytes": T * ((H + Hkv) * D * 4 + 4) + 4 * r, "flops": 3 * T * (H + Hkv) * r}
    counts, lengths = _sizes(case)
    T = sum(counts)
    blocks = sum((n - 1) // PAGE - (n - q) // PAGE + 1 for q, n in zip(counts, lengths))
    return {"bytes": T * (H * D * 4 + 2 * Hkv * D * 3) + blocks * (4 + 16 * Hkv) + 8 * case["B"] + 4 * r,
            "flops": T * (3 * (H + Hkv) * r + 4 * Hkv * D)}


# ---------------------------------------------------------------------------
# The same values in 64 bits
# ---------------------------------------------------------------------------
def _turned(x, angles, r, interleaved, scale):
    """Rows [T, heads, D] in 64 bits, as products of complex numbers."""
    x = x.double()
    pairs = x[..., :r].unflatten(-1, (r // 2, 2) if interleaved else (2, r // 2))
    pairs = pairs if interleaved else pairs.transpose(-1, -2)
    z = torch.view_as_complex(pairs.contiguous()) * torch.polar(torch.full_like(angles, scale), angles)[:, None]
    pairs = torch.view_as_real(z)
    return torch.cat(((pairs if interleaved else pairs.transpose(-1, -2)).flatten(-2), x[..., r:]), -1)


def _exact_rotary(case, seed):
    q, k, positions, f = _rotary_inputs(case, seed)
    angles = torch.outer(positions.double(), f)
    return tuple(_turned(x, angles, case["r"], case["interleaved"], case["scale"]) for x in (q, k))


def _pow2(e):
    return ((e + 1023) << 52).view(torch.float64)


def _e4m3(x):
    """x in 64 bits, |x| <= 448, to the nearest e4m3 value, half to even: steps of 2^(e - 3), at least 2^-9."""
    step = _pow2(torch.frexp(x)[1].long().sub(4).clamp(min=-9))
    return torch.round(x / step) * step


def _exact_append(case, seed):
    s = _append_inputs(case, seed)
    cu, lengths, table = s["cu"].tolist(), s["lengths"].tolist(), s["table"].tolist()
    p = torch.cat([torch.arange(n - (cu[b + 1] - cu[b]), n, device="cuda") for b, n in enumerate(lengths)])
    angles = torch.outer(p.double(), s["f"])
    q, k = (_turned(s[x], angles, case["r"], case["interleaved"], 1.0) for x in "qk")
    outs = [c.double() for c in s["cache"]]
    # The cache holds the codes of the keys as fp16 rows.
    for c, scales, x, transposed in ((outs[0], outs[2], k.half(), False), (outs[1], outs[3], s["v"], True)):
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
    return [q] + outs


def _exact_gated(case, seed):
    codes, a_scales, w, w_scales = _gated_inputs(case, seed)
    K, F = case["K"], case["F"]
    a, a_scales, w_scales = codes.double(), a_scales.double()[:, None], w_scales.double()
    outs = []
    for i in range(0, 2 * F, 4096):     # 4096 rows: 2048 gate channels and the same up channels
        rows = w[i:i + 4096]
        c = torch.empty((rows.shape[0], K), dtype=torch.float64, device="cuda")
        c[:, ::2], c[:, 1::2] = rows & 15, rows >> 4
        c = torch.where(c > 7, c - 16, c)
        y = (a @ c.t()) * a_scales * w_scales[i:i + 4096]
        y = y.view(len(a), -1, 16)
        g, u = y[..., :8], y[..., 8:]
        h = g * torch.sigmoid(g) if case["act"] == "silu" else \
            0.5 * g * (1 + torch.tanh(math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)))
        outs.append((h * u).flatten(1))
    return torch.cat(outs, 1)


def _exact_sample(case, seed):
    x, us, ts, ks, ps, ms = _sample_inputs(case, seed)
    tokens, probs = [], []
    for row, u, t, k, p, m in zip(x, us.tolist(), ts.tolist(), ks.tolist(), ps.tolist(), ms.tolist()):
        if not bool((row > -math.inf).any()):
            tokens.append(-1)
            probs.append(0.0)
            continue
        if t == 0:
            tokens.append(int((row == row.max()).nonzero()[0]))
            probs.append(1.0)
            continue
        order = torch.argsort(row, descending=True, stable=True)
        if k > 0:
            order = order[:k]
        z = row[order].double()
        w = torch.exp((z - z[0]) / t)
        sums = torch.cumsum(w, 0)
        n = len(w)
        if p < 1:
            n = max(1, 1 + int((sums[:-1] < p * sums[-1]).sum()))
        n = min(n, max(1, int((w >= m).sum())), int((w > 0).sum()))
        i = min(int((sums[:n] <= u * sums[n - 1]).sum()), n - 1)
        tokens.append(int(order[i]))
        probs.append(float(w[i] / sums[n - 1]))
    return torch.tensor(tokens, device="cuda"), torch.tensor(probs, dtype=torch.float64, device="cuda")


def exact(case, seed):
    return {"rotary": _exact_rotary, "append": _exact_append, "gated": _exact_gated,
            "sample": _exact_sample}[case["kind"]](case, seed)
