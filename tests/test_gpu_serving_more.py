"""Positions, the gated block and sampling in a serving step: in the example, in captured graphs, on other streams and
several at once."""

import os
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")
dptq = pytest.importorskip("paper_2606_12487_amd")

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

H, HKV, D, K, F, V, PAGES = 8, 2, 64, 512, 1024, 1008, 12


def test_drawn_answers():
    import serving_step as s
    model, prompts = s.Model(window=64, sinks=2), [[1, 2, 3], list(range(70))]
    answers, steps = s.generate(model, prompts, 5, top=8, temperature=0.9, top_k=8)
    again, _ = s.generate(model, prompts, 5, top=8, temperature=0.9, top_k=8)
    assert torch.equal(answers, again)
    for i, (_, _, _, ids) in enumerate(steps):
        assert bool((ids == answers[:, i:i + 1]).any(1).all())          # one of the eight likeliest
    others = [s.generate(model, prompts, 5, seed=seed, temperature=2.0)[0] for seed in range(3)]
    assert not all(torch.equal(others[0], o) for o in others[1:])
    greedy, _ = s.generate(model, prompts, 5)
    assert torch.equal(greedy, s.generate(model, prompts, 5, temperature=3.0, top_k=1)[0])


class Step:
    """One layer's step of a decode batch on fixed buffers, from the fused projection's rows to tokens."""

    def __init__(self, B, seed):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.qkv = torch.empty((B, H + 2 * HKV, D), dtype=torch.float16, device="cuda")
        self.h = torch.empty((B, K), dtype=torch.float16, device="cuda")
        self.uniform = torch.empty(B, device="cuda")
        self.lengths = torch.empty(B, dtype=torch.int32, device="cuda")
        self.cu = torch.arange(B + 1, dtype=torch.int32, device="cuda")
        self.table = torch.arange(B * PAGES, dtype=torch.int32, device="cuda").view(B, PAGES)
        self.cache = dptq.kv8_cache(B * PAGES, HKV, D)
        for x in self.cache[:2]:
            x.view(torch.uint8).zero_()
        self.f = dptq.rotary_inv_freq(D)
        self.norm = torch.ones(K, dtype=torch.float16, device="cuda")
        w = torch.randn((2 * F, K), generator=g, device="cuda") * K ** -0.5
        self.up = dptq.prepare_weights(dptq.gate_up_rows(*w.chunk(2)), 1)
        self.up_dec = dptq.prepack_weights(self.up[0], dptq.WEIGHTS_DECODE)
        self.head = dptq.prepare_weights(3 * torch.randn((V, F), generator=g, device="cuda") * F ** -0.5, 1)
        self.rows = dict(temperature=torch.linspace(0, 1.5, B, device="cuda"),
                         top_k=torch.arange(B, dtype=torch.int32, device="cuda") * 30,
                         top_p=torch.linspace(1.0, 0.5, B, device="cuda"), min_p=torch.zeros(B, device="cuda"))

    def fill(self, seed):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.qkv.copy_(torch.randn(self.qkv.shape, generator=g, device="cuda"))
        self.h.copy_(torch.randn(self.h.shape, generator=g, device="cuda"))
        self.uniform.copy_(torch.rand(self.uniform.shape, generator=g, device="cuda"))
        self.lengths.copy_(torch.randint(1, 64 * PAGES, self.lengths.shape, generator=g, device="cuda"))

    def run(self):
        q, k, v = self.qkv.split([H, HKV, HKV], dim=1)
        positions = self.lengths - 1
        q1, k1 = dptq.rotary(q, k, positions, self.f)
        q2 = dptq.rotary_kv8_append(q, k, v, self.cu, self.lengths, self.table, self.cache, self.f, max_new=1)
        y, lse = dptq.kv8_attention(q2, self.cu, self.lengths, self.table, self.cache, max_q=1)
        codes, scales, _ = dptq.rms_norm_quant(self.h, self.norm, 1e-5)
        a = dptq.qlinear_gated(codes, scales, 8, *self.up)
        if len(self.h) <= 16:
            b = dptq.qlinear_gated_decode_native(codes, scales, 8, self.up_dec, self.up[1])
        else:
            b = dptq.qlinear_gated_a8(codes, scales, dptq.pack_w4_a8(self.up[0]), self.up[1])
        codes, scales = dptq.rotate_quant(a, 1, 8)
        logits = dptq.qlinear(codes, scales, 8, *self.head)
        tokens, probs = dptq.sample_tokens(logits, self.uniform, **self.rows)
        wide = logits.repeat(1, 40)              # as long as rows in parts are
        more, _ = dptq.sample_tokens(wide, self.uniform, **self.rows)
        return [q1, k1, q2, y, lse, a, b, logits, tokens, probs, more]

    def caches(self):
        return [x.view(torch.uint8).clone() for x in self.cache]


def _same(got, want):
    assert len(got) == len(want)
    for i, (a, b) in enumerate(zip(got, want)):
        assert torch.equal(a.view(torch.uint8) if a.is_floating_point() else a,
                           b.view(torch.uint8) if b.is_floating_point() else b), i


@pytest.mark.parametrize("B", [3, 40])
def test_captured_step(B):
    """A graph of the step, replayed with eager work between: each replay against the eager step."""
    step, eager = Step(B, 1), Step(B, 1)
    for s in (step, eager):
        s.fill(0)
        s.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step.run()
    for x, y in zip(step.cache, eager.cache):
        x.view(torch.uint8).copy_(y.view(torch.uint8))
    for i in range(4):
        step.fill(10 + i)
        eager.fill(10 + i)
        graph.replay()
        if i % 2:
            torch.cuda.synchronize()
        want = eager.run()
        _same(outs, want)
        _same(step.caches(), eager.caches())


def test_two_graphs_and_streams_at_once():
    """Two captured steps and an eager one on three streams: their workspaces are their own."""
    steps = [Step(B, i) for i, B in enumerate((4, 20, 9))]
    graphs, outs = [], []
    for i, s in enumerate(steps):
        s.fill(i)
        s.run()
        torch.cuda.synchronize()
        if i < 2:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                outs.append(s.run())
            graphs.append(g)
    streams = [torch.cuda.Stream() for _ in steps]
    for turn in range(3):
        for i, s in enumerate(steps):
            s.fill(100 * turn + i)
        want = [[x.clone() for x in s.run()] for s in steps]      # the append's second call changes nothing
        torch.cuda.synchronize()
        for st in streams:
            st.wait_stream(torch.cuda.current_stream())
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                graphs[i].replay()
        with torch.cuda.stream(streams[2]):
            last = steps[2].run()
        torch.cuda.synchronize()
        for got, w in zip(outs + [last], want):
            _same(got, w)


def test_order_of_calls_on_a_stream_of_its_own():
    """Inputs made and outputs read on a side stream, without a synchronization in between."""
    step, side = Step(5, 3), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = []
    with torch.cuda.stream(side):
        for i in range(5):
            step.fill(i)
            got.append([x.clone() for x in step.run()])
    side.synchronize()
    other = Step(5, 3)
    for i in range(5):
        other.fill(i)
        _same(got[i], other.run())


def test_long_rows_of_many_sequences():
    """Offsets beyond 2^31: the last rows of a large batch of logits and of queries."""
    M, V2 = 17000, 131073
    x = torch.zeros((M, V2), dtype=torch.float16, device="cuda")
    assert x.numel() > 2 ** 31
    x[-1, 70001] = 20.0
    x[-2, V2 - 1] = 20.0
    tokens, probs = dptq.sample_tokens(x, torch.full((M,), 0.5, device="cuda"), top_k=1)
    assert tokens[-2:].tolist() == [V2 - 1, 70001] and int(tokens[0]) == 0 and probs.tolist()[-2:] == [1.0, 1.0]
    tokens, _ = dptq.sample_tokens(x[-2:], torch.tensor([0.5, 0.9999999], device="cuda"))
    # 1 - u of the sum, which is 1.00027 of the likely token's weight, is that of 57.9 tokens of weight exp(-20).
    assert tokens.tolist() == [V2 - 1, V2 - 1 - 57]
    del x
    T, heads = 2 ** 31 // (64 * 128) + 5, 64
    q = torch.ones((T, heads, 128), dtype=torch.float16, device="cuda")
    positions = torch.zeros(T, dtype=torch.int32, device="cuda")
    positions[-1] = 3
    f = dptq.rotary_inv_freq(128)
    out, _ = dptq.rotary(q, None, positions, f)
    assert bool((out[:-1] == 1).all())
    small, _ = dptq.rotary(q[-1:], None, positions[-1:], f)
    assert torch.equal(out[-1:], small) and not torch.equal(small, q[:1])


def test_more_tokens_than_a_launch_holds():
    """Rotary positions of 2^26 + 5 tokens of one small head, a wave each: more than 2^32 threads."""
    T, D, piece = (1 << 26) + 5, 8, 1 << 24
    q = torch.empty((T, 1, D), dtype=torch.float16, device="cuda")
    g = torch.Generator("cuda").manual_seed(3)
    for t in range(0, T, piece):
        q[t:t + piece] = torch.randn((min(piece, T - t), 1, D), device="cuda", generator=g).half()
    positions = torch.arange(T, dtype=torch.int32, device="cuda")
    f = dptq.rotary_inv_freq(D)
    out, _ = dptq.rotary(q, None, positions, f)
    for t in (0, (1 << 26) - 4100, T - 4097):
        want, _ = dptq.rotary(q[t:t + 4097], None, positions[t:t + 4097], f)
        assert torch.equal(out[t:t + 4097], want), t
    assert bool((out.view(torch.int16)[piece:] != q.view(torch.int16)[piece:]).any(-1).all())
