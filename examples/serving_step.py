"""Serving with dptq: prompts of several lengths and then single tokens through a
small random transformer, with the norm that gives 8-bit activations, the
quantized linears, the 8-bit paged KV cache with its attention, and the answers'
log probabilities with their alternatives.

    python examples/serving_step.py          # needs an MI355X and the built library
"""

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2606_12487_amd as dptq  # noqa: E402

D, HEADS, KV_HEADS, HIDDEN, FFN, LAYERS, VOCAB = 64, 8, 2, 512, 1024, 2, 1008


class Sequences:
    """The sequences of a batch: their pages, lengths, and the step's new tokens."""

    def __init__(self, batch, most_tokens):
        width = -(-most_tokens // dptq.KV8_PAGE)
        self.table = torch.arange(batch * width, dtype=torch.int32, device="cuda").reshape(batch, width)
        self.lengths = torch.zeros(batch, dtype=torch.int32, device="cuda")
        self.caches = [dptq.kv8_cache(batch * width, KV_HEADS, D) for _ in range(LAYERS)]

    def extend(self, counts):
        """Makes room for counts[b] new tokens of each sequence; the step's row offsets and their largest count."""
        new = torch.tensor(counts, dtype=torch.int32, device="cuda")
        self.lengths += new
        cu = torch.zeros(len(counts) + 1, dtype=torch.int32, device="cuda")
        cu[1:] = new.cumsum(0)
        return cu, max(counts)


class Model:
    def __init__(self, seed=0, window=0, sinks=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)

        def linear(n, k, had_size):
            w = torch.randn((n, k), generator=g, device="cuda") * k ** -0.5
            return dptq.prepare_weights(w, had_size)

        def norm():
            return (1 + 0.1 * torch.randn(HIDDEN, generator=g, device="cuda")).half()

        self.window, self.sinks = window, sinks
        self.embedding = torch.randn((VOCAB, HIDDEN), generator=g, device="cuda").half()
        # Linears behind a norm take its codes as they are (had_size 1: nothing to undo), the others rotate.
        self.layers = [dict(norm1=norm(), qkv=linear((HEADS + 2 * KV_HEADS) * D, HIDDEN, 1),
                            out=linear(HIDDEN, HEADS * D, HEADS * D), norm2=norm(),
                            up=linear(2 * FFN, HIDDEN, 1), down=linear(HIDDEN, FFN, FFN)) for _ in range(LAYERS)]
        self.norm, self.head = norm(), linear(VOCAB, HIDDEN, 1)

    def step(self, tokens, cu, most, seqs):
        """Logits [T, VOCAB] of the new tokens, whose keys and values go into the caches."""
        h = self.embedding[tokens]
        x = None
        for layer, cache in zip(self.layers, seqs.caches):
            codes, scales, h = dptq.rms_norm_quant(h if x is None else x, layer["norm1"], 1e-5,
                                                   residual=None if x is None else h)
            qkv = dptq.qlinear(codes, scales, 8, *layer["qkv"]).unflatten(1, (HEADS + 2 * KV_HEADS, D))
            q, k, v = qkv.split([HEADS, KV_HEADS, KV_HEADS], dim=1)
            dptq.kv8_append(k, v, cu, seqs.lengths, seqs.table, cache, max_new=most)
            y, _ = dptq.kv8_attention(q, cu, seqs.lengths, seqs.table, cache, window=self.window, sinks=self.sinks,
                                      max_q=most)
            codes, scales = dptq.rotate_quant(y.flatten(1), HEADS * D, 8)
            x = dptq.qlinear(codes, scales, 8, *layer["out"])
            codes, scales, h = dptq.rms_norm_quant(x, layer["norm2"], 1e-5, residual=h, sum=h)
            gate, up = dptq.qlinear(codes, scales, 8, *layer["up"]).chunk(2, dim=1)
            y = torch.nn.functional.silu(gate) * up
            codes, scales = dptq.rotate_quant(y, FFN, 8)
            x = dptq.qlinear(codes, scales, 8, *layer["down"])
        codes, scales, _ = dptq.rms_norm_quant(x, self.norm, 1e-5, residual=h, sum=h)
        return dptq.qlinear(codes, scales, 8, *self.head)


def generate(model, prompts, new_tokens, top=5):
    """Greedy answers to the prompts (lists of token ids): per sequence its tokens, and per step the log
    probabilities, entropies and alternatives."""
    seqs = Sequences(len(prompts), max(len(p) for p in prompts) + new_tokens)
    cu, most = seqs.extend([len(p) for p in prompts])
    tokens = torch.tensor([t for p in prompts for t in p], device="cuda")
    logits = model.step(tokens, cu, most, seqs)[cu[1:].long() - 1]      # of each prompt's last token
    answers, steps = [], []
    for i in range(new_tokens):
        tokens = logits.argmax(1)
        answers.append(tokens)
        steps.append(dptq.token_logprobs(logits, tokens, top=top))
        if i + 1 < new_tokens:
            cu, most = seqs.extend([1] * len(prompts))
            logits = model.step(tokens, cu, most, seqs)
    return torch.stack(answers, 1), steps


def main():
    g = torch.Generator()
    g.manual_seed(1)
    prompts = [torch.randint(0, VOCAB, (n,), generator=g).tolist() for n in (5, 130, 61)]
    answers, steps = generate(Model(window=96, sinks=4), prompts, 8)
    for b, prompt in enumerate(prompts):
        print(f"prompt of {len(prompt)} tokens -> {answers[b].tolist()}")
        for logprob, entropy, top, ids in steps[:2]:
            print(f"  logprob {logprob[b]:.3f}, entropy {entropy[b]:.3f}, alternatives "
                  + ", ".join(f"{t}: {p:.3f}" for t, p in zip(ids[b].tolist(), top[b].tolist())))


if __name__ == "__main__":
    main()
