"""Frequencies stretched for long contexts (rotary_inv_freq): the ramp by index, at lengths whose ramp ends behind the
last pair too (no GPU needed)."""

import math

import pytest

torch = pytest.importorskip("torch")
dptq = pytest.importorskip("paper_2606_12487_amd")


@pytest.mark.parametrize("length", [512, 4096, 8192, 32768, 65536, 131072, 1 << 20, 1 << 30])
@pytest.mark.parametrize("r,base,low,high", [(128, 10000.0, 1.0, 32.0), (64, 10000.0, 1.0, 32.0), (128, 500000.0, 1.0, 4.0),
                                             (32, 100.0, 2.0, 8.0)])
def test_ramp_by_index(r, base, low, high, length):
    n, factor = r // 2, 8.0

    def turns(i):   # of pair i over the length, the pairs behind the last one too
        return length * base ** (-i / n) / (2 * math.pi)

    # The last whole i with high turns or more, the first with low or fewer, from 0 to r - 1.
    first = max((i for i in range(r) if turns(i) >= high), default=0)
    last = min((i for i in range(r) if turns(i) <= low), default=r - 1)
    got = dptq.rotary_inv_freq(r, base=base, factor=factor, original_length=length, low_turns=low, high_turns=high,
                               ramp="index", device="cpu").tolist()
    for i, x in enumerate(got):
        kept = 1.0 if i <= first else max((last - i) / (last - first), 0.0)
        # A dozen roundings of 2^-53 of the frequency.
        assert x == pytest.approx(base ** (-i / n) * (kept + (1 - kept) / factor), rel=2.0 ** -49), (i, first, last)
