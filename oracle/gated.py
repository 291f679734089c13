"""The gated feed-forward block on quantized operands (oracle; test infrastructure):
exact integer accumulators, the activation and the product in float64."""

import numpy as np

from .gemm import qlinear_acc_ref

__all__ = ["gate_up_order", "gated_ref"]


def gate_up_order(F):
    """Rows of [gate; up] (2 F of them) in the order of a gated block's weights."""
    i = np.arange(2 * F)
    return np.where(i % 16 < 8, 0, F) + i // 16 * 8 + i % 8


def gated_ref(codes, a_scales, bits, w_packed, w_scales, act):
    """(y float64 [M, F], g, u) for weights in the interleaved order."""
    acc = qlinear_acc_ref(codes, bits, w_packed).astype(np.float64)
    z = acc * np.asarray(a_scales, np.float64)[:, None] * np.asarray(w_scales, np.float64)
    z = z.reshape(len(z), -1, 2, 8)
    g, u = (z[:, :, i].reshape(len(z), -1) for i in (0, 1))
    with np.errstate(over="ignore"):
        if act == "silu":
            h = g / (1 + np.exp(-g))
        else:
            h = 0.5 * g * (1 + np.tanh(np.sqrt(2 / np.pi) * (g + 0.044715 * g ** 3)))
    return h * u, g, u
