"""Embedding lookup and its gradient, in 64 bits."""
import numpy as np


def forward(table, tokens, scale):
    out = np.zeros((len(tokens), table.shape[1]))
    for i, v in enumerate(tokens):
        if 0 <= v < table.shape[0]:
            out[i] = scale * table[v]
    return out


def backward(grad_out, tokens, scale, vocab):
    """(gradient of the table, sum of the magnitudes of what was added, rows added per token)."""
    total, size = np.zeros((vocab, grad_out.shape[1])), np.zeros((vocab, grad_out.shape[1]))
    count = np.zeros(vocab, dtype=np.int64)
    for i, v in enumerate(tokens):
        if 0 <= v < vocab:
            total[v] += grad_out[i]
            size[v] += np.abs(grad_out[i])
            count[v] += 1
    return scale * total, abs(scale) * size, count
