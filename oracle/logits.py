"""Logit adjustment of a tree node (oracle; test infrastructure).

The token history of a node is the request's (prompt, then answered tokens)
plus the draft tokens on the node's root path without the root's. A token seen
in it is penalised by the repetition factor (towards -inf on both sides of 0);
tokens answered or drafted also by frequency times their count and once by
presence. Then the request's bias values are added, and tokens that the node's
mask leaves out become -inf. Everything is float64, token by token.
"""

from __future__ import annotations

import numpy as np


def path_tokens(parent, draft, n: int):
    """Draft tokens of node n and its ancestors, the root's left out."""
    out = []
    while parent[n] >= 0:
        out.append(int(draft[n]))
        n = int(parent[n])
    return out


def adjust_row(x, prompt, answered, path, repetition=1.0, presence=0.0, frequency=0.0, biases=(), allowed=None):
    """x [V] logits; prompt, answered, path: token lists; biases: (token, value)
    pairs; allowed [V] bool or None."""
    V = len(x)
    y = np.array(x, np.float64)
    count = np.zeros(V, np.int64)
    for j in list(answered) + list(path):
        if 0 <= j < V:
            count[j] += 1
    seen = count > 0
    for j in prompt:
        if 0 <= j < V:
            seen[j] = True
    for j in range(V):
        if seen[j]:
            y[j] = y[j] / repetition if y[j] > 0 else y[j] * repetition
        if count[j]:
            y[j] -= count[j] * frequency + presence
    for j, v in biases:
        if 0 <= j < V:
            y[j] += v
    if allowed is not None:
        y[~np.asarray(allowed, bool)] = -np.inf
    return y
