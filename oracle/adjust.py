"""Oracle of the penalties, biases and masks on a step's logits.  Test infrastructure only (see the package docstring).  fp64."""
from __future__ import annotations

from collections import Counter

import numpy as np

from .int4 import paths


def adjust_sequence(logits, tokens, n_rows, text, prompt_len, repetition=1.0, frequency=0.0, presence=0.0, bias=(), allowed=None, parents=None):
    """One sequence: logits [R, V] -> fp64 [n_rows, V].  bias: (token, value) pairs; allowed: [n_rows, V] truth values."""
    V = logits.shape[1]
    out = []
    for i, path in enumerate(paths(n_rows, parents)):
        drafts = [int(tokens[j]) for j in path if j > 0]
        made = Counter(t for t in list(map(int, text[prompt_len:])) + drafts if 0 <= t < V)
        seen = set(t for t in list(map(int, text)) + drafts if 0 <= t < V)
        x = logits[i].astype(np.float64)
        for t in seen:
            x[t] = x[t] / repetition if x[t] > 0 else x[t] * repetition
        for t, n in made.items():
            x[t] = x[t] - frequency * n - presence
        for t, b in bias:
            if 0 <= t < V:
                x[t] += b
        if allowed is not None:
            x[~allowed[i]] = -np.inf
        out.append(x)
    return np.stack(out) if out else np.zeros((0, V))
