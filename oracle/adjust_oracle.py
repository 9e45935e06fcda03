"""Rules of single requests on logits, in float64 numpy: penalties for tokens that a sequence already has, biases,
allowed-token masks, and the histories behind the penalties.  Written from the formulas, token by token."""
from __future__ import annotations

from typing import Dict, Iterable, Optional

import numpy as np


class History:
    """What one sequence has: tokens of its prompt, how often each token was generated, biases."""

    def __init__(self) -> None:
        self.prompt = set()
        self.generated: Dict[int, int] = {}
        self.bias: Dict[int, float] = {}

    def add(self, tokens: Iterable[int], in_prompt: bool, vocab: int) -> None:
        for v in tokens:
            v = int(v)
            if not 0 <= v < vocab:
                continue
            if in_prompt:
                self.prompt.add(v)
            else:
                self.generated[v] = self.generated.get(v, 0) + 1

    def set_bias(self, ids, values, vocab: int) -> None:
        for v, x in zip(ids, values):
            if 0 <= int(v) < vocab:
                self.bias[int(v)] = float(np.float32(x))

    def touched(self) -> set:
        return self.prompt | set(self.generated) | set(self.bias)


def adjusted_logits(row: np.ndarray, hist: Optional[History], repetition: float = 1.0, presence: float = 0.0,
                    frequency: float = 0.0, allowed: Optional[np.ndarray] = None) -> np.ndarray:
    """One row of logits (float64 [V]) under the rules, in their order: repetition, presence, frequency, bias, mask."""
    x = np.array(row, dtype=np.float64)
    if hist is not None:
        for v in hist.touched():
            c = hist.generated.get(v, 0)
            if v in hist.prompt or c > 0:
                x[v] = x[v] / repetition if x[v] > 0 else x[v] * repetition
            if c > 0:
                x[v] -= presence
            x[v] -= frequency * c
            x[v] += hist.bias.get(v, 0.0)
    if allowed is not None:
        x[~np.asarray(allowed, dtype=bool)] = -np.inf
    return x


def row_statistics(x: np.ndarray) -> Dict[str, float]:
    """arg-max (lowest index), lse, max-prob and entropy of softmax(x); a row that has nothing: -1, -inf, 0, 0."""
    top = x.max() if x.size else -np.inf
    if not top > -np.inf:
        return dict(argmax=-1, lse=-np.inf, maxprob=0.0, entropy=0.0)
    d = x - top
    e = np.exp(d)
    s = e.sum()
    t = np.where(e > 0, d * e, 0.0).sum() if np.isfinite(d).all() else np.sum([a * b for a, b in zip(d, e) if b > 0])
    return dict(argmax=int(np.argmax(x)), lse=float(top + np.log(s)), maxprob=float(1.0 / s), entropy=float(np.log(s) - t / s))


def pack_bits(on: np.ndarray) -> np.ndarray:
    """bool [..., V] -> int32 words [..., ceil(V / 128) * 4], token v in bit v % 32 of word v / 32."""
    v = on.shape[-1]
    words = -(-v // 128) * 4
    pad = np.zeros(on.shape[:-1] + (words * 32,), dtype=np.uint8)
    pad[..., :v] = on
    return np.packbits(pad, axis=-1, bitorder="little").view(np.uint32).view(np.int32)
