"""Constrained logits and token counts -- oracle (test infrastructure only), float64.

The text of row i is the request's counted tokens, its pending token and the drafts on
the way to row i.  For token v with n occurrences there, in the prompt or not:
  z += its bias entries;  seen: z = z / r if z > 0 else z r;  z -= f n;  n > 0: z -= p;
  -inf where the mask excludes v.
The greedy token is the lowest id among the largest allowed logits, a NaN being none of
them; -1 where there is none.
"""
from __future__ import annotations

from typing import Optional, Sequence

import numpy as np

from .verify import tree_path


def row_tokens(last: int, drafts: Sequence[int], parents: Optional[Sequence[int]], i: int):
    toks = [last] + list(drafts)
    path = range(i + 1) if parents is None else tree_path(parents, i)
    return [toks[j] for j in path]


def constrain(z, counts, prompt, text, r=1.0, f=0.0, p=0.0, bias=(), allowed=None) -> np.ndarray:
    """z [V]; counts [V] counted occurrences; prompt bool [V]; text: the row's own tokens;
    bias: (id, value) entries; allowed bool [V] or None."""
    z = np.array(z, dtype=np.float64)
    n = np.array(counts, dtype=np.int64)
    for t in text:
        if 0 <= t < z.size:
            n[t] += 1
    for t, by in bias:
        if 0 <= t < z.size:
            z[t] += by
    seen = (n > 0) | prompt
    with np.errstate(invalid="ignore"):
        z = np.where(seen, np.where(z > 0, z / r, z * r), z)
        z = z - np.where(n > 0, f * n + p, 0.0)
    return z if allowed is None else np.where(allowed, z, -np.inf)


def greedy(z: np.ndarray, allowed=None) -> int:
    ok = ~np.isnan(z) if allowed is None else ~np.isnan(z) & allowed
    return int(np.flatnonzero(ok & (z == z[ok].max()))[0]) if ok.any() else -1


def begin(table: np.ndarray, seq: int, prompt: Sequence[int]) -> None:
    """table uint16 [S, V]: bit 15 the prompt, the rest the counted occurrences."""
    table[seq] = 0
    for t in prompt:
        if 0 <= t < table.shape[1]:
            table[seq, t] = 0x8000


def add(table: np.ndarray, seq: int, tokens: Sequence[int]) -> None:
    for t in tokens:
        if 0 <= t < table.shape[1]:
            c = int(table[seq, t])
            table[seq, t] = (c & 0x8000) | min((c & 0x7FFF) + 1, 0x7FFF)
