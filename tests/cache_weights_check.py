"""Weights of cached keys against their sums in 64 bits, where a NaN is a difference as any other."""
from __future__ import annotations

import torch

import cache_steps_reference as steps


def close(got, want, tol):
    """Fails at the first place where got is not within tol of want, or is no number."""
    ok = (got - want).abs() <= tol
    if not bool(ok.all()):
        i = int((~ok).nonzero()[0])
        raise AssertionError(f"{int((~ok).sum())} of {ok.numel()} differ, the first at {i}: {float(got[i])} for "
                             f"{float(want[i])}, allowed {float(tol[i])}")


def weights(w, sums, before, table, start, lens):
    """Weights w [pages, heads, page_tokens] of all sequences with tokens: `sums` of cache_steps_reference.attend, and
    `before` (None: zeros) of the keys that were there.

    Tolerance: that of the sums whose l is one of the scores that become weights (every kernel's), with 2^-15 of
    the sum for the additions of up to 2^14 rows in chains of 2^9, 2^-23 for those of what was there, and what is
    below fp32.  Returns which weights belong to the sequences."""
    used = torch.zeros(w.shape, dtype=torch.bool)
    for (s, h), (total, _, near) in sums.items():
        L, n = lens[s], start[s + 1] - start[s]
        old = torch.zeros(L, dtype=torch.float64)
        if before is not None:
            old = steps.weights_of(before, table[s], L, h).double()
            old[max(L - n, 0):] = 0
        want = old + total
        close(steps.weights_of(w, table[s], L, h).double(), want, near + 2.0 ** -15 * total + 2.0 ** -23 * want.abs() + 1e-30)
        t = torch.arange(L)
        used[table[s][t // w.shape[2]].long(), h, t % w.shape[2]] = True
    return used
