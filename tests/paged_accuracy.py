"""Bounds for the attention over pages that are as narrow as what the kernels keep, and the attention itself in 64 bits with as many bf16
parts of a rotated key and of a probability as are asked for."""
import math

import torch

from paged_reference import Batch, turned


def rounded(x, parts):
    """x as the sum of `parts` bf16 numbers (None: as it is)."""
    if parts is None:
        return x
    total = torch.zeros_like(x)
    for _ in range(parts):
        total = total + (x - total).bfloat16().double()
    return total


def attention(b: Batch, d_head, key_parts=None, p_parts=None):
    """O (not rounded), lse, and what the bounds need: sum p |v|; of a token's keys the largest scale * sum |q k| and, twice with sums and
    then with roots of sums of squares, scale * |q| (|x0| + |x1|) over the pairs of a key before its turn."""
    T, heads = b.T, b.heads
    O, lse = torch.zeros(T, heads, b.rt3, dtype=torch.float64), torch.full((T, heads), -math.inf, dtype=torch.float64)
    mass, size, pairs, spread = torch.zeros_like(O), torch.zeros_like(lse), torch.zeros_like(lse), torch.zeros_like(lse)
    scale = 1.0 / math.sqrt(d_head)
    for s in range(b.B):
        at, q = b.rows_of(s)[:b.rows[s]], b.new[s]
        X = b.K.view(-1, b.r3)[at].double()
        V = X if b.shared else b.V.view(-1, b.rt3)[at].double()
        K = rounded(turned(X, torch.arange(len(at)), b.base), key_parts) if b.shared else X
        P2 = (X[:, 0::2].abs() + X[:, 1::2].abs()).repeat_interleave(2, 1)
        for j in range(q):
            t, n = int(b.q_start[s]) + j, b.rows[s] - q + j + 1
            if n <= 0:
                continue
            Q = b.Q[t].double()
            S = Q @ K[:n].T * scale
            p = torch.exp(S - S.amax(-1, keepdim=True))           # as the kernels have them: rounded before they are normalised
            total = p.sum(-1, keepdim=True)
            lse[t] = torch.logsumexp(S, -1)
            O[t], mass[t] = rounded(p, p_parts) @ V[:n] / total, (p / total) @ V[:n].abs()
            size[t] = (Q.abs() @ K[:n].abs().T * scale).amax(-1)
            pairs[t] = (Q.abs() @ P2[:n].T * scale).amax(-1)
            spread[t] = ((Q * Q) @ (P2[:n] * P2[:n]).T).sqrt().amax(-1) * scale
    return O, lse, mass, size, pairs, spread


def bounds(b: Batch, O, lse, mass, size, pairs, spread):
    """(largest error of an O not yet rounded, largest error of an lse, root mean square of the lse errors), bf16 storage, probabilities in
    two parts.

    A score is an fp32 sum of r3 products: (r3 + 2) 2^-24 of sum |q k|.  A shared latent's key is turned in fp32 by an angle put together
    from two (cosines and sines 2^-24 each, six roundings more: 2^-21 of |x0| + |x1|) and kept as two bf16 parts, of which the second
    is off by 2^-8 of the at most 2^-8 that the first leaves over: 2^-16 of the element, which is no more than |x0| + |x1|.  The rest: an
    exponential and its reference 2^-21, sums over n keys (n + 64) 2^-24, a logarithm 2^-22 of its result.
    Over many log-sum-exps these errors are independent: in the mean square m of them come to sqrt(m) of one, and a rounding error
    spread evenly up to its largest to that by sqrt(3)."""
    n = max(b.rows + [0])
    turn = 2.0 ** -21 + 2.0 ** -16 if b.shared else 0.0
    d = size * (b.r3 + 2) * 2.0 ** -24 + pairs * turn
    sums = 2.0 ** -21 + (n + 64) * 2.0 ** -24
    have, log = torch.isfinite(lse), lse.nan_to_num(0.0, 0.0, 0.0).abs() * 2.0 ** -22
    mean = size * math.sqrt(b.r3 + 2) * 2.0 ** -24 + spread * turn / math.sqrt(3.0) + 2.0 ** -21 + math.sqrt(n + 64) * 2.0 ** -24 + log
    return mass * (torch.expm1(2 * d)[..., None] + 2.0 ** -16 + sums) + 1e-30, d + sums + log, float(mean[have].square().mean().sqrt())


def half_step(x):
    """Half the distance between the bf16 numbers around x."""
    return torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=1e-30))) - 8)


# single tokens of up to 32 heads (the keys of a sequence in one workgroup and in several), of 33 heads and many rows of a sequence,
# behind a prefix: (new tokens, cached rows, prefix, heads, r, probabilities in two parts)
CASES = {
    "one": ([1, 1, 1], [300, 33, 500], 0, 32, 128, True),
    "split": ([1, 1], [1500, 700], 0, 12, 64, True),
    "proposed": ([2, 1], [900, 70], 0, 5, 96, True),
    "wide": ([1, 1], [700, 300], 0, 33, 128, False),
    "pieces": ([40, 3], [600, 100], 0, 12, 64, False),
    "prefix": ([1, 2, 1], [500, 410, 700], 400, 12, 64, False),
}


def batch(name, shared):
    new, rows, prefix, heads, r, _ = CASES[name]
    return Batch(new, rows, 16, r, r, heads, torch.bfloat16, shared=shared, prefix=prefix, seed=101)
