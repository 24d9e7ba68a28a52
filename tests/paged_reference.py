"""The paged latent cache written from its definition in 64 bits, sequence by sequence, and seeded batches for its tests."""
import math

import torch


def turned(x, positions, base):
    """Channel pairs (2j, 2j+1) of the last axis rotated by position * base^(-2j/r); positions along the first axis."""
    r = x.shape[-1]
    a = positions.double().reshape(-1, *([1] * (x.dim() - 1))) * base ** (-torch.arange(0, r, 2, dtype=torch.float64) / r)
    x0, x1 = x.double()[..., 0::2], x.double()[..., 1::2]
    return torch.stack((x0 * a.cos() - x1 * a.sin(), x0 * a.sin() + x1 * a.cos()), -1).reshape(x.shape)


class Batch:
    """Host arrays of a step: `new` and `rows` per sequence, a pool with as many rows as they need and some pages more."""

    def __init__(self, new, rows, page, r3, rt3, heads, dtype, *, shared=False, prefix=0, base=1e4, seed=0, padding=0, fill=float("nan"),
                 table_extra=1):
        g = torch.Generator().manual_seed(seed)
        self.new, self.rows, self.page, self.prefix, self.shared, self.base = list(new), list(rows), page, prefix, shared, base
        self.r3, self.rt3, self.heads, self.dtype = r3, rt3, heads, dtype
        B, T = len(new), sum(new) + padding
        self.B, self.T = B, T

        def normal(*shape):
            return torch.randn(*shape, generator=g).to(dtype)

        whole = prefix // page
        need = [max(0, -(-n // page) - whole) for n in rows]
        common = -(-prefix // page)
        order = torch.randperm(sum(need) + common + 2, generator=g)
        self.max_pages = whole + max(need + [0]) + table_extra
        # entries that are not looked at name no page
        self.table = torch.full((B, self.max_pages), 2 ** 31 - 1, dtype=torch.int32)
        self.prefix_table = order[:common].to(torch.int32)
        at = common
        for b, n in enumerate(need):
            self.table[b, whole:whole + n] = order[at:at + n].to(torch.int32)
            at += n
        self.q_start = torch.tensor([sum(new[:b]) for b in range(B + 1)], dtype=torch.int32)
        self.kv_len = torch.tensor(rows, dtype=torch.int32)
        # rows that belong to nobody hold `fill`
        self.K = torch.full((len(order), page, r3), fill).to(dtype)
        self.V = None if shared else torch.full((len(order), page, rt3), fill).to(dtype)
        for pool, r in ((self.K, r3), (self.V, rt3)):
            if pool is None:
                continue
            flat = pool.view(-1, r)
            flat[self.prefix_rows()] = normal(prefix, r)
            for b in range(B):
                at_b = self.rows_of(b)[prefix:]
                flat[at_b] = normal(len(at_b), r)
        self.Q = normal(T, heads, r3)

    def prefix_rows(self):
        n = torch.arange(self.prefix)
        return self.prefix_table[n // self.page].long() * self.page + n % self.page

    def rows_of(self, b):
        """Pool row of every cached row of sequence b, those of the prefix in the common pages."""
        n = torch.arange(self.prefix, max(self.rows[b], self.prefix))
        own = self.table[b, n // self.page].long() * self.page + n % self.page
        return torch.cat([self.prefix_rows(), own])

    def attention(self, d_head, causal=True, rope=True):
        """O and lse in 64 bits, with sum_n p |v| and the largest scale * sum_c |q k| of a row, which error bounds need."""
        heads, T = self.heads, self.T
        O = torch.zeros(T, heads, self.rt3, dtype=torch.float64)
        lse = torch.full((T, heads), -math.inf, dtype=torch.float64)
        mass, size = torch.zeros_like(O), torch.zeros_like(lse)
        scale = 1.0 / math.sqrt(d_head)
        for b in range(self.B):
            at, q = self.rows_of(b)[:self.rows[b]], self.new[b]
            K = self.K.view(-1, self.r3)[at].double()
            V = K if self.shared else self.V.view(-1, self.rt3)[at].double()
            if self.shared and rope:
                K = turned(K, torch.arange(len(at)), self.base)
            for j in range(q):
                t = int(self.q_start[b]) + j
                n = self.rows[b] - q + j + 1 if causal else self.rows[b]
                if n <= 0:
                    continue
                Qt = self.Q[t].double()
                S = Qt @ K[:n].T * scale
                P = torch.softmax(S, -1)
                lse[t] = torch.logsumexp(S, -1)
                O[t], mass[t] = P @ V[:n], P @ V[:n].abs()
                size[t] = (Qt.abs() @ K[:n].abs().T * scale).amax(-1)
        return O, lse, mass, size


def attention_bounds(b: Batch, O, lse, mass, size, rope=True):
    """Largest errors of O and lse.  Storage rounding: u = 2^-8 (bf16) or 2^-24 of the value, half a step.  A score is a sum of r3
    products in fp32, so off by at most (r3 + 2) 2^-24 of scale * sum |q k| (bf16: also by u of it where a shared latent's key is
    rounded after its rotation, one rounding an element); an error d of the scores changes every probability by a factor within
    e^(2d), so O by 2d sum p |v|.  Probabilities: exponential and reference 2^-21 together, bf16 rounds them once more (u); sums over
    n keys (n + 64) 2^-24."""
    u = 2.0 ** -8 if b.dtype == torch.bfloat16 else 2.0 ** -24
    d = size * (b.r3 + 2) * 2.0 ** -24
    if b.shared and rope and b.dtype == torch.bfloat16:
        d = d + size * u
    sums = (max(b.rows + [0]) + 64) * 2.0 ** -24
    p = 2.0 ** -21 + sums + (u if b.dtype == torch.bfloat16 else 0.0)
    to = u * O.abs() + mass * (torch.expm1(2 * d)[..., None] + p) * (1 + u) + 1e-30
    tl = d + 2.0 ** -21 + sums + lse.nan_to_num(0.0, 0.0, 0.0).abs() * 2.0 ** -22
    return to, tl
