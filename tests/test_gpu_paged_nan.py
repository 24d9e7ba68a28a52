"""NaN and Inf that a token of a paged call sees, in queries and in keys: they reach its whole result, however the keys are dealt to
workgroups.  A softmax over a NaN score is NaN in every channel and in the log-sum-exp; a token that sees none of them keeps its bits."""
import math

import numpy as np
import pytest
import torch

from paged_reference import Batch, turned
from paper_2603_30033_amd import workloads as wl
from paper_2603_30033_amd.device import Layer, to_device, to_host
from test_gpu_forward_paged import Server, inputs
from test_gpu_paged import DT, Context, attend, on_gpu

pytestmark = pytest.mark.gpu

# (new tokens, cached rows, prefix): one workgroup a sequence; keys of a sequence dealt to several; many rows; behind a prefix
CALLS = {
    "short": ([1, 1], [300, 70], 0),
    "long": ([1, 1], [4097, 70], 0),
    "proposed": ([2, 2], [4097, 1100], 0),
    "pieces": ([40, 3], [1500, 700], 0),
    "many": ([1] * 300, [520 + i for i in range(300)], 0),
    "prefix": ([1, 2, 1], [800, 702, 1900], 700),
}
LAYERS = [("bf16", 32, 128), ("bf16", 12, 64), ("f32", 12, 64)]


def run(b, heads, r, dtype, shared=False):
    with Context(heads, r, r, dtype, shared=shared, positions=4200) as c:
        return attend(c, b, *on_gpu(b))


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("dtype,heads,r", LAYERS)
@pytest.mark.parametrize("call", sorted(CALLS))
def test_a_query_that_is_nan(call, dtype, heads, r, shared):
    new, rows, prefix = CALLS[call]
    b = Batch(new, rows, 16, r, r, heads, DT[dtype], shared=shared, prefix=prefix, seed=31, fill=0.0)
    O, L = run(b, heads, r, dtype, shared)
    b.Q[0, 3, 5] = math.nan                                       # one head of the first token
    O2, L2 = run(b, heads, r, dtype, shared)
    assert torch.isnan(O2[0, 3]).all() and torch.isnan(L2[0, 3])
    others = torch.ones(b.T, heads, dtype=torch.bool)
    others[0, 3] = False
    assert torch.equal(O[others], O2[others]) and torch.equal(L[others], L2[others])


@pytest.mark.parametrize("dtype,heads,r", LAYERS)
@pytest.mark.parametrize("call,where", [(c, w) for c in ("long", "pieces", "many", "prefix") for w in ("last", "later half", "prefix", "own")
                                        if w != "prefix" or c == "prefix"])
def test_keys_that_are_nan(call, where, dtype, heads, r):
    new, rows, prefix = CALLS[call]
    b = Batch(new, rows, 16, r, r, heads, DT[dtype], prefix=prefix, seed=32, fill=0.0)
    O, L = run(b, heads, r, dtype)
    at = b.rows_of(0)
    lo, hi = {"last": (rows[0] - 1, rows[0]), "later half": (rows[0] // 2, rows[0]), "prefix": (0, prefix), "own": (prefix, rows[0])}[where]
    b.K.view(-1, r)[at[lo:hi], 7] = math.nan
    O2, L2 = run(b, heads, r, dtype)
    t = torch.arange(b.T)
    sees = (t < new[0]) & (rows[0] - new[0] + t >= lo) if lo >= prefix else torch.ones(b.T, dtype=torch.bool)
    assert torch.isnan(O2[sees]).all() and torch.isnan(L2[sees]).all()
    assert torch.equal(O[~sees], O2[~sees]) and torch.equal(L[~sees], L2[~sees])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("prefix", [0, 64])
def test_a_token_of_the_layer_that_is_nan(prefix, dtype):
    w, inp, _ = inputs(wl.scaled(wl.WORKLOADS["tiny_f32"], dtype=dtype, seed=53), B=2, N=900)
    inp["X"][1, :prefix] = inp["X"][0, :prefix]
    inp["X"][0, 899, 0] = np.nan
    with Layer(w, inp, max_positions=900) as layer:
        X = [to_device(inp["X"][b], w.dtype) for b in range(2)]
        s = Server(w, layer, 2, 16, pages=120)
        s.step(X, [899, 899])
        kw = {}
        if prefix:
            kw = dict(prefix_table=torch.tensor(s.tables[0][:prefix // 16], dtype=torch.int32).cuda(), prefix_len=prefix)
        y = s.step(X, [1, 1], **kw)
    assert np.isnan(y[0]).all() and np.isfinite(y[1]).all()


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("dtype,heads,r", LAYERS + [("bf16", 4, 32), ("bf16", 40, 96)])
@pytest.mark.parametrize("call", sorted(CALLS))
def test_an_infinite_channel_of_a_shared_latent(call, dtype, heads, r, sign):
    # row 1 turned by one radian: both channels of its first pair become sign * inf, and scores -inf where the query's are -sign.  A key
    # of weight 0 leaves the log-sum-exp and all channels but its infinite one (0 * inf) as the sums over the other rows have them
    new, rows, prefix = CALLS[call]
    b = Batch(new, rows, 16, r, r, heads, DT[dtype], shared=True, prefix=prefix, seed=33, fill=0.0)
    b.Q[..., :2] = -sign * (b.Q[..., :2].float().abs() + 0.5).to(DT[dtype])
    at = b.rows_of(0)[1]                                          # of the prefix every sequence's, else of the first sequence
    b.K.view(-1, r)[at, 0] = -sign * 30.0                         # its weight is large: the sums without it are others
    far = run(b, heads, r, dtype, True)
    b.K.view(-1, r)[at, 0] = sign * math.inf
    O, L = run(b, heads, r, dtype, True)
    sees = torch.arange(b.T) < (b.T if prefix else new[0])
    assert torch.isfinite(L).all() and torch.isfinite(O[..., 1:]).all()
    assert not torch.isfinite(O[sees][..., 0]).any() and torch.isfinite(O[~sees]).all()
    assert torch.equal(O[~sees], far[0][~sees])
    with_zero = b.K.view(-1, r)[at].clone()
    b.K.view(-1, r)[at] = 0.0                                     # the definition: the row taken out
    K = b.K.double()
    for t in range(min(int(sees.sum()), 8)):
        s = next(i for i in range(b.B) if t < int(b.q_start[i + 1]))
        keep = [i for i in range(rows[s] - new[s] + t - int(b.q_start[s]) + 1) if i != 1]
        X = K.view(-1, r)[b.rows_of(s)[keep]]
        S = b.Q[t].double() @ turned(X, torch.tensor(keep), b.base).T / 8.0
        ref, lse = torch.softmax(S, -1) @ X, torch.logsumexp(S, -1)
        err = (O[t, :, 1:].cpu().double() - ref[:, 1:]).norm() / ref[:, 1:].norm()
        assert err <= (4e-3 if dtype == "bf16" else 1e-5)
        # a rotated key is two bf16 parts (2^-8 of 2^-8 of it is lost) of a turn in fp32, a score an fp32 sum, exponentials 2^-21
        pairs = (X[:, 0::2].abs() + X[:, 1::2].abs()).repeat_interleave(2, 1)
        size = (b.Q[t].double().abs() @ pairs.T / 8.0).amax(-1)
        tol = size * ((2.0 ** -16 if dtype == "bf16" else 0) + (r + 2) * 2.0 ** -24 + 2.0 ** -21) + 2.0 ** -21 + (len(keep) + 64) * 2.0 ** -24
        assert ((L[t].cpu().double() - lse).abs() <= tol + lse.abs() * 2.0 ** -22).all()
    assert torch.isinf(with_zero[0])


@pytest.mark.parametrize("dtype,heads,r", LAYERS)
@pytest.mark.parametrize("new,rows,prefix", [([1, 1, 1], [1, 4097, 70], 0), ([40, 1, 3], [40, 1500, 70], 0), ([1, 1, 1], [701, 1900, 750], 700)])
def test_keys_without_any_weight(new, rows, prefix, dtype, heads, r):
    # all scores -infinity: as if the tokens saw no row
    b = Batch(new, rows, 16, r, r, heads, DT[dtype], prefix=prefix, seed=34, fill=0.0)
    b.Q[..., 0] = -(b.Q[..., 0].float().abs() + 0.5).to(DT[dtype])
    others = run(b, heads, r, dtype)
    for s in range(3 if prefix else 2):
        b.K.view(-1, r)[b.rows_of(s), 0] = math.inf
    O, L = run(b, heads, r, dtype)
    n = int(b.q_start[3 if prefix else 2])
    assert (O[:n] == 0).all() and (L[:n] == -math.inf).all()
    assert torch.equal(O[n:], others[0][n:]) and torch.equal(L[n:], others[1][n:])
