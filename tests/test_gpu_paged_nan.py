"""NaN and Inf that a token of a paged call sees, in queries and in keys: they reach its whole result, however the keys are dealt to
workgroups.  A softmax over a NaN score is NaN in every channel and in the log-sum-exp; a token that sees none of them keeps its bits."""
import math

import numpy as np
import pytest
import torch

from paged_reference import Batch
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
@pytest.mark.parametrize("where", ["last", "later half", "prefix", "own"])
@pytest.mark.parametrize("call", ["long", "pieces", "many", "prefix"])
def test_keys_that_are_nan(call, where, dtype, heads, r):
    new, rows, prefix = CALLS[call]
    b = Batch(new, rows, 16, r, r, heads, DT[dtype], prefix=prefix, seed=32, fill=0.0)
    if where == "prefix" and not prefix:
        pytest.skip("no prefix")
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
