"""NaN in cached rows of a decode step reaches the sequence's output, and no other's, however its rows are dealt to workgroups."""
import numpy as np
import pytest
import torch

from paper_2603_30033_amd import workloads as wl
from paper_2603_30033_amd.device import Layer, to_device, to_host

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("b,lo,hi", [(0, 4095, 4096), (0, 2048, 4096), (0, 0, 4096), (1, 0, 128), (1, 128, 256), (1, 0, 299)])
@pytest.mark.parametrize("kv_len", [[4097, 300], [4097, 300, 4097, 1, 2000]])
@pytest.mark.parametrize("dtype,heads,r", [("bf16", 32, 128), ("bf16", 12, 64), ("f32", 12, 64)])
@pytest.mark.parametrize("shared", [False, True])
def test_cached_keys_that_are_nan(shared, dtype, heads, r, kv_len, b, lo, hi):
    w = wl.scaled(wl.WORKLOADS["tiny_f32"], dtype=dtype, d_model=256, n_heads=heads, r2=64, r3=r, shared_kv=shared, B=len(kv_len), N=1, seed=61)
    inp = wl.make_inputs(w)
    g = torch.Generator().manual_seed(5)
    dt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    K = torch.randn(len(kv_len), 4160, w.r3, generator=g).to(dt).cuda()
    V = None if shared else torch.randn(len(kv_len), 4160, w.ranks_post()[2], generator=g).to(dt).cuda()
    with Layer(w, inp, max_positions=4200) as layer:
        x = to_device(inp["X"][:, 0], dtype)
        y = to_host(layer.decode(x, K, V, kv_len))
        K[b, lo:hi] = float("nan")
        y2 = to_host(layer.decode(x, K, V, kv_len))
    assert np.isfinite(y).all()
    assert np.isnan(y2[b]).all()
    others = np.arange(len(kv_len)) != b
    assert np.array_equal(y[others], y2[others])
