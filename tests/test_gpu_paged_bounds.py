"""Batches whose bounds are looser than they need be: the same results, bit for bit where the same kernels run."""
import pytest
import torch

from paged_reference import Batch
from paper_2603_30033_amd import binding as ta
from test_gpu_paged import DT, Context, appended, attend, check, check_appended, on_gpu

pytestmark = pytest.mark.gpu

LOOSE = [2 ** 26, 2 ** 27, 130150525, 2 ** 31 - 1]                # times 32 or 33 heads: 2^31, 2^32, 29 more than 2^32, ..


@pytest.mark.parametrize("max_new", LOOSE)
@pytest.mark.parametrize("prefix", [0, 300])
@pytest.mark.parametrize("dtype,heads,r", [("bf16", 32, 128), ("bf16", 33, 96), ("f32", 32, 32)])
@pytest.mark.parametrize("new,rows", [([40, 0, 9, 1], [1700, 310, 900, 1333]), ([1, 1, 1], [3000, 301, 1200])])
def test_any_bound_of_new_tokens(new, rows, dtype, heads, r, prefix, max_new):
    b = Batch(new, rows, 16, r, r, heads, DT[dtype], prefix=prefix, seed=71, padding=2)
    with Context(heads, r, r, dtype) as c:
        exact = attend(c, b, *on_gpu(b, max_new=b.T))
        loose = attend(c, b, *on_gpu(b, max_new=max_new))
        check(c, b, *loose)
        for x, y in zip(exact, loose):
            assert torch.equal(x.nan_to_num(7.0), y.nan_to_num(7.0))
        if not prefix:
            K = torch.randn(b.T, r).to(b.dtype).cuda()
            check_appended(b, appended(c, b, K, K, b.Q, max_new=max_new), K, K, b.Q)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("prefix", [0, 300])
@pytest.mark.parametrize("max_new,max_len", [(1, 400), (1, 2000), (60, 400), (60, 2000)])
def test_a_step_without_a_token(max_new, max_len, prefix, dtype):
    # as a captured step meets it when all its sequences have ended: all rows are padding
    b = Batch([0, 0, 0], [700, 310, 0], 16, 64, 64, 12, DT[dtype], prefix=0, seed=72, padding=5, table_extra=90)
    b.prefix, b.prefix_table = prefix, b.table[0, :-(-prefix // 16)].clone()
    with Context(12, 64, 64, dtype) as c:
        pages, batch = on_gpu(b, max_new=max_new, max_len=max_len)
        O, L = attend(c, b, pages, batch)
        assert torch.isnan(O.float()).all() and torch.isnan(L).all()
        K = torch.randn(b.T, 64).to(b.dtype).cuda()
        got, _, R = appended(c, b, K, K, b.Q, max_new=max_new, max_len=max_len)
        assert torch.equal(got.nan_to_num(7.0), b.K.nan_to_num(7.0)) and torch.isnan(R.float()).all()
