"""What the binding refuses of the calls over pages before their addresses go to the device (no GPU)."""
import pytest

from paper_2603_30033_amd import binding as ta

torch = pytest.importorskip("torch")


def test_pools_whose_pages_overlap():
    K = torch.zeros(4, 16, 32)
    for bad in (K[:1].expand(4, -1, -1), K.view(-1).as_strided((4, 16, 32), (256, 32, 1))):
        with pytest.raises(ta.TuckerAttnError, match="pages"):
            ta.tucker_attn_pages.of(bad)
        with pytest.raises(ta.TuckerAttnError, match="pages"):
            ta.tucker_attn_pages.of(K, bad)
    one = K[:1].expand(1, -1, -1).as_strided((1, 16, 32), (0, 32, 1))    # a single page has no distance
    assert ta.tucker_attn_pages.of(one).k_stride == 0
    apart = torch.zeros(4, 2, 16, 32)[:, 1]
    assert ta.tucker_attn_pages.of(apart).k_stride == 2 * 16 * 32
