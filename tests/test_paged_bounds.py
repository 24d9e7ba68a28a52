"""Bounds of a paged batch that are looser than they need be, or as large as their type allows: the host's part (no GPU)."""
import pytest

from paper_2603_30033_amd import binding as ta
from test_paged_refusals import batch, ctx  # noqa: F401  (ctx: a fixture)

I32 = 2 ** 31 - 1


@pytest.mark.parametrize("prefix", [0, 64])
@pytest.mark.parametrize("max_new", [17, 2 ** 27, 2 ** 29, 1610612737, I32])
def test_more_new_tokens_than_there_are_tokens_is_the_bound_of_all_tokens(ctx, max_new, prefix):  # noqa: F811
    for T in (1, 2, 8, 16):
        size = lambda n: ta.tucker_attn_attend_workspace_bytes(ctx, batch(T=T, max_new=n, max_pages=64, max_len=1024), prefix)
        layer = lambda n: ta.tucker_attn_forward_paged_workspace_bytes(ctx, batch(T=T, max_new=n, max_pages=64, max_len=1024), prefix)
        assert size(max_new) == size(T) > 0
        assert layer(max_new) == layer(T) > 0
