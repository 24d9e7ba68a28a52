"""Bounds of a paged batch that are looser than they need be, or as large as their type allows: the host's part (no GPU)."""
import ctypes as C

import pytest

from paper_2603_30033_amd import binding as ta
from test_paged_refusals import batch, ctx, pages  # noqa: F401  (ctx: a fixture)

I32 = 2 ** 31 - 1


@pytest.mark.parametrize("prefix", [0, 64])
@pytest.mark.parametrize("max_new", [17, 2 ** 27, 2 ** 29, 1610612737, I32])
def test_more_new_tokens_than_there_are_tokens_is_the_bound_of_all_tokens(ctx, max_new, prefix):  # noqa: F811
    for T in (1, 2, 8, 16):
        size = lambda n: ta.tucker_attn_attend_workspace_bytes(ctx, batch(T=T, max_new=n, max_pages=64, max_len=1024), prefix)
        layer = lambda n: ta.tucker_attn_forward_paged_workspace_bytes(ctx, batch(T=T, max_new=n, max_pages=64, max_len=1024), prefix)
        assert size(max_new) == size(T) > 0
        assert layer(max_new) == layer(T) > 0


CALLS = {
    # (all with a workspace of no bytes: what is not refused for its size is refused for want of that, and nothing is launched)
    "attend": lambda lib, c, b: lib.tucker_attn_attend_paged(c, P, b, 256, 256, 256, 256, 0, None),
    "prefix": lambda lib, c, b: lib.tucker_attn_attend_prefix(c, P, b, 256, 8, 256, 256, 256, 256, 0, None),
    "layer": lambda lib, c, b: lib.tucker_attn_forward_paged(c, W, 256, 256, P, b, 256, 8, 256, 0, None),
}
P = C.byref(pages(n_pages=1, page_size=2 ** 20))
W = C.byref(ta.tucker_attn_weights(*[256] * 8))


def status(call, c, **kw):
    return CALLS[call](ta.load_library(), c, C.byref(batch(max_pages=2 ** 12, **kw)))


@pytest.mark.parametrize("call", sorted(CALLS))
def test_sequences_whose_rows_cannot_be_counted_in_31_bits(ctx, call):  # noqa: F811
    # units of 128 rows and parts of a multiple of 64 reach past the last row
    assert status(call, ctx, max_len=2 ** 31 - 2 ** 17) == -3
    for n in (2 ** 31 - 2 ** 17 + 1, I32):
        assert status(call, ctx, max_len=n) == -2
        assert ta.tucker_attn_attend_workspace_bytes(ctx, batch(max_pages=2 ** 12, max_len=n), 8) == 0
        assert ta.load_library().tucker_attn_append_paged(ctx, P, C.byref(batch(max_pages=2 ** 12, max_len=n)), 256, 32, 256, 64, None, None, 1, None) == -2


@pytest.mark.parametrize("dtype,r3,rt3,joined,alone", [("bf16", 32, 64, 2 ** 28 - 16, 2 ** 31 - 256), ("bf16", 32, 32, 2 ** 29 - 32, 2 ** 31 - 256),
                                                       ("bf16", 128, 32, 2 ** 27 - 8, 2 ** 31 - 256), ("f32", 32, 32, 2 ** 29 - 64, 2 ** 29 - 64)])
def test_more_rows_than_a_launch_has_workgroups(dtype, r3, rt3, joined, alone):
    # 2^24 workgroups of 256 threads are refused by the device.  D/4 threads a row where a prefix's results are joined; without one
    # only blocks of 128 rows (fp32: 32), one more than the rows fill for every sequence
    c = ta.tucker_attn_create(d_model=64, n_heads=1, d_head=16, r1=1, r2=32, r3=r3, rt3=rt3, dtype=dtype, max_positions=8)
    try:
        for prefix, most in ((8, joined), (0, alone)):
            for T, ok in ((most, True), (most + 1, False), (I32, False)):
                kw = dict(T=T, max_new=T, max_pages=2 ** 12, max_len=1000, B=1)
                need = ta.tucker_attn_attend_workspace_bytes(c, batch(**kw), prefix)
                if ok and need == 0:                              # (fp32 rows of one part each: would be launched)
                    assert dtype == "f32" and prefix == 0
                    continue
                got = ta.load_library().tucker_attn_attend_prefix(c, C.byref(pages()), C.byref(batch(**kw)), 256, prefix, 256, 256, 256, 256, 0, None)
                assert got == (-3 if ok else -2) and (need > 0) == ok, (prefix, T)
    finally:
        ta.tucker_attn_destroy(c)


def test_more_tokens_than_an_append_has_workgroups():
    c = ta.tucker_attn_create(d_model=64, n_heads=1, d_head=16, r1=1, r2=32, r3=128, rt3=128, dtype="bf16", max_positions=8)
    try:
        append = lambda T: ta.load_library().tucker_attn_append_paged(c, C.byref(pages()), C.byref(batch(T=T)), 256, 128, 256, 128, 256, 256, 1, None)
        for T in (2 ** 27 - 7, 2 ** 28, I32):                     # a group of 16 lanes for the queries of a token and one for its rows
            assert append(T) == -2, T
    finally:
        ta.tucker_attn_destroy(c)


@pytest.mark.parametrize("T", [1, 8, 48, 256, 300])
def test_no_part_of_a_prefix_is_empty(T):
    # fp32: partial results of the prefix's parts and one of the sequences' own keys, D floats and two more a row
    c = ta.tucker_attn_create(d_model=64, n_heads=4, d_head=16, r1=1, r2=32, r3=64, rt3=64, dtype="f32", max_positions=8)
    try:
        for keys in list(range(100, 1000, 37)) + [4097, 5000, 16384]:
            b = batch(B=1, T=T, max_new=T, max_pages=2 ** 12, max_len=keys + 64)
            rows, n = 4 * T, ta.tucker_attn_attend_workspace_bytes(c, b, keys)
            pad = lambda x: (x + 255) // 256 * 256
            parts = next(p for p in range(1, 2000) if pad(p * rows * 256) + pad(p * rows * 8) == n) - 1
            assert any(-(-keys // each) == parts for each in range(64, keys + 64, 64)), (keys, parts)
    finally:
        ta.tucker_attn_destroy(c)
