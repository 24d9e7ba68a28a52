"""What the paged entry points refuse on the host, before anything is enqueued (no GPU: the contexts have no rotation table)."""
import ctypes as C

import pytest

from paper_2603_30033_amd import binding as ta


@pytest.fixture
def ctx():
    c = ta.tucker_attn_create(d_model=64, n_heads=4, d_head=16, r1=1, r2=32, r3=32, rt3=64, dtype="bf16", max_positions=8)
    yield c
    ta.tucker_attn_destroy(c)


def pages(**kw):
    base = dict(K=256, V=256, k_stride=0, v_stride=0, n_pages=10, page_size=16)
    base.update(kw)
    return ta.tucker_attn_pages(*[base[n] for n, _ in ta.tucker_attn_pages._fields_])


def batch(**kw):
    base = dict(q_start=256, kv_len=256, page_table=256, B=2, T=2, max_pages=4, max_new=1, max_len=64)
    base.update(kw)
    return ta.tucker_attn_batch(*[base[n] for n, _ in ta.tucker_attn_batch._fields_])


BAD_POOLS = [dict(K=None), dict(V=None), dict(K=264), dict(V=264), dict(n_pages=0), dict(page_size=0), dict(page_size=8),
             dict(k_stride=511), dict(k_stride=516), dict(v_stride=1023), dict(v_stride=-1)]
BAD_BATCHES = [dict(q_start=None), dict(kv_len=None), dict(page_table=None), dict(B=0), dict(T=0), dict(max_pages=0), dict(max_new=0),
               dict(max_len=0), dict(max_len=65)]
CALLS = {
    "append": lambda lib, c, p, b: lib.tucker_attn_append_paged(c, p, b, 256, 32, 256, 64, 256, 256, 1, None),
    "attend": lambda lib, c, p, b: lib.tucker_attn_attend_paged(c, p, b, 256, 256, 256, 256, 1 << 40, None),
    "prefix": lambda lib, c, p, b: lib.tucker_attn_attend_prefix(c, p, b, 256, 8, 256, 256, 256, 256, 1 << 40, None),
}


@pytest.mark.parametrize("call", sorted(CALLS))
def test_pools_and_batches(call, ctx):
    lib = ta.load_library()
    run = CALLS[call]
    for bad in BAD_POOLS:
        assert run(lib, ctx, C.byref(pages(**bad)), C.byref(batch())) == -1, bad
    for bad in BAD_BATCHES:
        assert run(lib, ctx, C.byref(pages()), C.byref(batch(**bad))) == -1, bad
    assert run(lib, ctx, None, C.byref(batch())) == -1
    assert run(lib, ctx, C.byref(pages()), None) == -1
    assert run(lib, None, C.byref(pages()), C.byref(batch())) == -1
    assert run(lib, ctx, C.byref(pages()), C.byref(batch(T=1 << 29))) == -2          # (token, head) rows beyond 31 bits


@pytest.mark.parametrize("call", sorted(CALLS))
def test_rows_that_are_no_multiple_of_16_bytes_and_positions_beyond_the_table(call):
    lib = ta.load_library()
    c = ta.tucker_attn_create(d_model=64, n_heads=4, d_head=16, r1=1, r2=32, r3=36, rt3=64, dtype="bf16", max_positions=8)
    try:
        assert CALLS[call](lib, c, C.byref(pages()), C.byref(batch())) == -2
    finally:
        ta.tucker_attn_destroy(c)
    c = ta.tucker_attn_create(d_model=64, n_heads=4, d_head=16, r1=1, r2=32, r3=32, rt3=32, dtype="bf16", max_positions=8, shared_kv=True)
    try:
        assert CALLS[call](lib, c, C.byref(pages()), C.byref(batch())) == -1         # a shared latent has no value pool
    finally:
        ta.tucker_attn_destroy(c)


def test_arguments_of_append(ctx):
    lib = ta.load_library()
    p, b = C.byref(pages()), C.byref(batch())
    call = lambda *a: lib.tucker_attn_append_paged(ctx, p, b, *a, None)
    for bad in [(None, 32, 256, 64, 256, 256, 1), (256, 32, None, 64, 256, 256, 1), (256, 31, 256, 64, 256, 256, 1),
                (256, 32, 256, 63, 256, 256, 1), (256, 32, 256, 64, 256, None, 1), (256, 32, 256, 64, None, 256, 1),
                (256, 32, 256, 64, 256, 256, 2), (256, 32, 256, 64, 256, 256, 0), (257, 32, 256, 64, 256, 256, 1)]:
        assert call(*bad) == -1, bad


def test_arguments_of_attend(ctx):
    lib = ta.load_library()
    p, b = C.byref(pages()), C.byref(batch(max_len=64))
    attend = lambda *a: lib.tucker_attn_attend_paged(ctx, p, b, *a, None)
    for bad in [(None, 256, 256, 256, 1 << 40), (256, None, 256, 256, 1 << 40), (264, 256, 256, 256, 1 << 40), (256, 264, 256, 256, 1 << 40),
                (256, 256, 258, 256, 1 << 40), (256, 256, 256, 257, 1 << 40)]:
        assert attend(*bad) == -1, bad
    prefix = lambda *a: lib.tucker_attn_attend_prefix(ctx, p, b, *a, None)
    need = ta.tucker_attn_attend_workspace_bytes(ctx, batch(), 8)
    assert need > 0 and need % 256 == 0
    assert prefix(None, 8, 256, 256, 256, 256, 1 << 40) == -1
    assert prefix(256, -1, 256, 256, 256, 256, 1 << 40) == -1
    assert prefix(256, 65, 256, 256, 256, 256, 1 << 40) == -1
    assert prefix(256, 8, 256, 256, 256, None, 1 << 40) == -1
    assert prefix(256, 8, 256, 256, 256, 256, need - 1) == -3


def test_workspace_sizes(ctx):
    size = lambda prefix=0, **kw: ta.tucker_attn_attend_workspace_bytes(ctx, batch(**kw), prefix)
    assert size(B=0) == 0 and size(T=0) == 0 and size(-1) == 0 and size(65) == 0
    assert size(8) > 0
    # the arrays are not looked at
    assert size(8, q_start=None, kv_len=None, page_table=None) == size(8)


def test_the_binding_checks_shapes_and_types():
    torch = pytest.importorskip("torch")
    K = torch.zeros(4, 16, 32, dtype=torch.bfloat16)
    p = ta.tucker_attn_pages.of(K, torch.zeros(4, 16, 64, dtype=torch.bfloat16))
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)
    b = ta.tucker_attn_batch.of(i32(3), i32(2), i32(2, 4), tokens=2, max_new=1, max_len=64)
    for bad in [lambda: ta.tucker_attn_pages.of(K[:, :, ::2]), lambda: ta.tucker_attn_pages.of(K[0]), lambda: ta.tucker_attn_pages.of(K, K[:2]),
                lambda: ta.tucker_attn_pages.of(K, K.float()), lambda: ta.tucker_attn_pages.of(K[:, :8, :16]),
                lambda: ta.tucker_attn_batch.of(i32(2), i32(2), i32(2, 4), tokens=2, max_new=1, max_len=64),
                lambda: ta.tucker_attn_batch.of(i32(3), i32(2), i32(3, 4), tokens=2, max_new=1, max_len=64),
                lambda: ta.tucker_attn_batch.of(i32(3).long(), i32(2), i32(2, 4), tokens=2, max_new=1, max_len=64),
                lambda: ta.tucker_attn_batch.of(i32(3), i32(2), i32(2, 8)[:, ::2], tokens=2, max_new=1, max_len=64)]:
        with pytest.raises(ta.TuckerAttnError):
            bad()
    Q, O = torch.zeros(2, 4, 32, dtype=torch.bfloat16), torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    for q, o in [(Q[:1], O), (Q, O[:, :, :32]), (Q.float(), O), (Q, O.float()), (Q.transpose(0, 1).contiguous().transpose(0, 1)[:2, :2], O)]:
        with pytest.raises(ta.TuckerAttnError):
            ta.tucker_attn_attend_paged(None, p, b, q, o)
    with pytest.raises(ta.TuckerAttnError):
        ta.tucker_attn_attend_prefix(None, p, b, i32(1), 17, Q, O)
    with pytest.raises(ta.TuckerAttnError):
        ta.tucker_attn_append_paged(None, p, b, Q[:, 0], O[:, 0, :32])


def test_arguments_of_the_layer(ctx):
    lib = ta.load_library()
    w = C.byref(ta.tucker_attn_weights(*[256] * 8))
    p, b = C.byref(pages()), C.byref(batch())
    need = ta.tucker_attn_forward_paged_workspace_bytes(ctx, batch(), 8)
    assert need > ta.tucker_attn_attend_workspace_bytes(ctx, batch(), 8)
    run = lambda w=w, x=256, y=256, p=p, b=b, table=256, prefix=8, ws=256, size=need, c=ctx: lib.tucker_attn_forward_paged(
        c, w, x, y, p, b, table, prefix, ws, size, None)
    for bad in [dict(w=None), dict(w=C.byref(ta.tucker_attn_weights(*[256] * 7, None))), dict(x=None), dict(y=None), dict(table=None),
                dict(prefix=-1), dict(prefix=65), dict(ws=None), dict(ws=264), dict(c=None), dict(p=None), dict(b=None)]:
        assert run(**bad) == -1, bad
    for bad in BAD_POOLS:
        assert run(p=C.byref(pages(**bad))) == -1, bad
    for bad in BAD_BATCHES:
        assert run(b=C.byref(batch(**bad))) == -1, bad
    assert run(size=need - 1) == -3
    assert run(b=C.byref(batch(T=65535 * 32 + 1)), size=1 << 60) == -2
    assert ta.tucker_attn_forward_paged_workspace_bytes(ctx, batch(T=65535 * 32 + 1)) == 0
    assert ta.tucker_attn_forward_paged_workspace_bytes(ctx, batch(B=0)) == 0
    assert ta.tucker_attn_forward_paged_workspace_bytes(ctx, batch(), -1) == 0
