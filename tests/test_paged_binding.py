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


BF16 = torch.bfloat16


def zeros(*shape, dtype=BF16):
    return torch.zeros(*shape, dtype=dtype)


@pytest.fixture
def ctx():
    c = ta.tucker_attn_create(d_model=64, n_heads=4, d_head=16, r1=1, r2=32, r3=32, rt3=64, dtype="bf16", max_positions=8)
    yield c
    ta.tucker_attn_destroy(c)


@pytest.fixture
def pages():
    return ta.tucker_attn_pages.of(zeros(4, 16, 32), zeros(4, 16, 64))


def batch(T=2, device="cpu"):
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device=device)
    return ta.tucker_attn_batch.of(i32(3), i32(2), i32(2, 4), tokens=T, max_new=1, max_len=64)


GOOD = dict(Q=zeros(2, 4, 32), O=zeros(2, 4, 64), K=zeros(2, 32), V=zeros(2, 64), X=zeros(2, 64), Y=zeros(2, 64), lse=None, Qrot=zeros(2, 4, 32),
            workspace=torch.zeros(1 << 20, dtype=torch.uint8), prefix_table=torch.zeros(1, dtype=torch.int32))
CALLS = {
    "append": lambda c, p, b, a: ta.tucker_attn_append_paged(c, p, b, a["K"], a["V"], a["Q"], a["Qrot"]),
    "attend": lambda c, p, b, a: ta.tucker_attn_attend_paged(c, p, b, a["Q"], a["O"], a["lse"], a["workspace"]),
    "prefix": lambda c, p, b, a: ta.tucker_attn_attend_prefix(c, p, b, a["prefix_table"], 8, a["Q"], a["O"], a["lse"], a["workspace"]),
    "layer": lambda c, p, b, a: ta.tucker_attn_forward_paged(c, {}, a["X"], a["Y"], p, b, a["prefix_table"], 8, a["workspace"]),
}
BAD = [
    # fewer heads than the context's: rows would be read, or written, behind the tensor's end
    ("append", dict(Q=zeros(2, 1, 32))), ("append", dict(Qrot=zeros(2, 3, 32))), ("append", dict(Q=zeros(2, 32))), ("append", dict(Qrot=zeros(2, 4, 2, 32))),
    ("append", dict(K=zeros(2, 4, 32))), ("append", dict(K=zeros(1, 32))), ("append", dict(V=zeros(2, 32))), ("append", dict(V=zeros(2, 64, dtype=torch.float32))),
    ("attend", dict(Q=zeros(2, 1, 32))), ("attend", dict(O=zeros(2, 1, 64))), ("prefix", dict(O=zeros(2, 3, 64))), ("prefix", dict(Q=zeros(2, 8, 32))),
    # a log-sum-exp for every head, in fp32
    ("attend", dict(lse=zeros(2, dtype=torch.float32))), ("attend", dict(lse=zeros(2, 4))), ("prefix", dict(lse=zeros(2, 4, dtype=torch.float64))),
    ("prefix", dict(lse=zeros(4, 2, dtype=torch.float32).T)), ("attend", dict(lse=zeros(2, 1, dtype=torch.float32).expand(2, 4))),
    # rows of the model's width
    ("layer", dict(X=zeros(2, 32), Y=zeros(2, 32))), ("layer", dict(Y=zeros(2, 32))), ("layer", dict(X=zeros(1, 64))), ("layer", dict(X=zeros(2, 64, dtype=torch.float32))),
]


@pytest.mark.parametrize("call,bad", BAD, ids=[f"{c}-{next(iter(b))}-{i}" for i, (c, b) in enumerate(BAD)])
def test_arrays_that_are_not_the_contexts(ctx, pages, call, bad):
    with pytest.raises(ta.TuckerAttnError, match="expected|contiguous"):
        CALLS[call](ctx, pages, batch(), dict(GOOD, **bad))


@pytest.mark.parametrize("call", sorted(CALLS))
def test_pools_of_other_rows_than_the_contexts(ctx, call):
    for K, V in ((zeros(4, 16, 64), zeros(4, 16, 64)), (zeros(4, 16, 32), zeros(4, 16, 32)), (zeros(4, 16, 32).float(), zeros(4, 16, 64).float())):
        with pytest.raises(ta.TuckerAttnError, match="pages of rows"):
            CALLS[call](ctx, ta.tucker_attn_pages.of(K, V), batch(), GOOD)


@pytest.mark.parametrize("call", sorted(CALLS))
def test_handles_that_are_no_context(pages, call):
    c = ta.tucker_attn_create(d_model=64, n_heads=4, d_head=16, r1=1, r2=32, r3=32, rt3=64, dtype="bf16", max_positions=8)
    ta.tucker_attn_destroy(c)
    for bad in (c, None, 0):
        with pytest.raises(ta.TuckerAttnError, match="no context"):
            CALLS[call](bad, pages, batch(), GOOD)


@pytest.mark.parametrize("call", sorted(CALLS))
def test_host_memory(ctx, pages, call):
    with pytest.raises(ta.TuckerAttnError, match="one GPU"):
        CALLS[call](ctx, pages, batch(), GOOD)


def test_batches_on_two_devices():
    i32 = lambda *s, **kw: torch.zeros(*s, dtype=torch.int32, **kw)
    with pytest.raises(ta.TuckerAttnError, match="one device"):
        ta.tucker_attn_batch.of(i32(3), i32(2, device="meta"), i32(2, 4), tokens=2, max_new=1, max_len=64)


@pytest.mark.gpu
@pytest.mark.parametrize("call,names", [("append", ["K", "V", "Q", "Qrot"]), ("attend", ["Q", "O", "lse", "workspace"]),
                                        ("prefix", ["Q", "O", "lse", "workspace", "prefix_table"]), ("layer", ["X", "Y", "workspace", "prefix_table"])])
def test_arrays_in_host_memory_beside_a_pool_on_the_gpu(ctx, call, names):
    good = dict({k: None if v is None else v.cuda() for k, v in GOOD.items()}, lse=torch.zeros(2, 4, device="cuda"))
    pool = ta.tucker_attn_pages.of(zeros(4, 16, 32).cuda(), zeros(4, 16, 64).cuda())
    for name in names:
        with pytest.raises(ta.TuckerAttnError, match="one GPU"):
            CALLS[call](ctx, pool, batch(device="cuda"), dict(good, **{name: good[name].cpu()}))
    with pytest.raises(ta.TuckerAttnError, match="one GPU"):
        CALLS[call](ctx, pool, batch(), good)
    if call == "layer":
        with pytest.raises(ta.TuckerAttnError, match="one GPU"):
            ta.tucker_attn_forward_paged(ctx, {"C": zeros(4)}, good["X"], good["Y"], pool, batch(device="cuda"), workspace=good["workspace"])


def test_bounds_that_need_more_than_31_bits():
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)
    for bad in (dict(tokens=2 ** 32 + 2), dict(max_new=2 ** 31), dict(max_new=2 ** 32 + 1), dict(max_len=2 ** 32 + 64), dict(max_len=-1)):
        with pytest.raises(ta.TuckerAttnError, match="31 bits"):
            ta.tucker_attn_batch.of(i32(3), i32(2), i32(2, 4), **dict(dict(tokens=2, max_new=1, max_len=64), **bad))
