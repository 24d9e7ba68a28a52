"""The paged latent cache on the GPU against its definition in 64 bits (tests/paged_reference.py), through the binding.

Every element of O and lse is held to the bound that attention_bounds derives from the roundings there are; over an array the
relative L2 error may reach 4e-3 in bf16 (three independent roundings -- a probability, a key where a shared latent is rotated, the
result -- of at most 2^-8 / sqrt(3) in the mean square each) and the library's 1e-5 in fp32.  Appended rows: one rounding to the
storage type of fp32 sums of two products."""
import math

import pytest
import torch

from paged_reference import Batch, attention_bounds, turned
from paper_2603_30033_amd import binding as ta

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


class Context:
    def __init__(self, heads, r3, rt3, dtype, *, shared=False, causal=True, base=1e4, d_head=64, positions=4096):
        self.d_head = d_head
        self.ctx = ta.tucker_attn_create(d_model=64, n_heads=heads, d_head=d_head, r1=1, r2=32, r3=r3, rt3=rt3, causal=causal, rope_base=base,
                                         dtype=dtype, max_positions=positions, shared_kv=shared)

    def __enter__(self):
        return self

    def __exit__(self, *e):
        ta.tucker_attn_destroy(self.ctx)


def on_gpu(b: Batch, max_new=None, max_len=None):
    K, V = b.K.cuda(), None if b.V is None else b.V.cuda()
    pages = ta.tucker_attn_pages.of(K, V)
    batch = ta.tucker_attn_batch.of(b.q_start.cuda(), b.kv_len.cuda(), b.table.cuda(), tokens=b.T, max_new=max_new or max(b.new + [1]),
                                    max_len=max_len or max(b.rows + [1]))
    return pages, batch


def attend(c, b: Batch, pages, batch, lse=True, workspace=None):
    """O and lse from NaN-filled buffers; the call with a prefix where the batch has one."""
    O = torch.full((b.T, b.heads, b.rt3), math.nan, dtype=b.dtype, device="cuda")
    L = torch.full((b.T, b.heads), math.nan, device="cuda") if lse else None
    Q = b.Q.cuda()
    n = ta.tucker_attn_attend_workspace_bytes(c.ctx, batch, b.prefix)
    ws = torch.full((max(n, 256),), 255, dtype=torch.uint8, device="cuda") if workspace is None else workspace
    if b.prefix:
        ta.tucker_attn_attend_prefix(c.ctx, pages, batch, b.prefix_table.cuda(), b.prefix, Q, O, L, ws)
    else:
        ta.tucker_attn_attend_paged(c.ctx, pages, batch, Q, O, L, ws)
    torch.cuda.synchronize()
    return O, L


def check(c, b: Batch, O, L, causal=True, rope=True):
    ref = b.attention(c.d_head, causal, rope)
    to, tl = attention_bounds(b, *ref, rope=rope)
    n = int(b.q_start[-1])
    o, l = O.cpu().double(), L.cpu().double()
    assert torch.isnan(o[n:]).all() and torch.isnan(l[n:]).all(), "rows behind the last sequence"
    o, l, r, rl = o[:n], l[:n], ref[0][:n], ref[1][:n]
    assert torch.isfinite(o).all()
    none = torch.isinf(rl)
    assert torch.equal(torch.isinf(l) & (l < 0), none) and (o[none] == 0).all()
    over = (o - r).abs() / to[:n]
    assert over.max() <= 1, f"O: {over.max():.3g} of its bound at {[int(i) for i in torch.unravel_index(over.argmax(), over.shape)]}"
    over = ((l - rl).abs() / tl[:n])[~none]
    assert over.numel() == 0 or over.max() <= 1, f"lse: {over.max():.3g} of its bound"
    rel = float((o - r).norm() / r.norm().clamp(min=1e-30))
    assert rel <= (4e-3 if b.dtype == torch.bfloat16 else 1e-5), f"relative L2 {rel:.3g}"


# new tokens and cached rows around the tiles of 32, 64 and 128 keys, sequences of no token among them
NEW = [1, 1, 0, 1, 1, 1, 1, 1, 1, 1]
ROWS = [1, 31, 40, 32, 33, 64, 127, 129, 500, 257]

SHAPES = [(12, 64, 64), (4, 32, 32), (32, 128, 128), (1, 128, 64), (33, 96, 96), (64, 64, 128), (5, 48, 32), (70, 64, 64)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,r3,rt3", SHAPES)
def test_one_new_token(heads, r3, rt3, dtype):
    b = Batch(NEW, ROWS, 16, r3, rt3, heads, DT[dtype], seed=heads + r3)
    with Context(heads, r3, rt3, dtype) as c:
        check(c, b, *attend(c, b, *on_gpu(b)))


@pytest.mark.parametrize("page", [1, 3, 7, 32, 48, 64, 100, 1024])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_page_sizes(page, dtype):
    b = Batch([1, 4, 1], [300, 97, 64], page, 64, 64, 12, DT[dtype], seed=page)
    with Context(12, 64, 64, dtype) as c:
        check(c, b, *attend(c, b, *on_gpu(b)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("heads,r3,rt3", [(12, 64, 64), (32, 128, 128), (3, 32, 32), (7, 96, 48)])
@pytest.mark.parametrize("new,rows", [([5, 2, 3], [5, 130, 64]), ([33, 0, 100, 1], [400, 17, 100, 65]), ([129], [129])])
def test_several_new_tokens(new, rows, heads, r3, rt3, causal, dtype):
    b = Batch(new, rows, 16, r3, rt3, heads, DT[dtype], seed=len(new) + heads, padding=3)
    with Context(heads, r3, rt3, dtype, causal=causal) as c:
        check(c, b, *attend(c, b, *on_gpu(b)), causal=causal)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rope", [True, False])
@pytest.mark.parametrize("heads,r", [(12, 64), (32, 128), (4, 32), (5, 96), (40, 128)])
@pytest.mark.parametrize("new,rows", [(NEW, ROWS), ([40, 3], [200, 300])])
def test_shared_latent(new, rows, heads, r, rope, dtype):
    b = Batch(new, rows, 32, r, r, heads, DT[dtype], shared=True, seed=heads)
    with Context(heads, r, r, dtype, shared=True, base=1e4 if rope else None) as c:
        check(c, b, *attend(c, b, *on_gpu(b)), rope=rope)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("prefix,page", [(1, 16), (63, 64), (64, 64), (200, 16), (777, 48), (1500, 128)])
@pytest.mark.parametrize("new,own", [([1] * 6, [1, 2, 33, 64, 129, 300]), ([1, 5, 0, 40], [7, 5, 9, 90])])
def test_common_prefix(new, own, prefix, page, shared, dtype):
    b = Batch(new, [prefix + n for n in own], page, 64, 64, 12, DT[dtype], shared=shared, prefix=prefix, seed=prefix)
    with Context(12, 64, 64, dtype, shared=shared) as c:
        check(c, b, *attend(c, b, *on_gpu(b)))


@pytest.mark.parametrize("heads,r3,rt3,B", [(32, 128, 128, 40), (3, 32, 32, 2), (64, 128, 64, 5), (20, 96, 96, 300)])
def test_common_prefix_shapes(heads, r3, rt3, B):
    new = [1 + (i % 3 == 0) for i in range(B)]
    b = Batch(new, [700 + 2 + (37 * i) % 200 for i in range(B)], 16, r3, rt3, heads, torch.bfloat16, prefix=700, seed=B, padding=1)
    with Context(heads, r3, rt3, "bf16") as c:
        check(c, b, *attend(c, b, *on_gpu(b)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_sequences_and_a_long_one(dtype):
    B = 1100 if dtype == "bf16" else 300                          # more sequences than a workgroup has threads
    rows = [1 + (i * 7) % 90 for i in range(B)]
    rows[B // 2] = 3000
    new = [1 if i % 5 else 0 for i in range(B)]
    new[B // 2] = 1
    b = Batch(new, rows, 16, 32, 32, 4, DT[dtype], seed=5)
    with Context(4, 32, 32, dtype) as c:
        check(c, b, *attend(c, b, *on_gpu(b)))


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("heads,r,B", [(32, 128, 128), (32, 128, 129), (12, 64, 140), (32, 128, 257), (3, 32, 300)])
def test_a_step_of_many_sequences_of_hundreds_of_rows(heads, r, B, shared):
    # around the number of sequences from which row blocks in place of sequences are dealt to the workgroups
    rows = [1 + (53 * i) % 700 for i in range(B)]
    b = Batch([int(i % 9 != 4) for i in range(B)], rows, 16, r, r, heads, torch.bfloat16, shared=shared, seed=B)
    with Context(heads, r, r, "bf16", shared=shared) as c:
        check(c, b, *attend(c, b, *on_gpu(b)))


@pytest.mark.parametrize("heads,r3,rt3", [(32, 128, 128), (12, 64, 32), (1, 32, 32), (70, 64, 64), (130, 32, 32)])
@pytest.mark.parametrize("causal", [True, False])
def test_whole_prompts(causal, heads, r3, rt3):
    # row blocks that see from a few keys to all of them
    new = [300, 0, 701, 40, 1]
    b = Batch(new, new, 16, r3, rt3, heads, torch.bfloat16, seed=heads, padding=3)
    with Context(heads, r3, rt3, "bf16", causal=causal) as c:
        check(c, b, *attend(c, b, *on_gpu(b)), causal=causal)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("heads,r", [(12, 64), (32, 128), (3, 32)])
@pytest.mark.parametrize("new,own", [([1, 3, 60, 0, 1], [1200, 700, 1900, 5, 1]), ([1] * 20, [1 + 90 * i for i in range(20)])])
def test_many_own_keys_behind_a_prefix(new, own, heads, r, shared, dtype):
    b = Batch(new, [70 + n for n in own], 16, r, r, heads, DT[dtype], shared=shared, prefix=70, seed=heads, padding=1)
    with Context(heads, r, r, dtype, shared=shared) as c:
        check(c, b, *attend(c, b, *on_gpu(b)))


@pytest.mark.parametrize("bad", [math.inf, math.nan])
@pytest.mark.parametrize("heads,r", [(32, 128), (12, 64)])
def test_what_a_token_behind_a_prefix_does_not_see_does_not_reach_it(heads, r, bad):
    b = Batch([4, 1, 1], [510, 480, 433], 16, r, r, heads, torch.bfloat16, prefix=433, seed=17)
    with Context(heads, r, r, "bf16") as c:
        O, L = attend(c, b, *on_gpu(b))
        at = b.rows_of(0)
        b.K.view(-1, r)[at[-1]] = bad                             # rows of the last token of the first sequence only
        b.V.view(-1, r)[at[-1]] = bad
        O2, L2 = attend(c, b, *on_gpu(b))
        others = [0, 1, 2, 4, 5]
        assert torch.equal(O[others], O2[others]) and torch.equal(L[others], L2[others])
        assert not torch.isfinite(O2[3].float()).any()


@pytest.mark.parametrize("rows", [4096, 32768])
def test_one_long_sequence(rows):
    b = Batch([1], [rows], 64, 128, 128, 32, torch.bfloat16, seed=9)
    with Context(32, 128, 128, "bf16", positions=rows) as c:
        check(c, b, *attend(c, b, *on_gpu(b)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("many", [False, True])
def test_tokens_that_see_nothing(many, dtype):
    # fewer cached rows than new tokens: the first tokens lie before the first row
    new, rows = ([3, 1, 2], [1, 0, 50]) if not many else ([40, 9, 2], [30, 0, 50])
    b = Batch(new, rows, 16, 64, 64, 12, DT[dtype], seed=3)
    with Context(12, 64, 64, dtype) as c:
        check(c, b, *attend(c, b, *on_gpu(b)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,r,new", [(4, 32, 6), (32, 128, 9), (12, 64, 40)])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_what_a_token_does_not_see_does_not_reach_it(bad, heads, r, new, dtype):
    b = Batch([new, 1], [new + 45, 70], 16, r, r, heads, DT[dtype], seed=11)
    with Context(heads, r, r, dtype) as c:
        O, L = attend(c, b, *on_gpu(b))
        at = b.rows_of(0)
        first = new - 3                                           # the last three tokens see it, the last row is theirs
        b.K.view(-1, r)[at[-2:]] = bad
        b.V.view(-1, r)[at[45 + first], 5] = bad
        O2, L2 = attend(c, b, *on_gpu(b))
        assert torch.equal(O[:first], O2[:first]) and torch.equal(L[:first], L2[:first])
        assert torch.equal(O[new:], O2[new:])
        seen = O2[first, :, 5].float()                            # the token that sees the value but not the keys
        assert (torch.isnan(seen).all() if math.isnan(bad) else (seen == bad).all())
        assert torch.isfinite(O2[first].float()).sum() == heads * (r - 1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_infinite_last_value_is_the_only_key(dtype):
    b = Batch([1, 1], [1, 33], 16, 64, 64, 12, DT[dtype], seed=2)
    b.V.view(-1, 64)[b.rows_of(0)[0], 3] = math.inf
    with Context(12, 64, 64, dtype) as c:
        O, _ = attend(c, b, *on_gpu(b))
        assert (O[0, :, 3] == math.inf).all() and torch.isfinite(O[1].float()).all() and torch.isfinite(O[0, :, 4:].float()).all()


@pytest.mark.parametrize("scale", [1e-20, 30.0])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_score_sizes(scale, dtype):
    b = Batch([1, 4, 30], [300, 97, 120], 16, 64, 64, 12, DT[dtype], seed=7)
    b.Q = (b.Q.float() * scale).to(DT[dtype])
    with Context(12, 64, 64, dtype) as c:
        check(c, b, *attend(c, b, *on_gpu(b)))


def test_pool_larger_than_32_bit_offsets():
    b = Batch([1, 3], [300, 200], 64, 128, 128, 8, torch.bfloat16, seed=13)
    far = 2 ** 32 // (64 * 128) + 7                               # first element of that page: beyond 2^32
    big = {}
    for name in ("K", "V"):
        pool = getattr(b, name)
        big[name] = torch.empty(far + len(pool), 64, 128, dtype=torch.bfloat16, device="cuda")
        big[name][far:] = pool.cuda()
    table = torch.where(b.table < len(b.K), b.table + far, b.table)
    pages = ta.tucker_attn_pages.of(big["K"], big["V"])
    batch = ta.tucker_attn_batch.of(b.q_start.cuda(), b.kv_len.cuda(), table.cuda(), tokens=b.T, max_new=3, max_len=300)
    with Context(8, 128, 128, "bf16") as c:
        check(c, b, *attend(c, b, pages, batch))
        rows = torch.randn(4, 128, dtype=torch.bfloat16, device="cuda")
        ta.tucker_attn_append_paged(c.ctx, pages, batch, rows, rows, rotate=False)
        at = table[1, 199 // 64].long() * 64 + 199 % 64
        assert torch.equal(big["K"].view(-1, 128)[at], rows[3]) and torch.equal(big["V"].view(-1, 128)[at], rows[3])


def test_pages_of_both_pools_in_one_allocation():
    b = Batch([1, 20], [70, 100], 16, 64, 32, 12, torch.bfloat16, seed=4)
    both = torch.full((len(b.K), 16 * (64 + 32) + 8), math.nan, dtype=torch.bfloat16, device="cuda")
    both[:, :16 * 64] = b.K.flatten(1).cuda()
    both[:, 16 * 64:16 * 96] = b.V.flatten(1).cuda()
    K, V = both[:, :16 * 64].unflatten(1, (16, 64)), both[:, 16 * 64:16 * 96].unflatten(1, (16, 32))
    pages = ta.tucker_attn_pages.of(K, V)
    with Context(12, 64, 32, "bf16") as c:
        check(c, b, *attend(c, b, pages, on_gpu(b)[1]))


def test_bounds_larger_than_the_batch_and_without_lse():
    b = Batch([1, 2], [70, 40], 16, 64, 64, 12, torch.bfloat16, seed=4, table_extra=60)
    with Context(12, 64, 64, "bf16") as c:
        pages, batch = on_gpu(b, max_new=3, max_len=1000)
        O, L = attend(c, b, pages, batch)
        check(c, b, O, L)
        O2, _ = attend(c, b, pages, batch, lse=False)
        assert torch.equal(O, O2) or (O[~torch.isnan(O)] == O2[~torch.isnan(O2)]).all()


@pytest.mark.parametrize("new,rows,prefix", [([1] * 5, [300, 1, 64, 200, 77], 0), ([1] * 5, [600, 501, 564, 700, 577], 500), ([60, 1], [200, 90], 0)])
def test_captured_and_replayed_with_other_lengths_and_pages(new, rows, prefix):
    c = Context(12, 64, 64, "bf16")
    first = Batch(new, rows, 16, 64, 64, 12, torch.bfloat16, prefix=prefix, seed=21)
    second = Batch(new, [n - (n - prefix) // 3 if n - prefix > 2 * q else n for n, q in zip(rows, new)], 16, 64, 64, 12, torch.bfloat16, prefix=prefix, seed=22)
    with c:
        n_pages, width = max(len(first.K), len(second.K)), max(first.max_pages, second.max_pages)
        pool = {k: torch.zeros(n_pages, 16, 64, dtype=torch.bfloat16, device="cuda") for k in "KV"}
        table = torch.zeros(len(new), width, dtype=torch.int32, device="cuda")
        q_start, kv_len = first.q_start.cuda(), first.kv_len.cuda()
        ptable = torch.zeros(max(len(first.prefix_table), 1), dtype=torch.int32, device="cuda")
        Q = torch.zeros_like(first.Q, device="cuda")
        O = torch.zeros(first.T, 12, 64, dtype=torch.bfloat16, device="cuda")
        L = torch.zeros(first.T, 12, device="cuda")
        pages = ta.tucker_attn_pages.of(pool["K"], pool["V"])
        batch = ta.tucker_attn_batch.of(q_start, kv_len, table, tokens=first.T, max_new=max(new), max_len=max(rows))
        ws = torch.empty(max(ta.tucker_attn_attend_workspace_bytes(c.ctx, batch, prefix), 256), dtype=torch.uint8, device="cuda")

        def load(b):
            for k in "KV":
                pool[k][:len(b.K)] = getattr(b, k).cuda()
            table[:, :b.max_pages] = b.table.cuda()
            kv_len.copy_(b.kv_len)
            ptable[:len(b.prefix_table)] = b.prefix_table.cuda()
            Q.copy_(b.Q)

        def step():
            ta.tucker_attn_attend_prefix(c.ctx, pages, batch, ptable, prefix, Q, O, L, ws)

        load(first)
        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        for b in (second, first, second):
            load(b)
            O.fill_(math.nan)
            L.fill_(math.nan)
            graph.replay()
            torch.cuda.synchronize()
            check(c, b, O, L)
            got = O.clone()
            step()                                                # eager work between the replays, with the same result
            torch.cuda.synchronize()
            assert torch.equal(got, O)


def test_on_another_stream_and_twice_alike():
    b = Batch([1] * 4, [900, 30, 257, 64], 16, 128, 128, 32, torch.bfloat16, seed=6)
    with Context(32, 128, 128, "bf16") as c:
        pages, batch = on_gpu(b)
        O, L = attend(c, b, pages, batch)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        Q, O2, L2 = b.Q.cuda(), torch.empty_like(O), torch.empty_like(L)
        ws = torch.empty(max(ta.tucker_attn_attend_workspace_bytes(c.ctx, batch), 256), dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        ta.tucker_attn_attend_paged(c.ctx, pages, batch, Q, O2, L2, ws, stream=s)
        s.synchronize()
        assert torch.equal(O, O2) and torch.equal(L, L2)


def test_numbers_that_are_no_page_read_page_0():
    # a caller's mistake: the sequence's result means nothing, the others' are right and nothing outside the pool is touched
    b = Batch([1, 1, 1], [40, 40, 70], 16, 64, 64, 12, torch.bfloat16, seed=8, fill=0.0)
    good = b.attention(64)
    table = b.table.clone()
    table[1, :3] = torch.tensor([-1, 2 ** 31 - 1, len(b.K)])
    pages, _ = on_gpu(b)
    batch = ta.tucker_attn_batch.of(b.q_start.cuda(), b.kv_len.cuda(), table.cuda(), tokens=3, max_new=1, max_len=70)
    with Context(12, 64, 64, "bf16") as c:
        O, L = attend(c, b, pages, batch)
        to, _ = attention_bounds(b, *good)
        for t in (0, 2):
            assert ((O[t].cpu().double() - good[0][t]).abs() <= to[t]).all()
        assert torch.isfinite(O[1].float()).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("prefix", [0, 70])
@pytest.mark.parametrize("starts,lens", [([0, 40, 10, 50, 50], [700, 400, 900, 33]), ([-5, 20, 90, 2 ** 31 - 1, 0], [-3, 5000, 800, 2 ** 31 - 1]),
                                         ([30, 20, 10, 0, -1], [600] * 4)])
def test_ranges_and_lengths_that_break_the_rules_end_inside_the_buffers(starts, lens, prefix, dtype):
    # a caller's mistake: results mean nothing, but the call ends, the pool stays as it is and a good call behind it is right
    b = Batch([40, 0, 9, 1], [700, 400, 900, 333], 16, 64, 64, 12, DT[dtype], prefix=prefix, seed=21)
    with Context(12, 64, 64, dtype) as c:
        pages, good = on_gpu(b)
        before = [t.clone() for t in pages.tensors if t is not None]
        bad = ta.tucker_attn_batch.of(torch.tensor(starts, dtype=torch.int32).cuda(), torch.tensor(lens, dtype=torch.int32).cuda(),
                                      torch.where(b.table < len(b.K), b.table, 0).cuda(), tokens=b.T, max_new=40, max_len=900)
        attend(c, b, pages, bad)
        assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(before, [t for t in pages.tensors if t is not None]))
        check(c, b, *attend(c, b, pages, good))


# ---- append ----------------------------------------------------------------------------------------------------------

def appended(c, b: Batch, K, V, Q, rotate=True, inplace=False, **kw):
    pages, batch = on_gpu(b, **kw)
    Qd = None if Q is None else Q.cuda()
    R = Qd if inplace or Q is None else torch.full_like(Qd, math.nan)
    ta.tucker_attn_append_paged(c.ctx, pages, batch, K, V, Qd, R, rotate=rotate)
    torch.cuda.synchronize()
    return pages.tensors[0].cpu(), None if V is None else pages.tensors[1].cpu(), None if R is None else R.cpu()


def check_appended(b: Batch, got, K, V, Q, rotate=True, rope=True, untouched=True):
    u = 2.0 ** -8 if b.dtype == torch.bfloat16 else 2.0 ** -24
    gk, gv, gq = got
    wk, wv = b.K.clone().double(), None if b.V is None else b.V.clone().double()
    slack = torch.zeros_like(wk)
    n = int(b.q_start[-1])
    for s in range(b.B):
        q, t0 = b.new[s], int(b.q_start[s])
        pos = torch.arange(b.rows[s] - q, b.rows[s])
        live = pos >= 0
        at = b.rows_of(s)[pos[live]]
        x = K.cpu().double()[t0:t0 + q][live]
        turn = rotate and rope and not b.shared
        wk.view(-1, b.r3)[at] = turned(x, pos[live], b.base) if turn else x
        if turn:                                                  # cosines in fp32, two products, one sum
            slack.view(-1, b.r3)[at] = (x[:, 0::2].abs() + x[:, 1::2].abs()).repeat_interleave(2, 1) * 2.0 ** -22
        if V is not None:
            wv.view(-1, b.rt3)[at] = V.cpu().double()[t0:t0 + q][live]
        if Q is not None:
            x = Q.double()[t0:t0 + q][live]
            want = turned(x, pos[live], b.base) if rope else x
            have = gq.double()[t0:t0 + q][live]
            tol = u * want.abs() + (x[..., 0::2].abs() + x[..., 1::2].abs()).repeat_interleave(2, -1) * 2.0 ** -22
            assert ((have - want).abs() <= tol).all()
    same = torch.isnan(wk) & torch.isnan(gk.double())
    assert (same | ((gk.double() - wk).abs() <= (u * wk.abs() if rope and rotate and not b.shared else 0) + slack)).all()
    if V is not None:
        assert ((torch.isnan(wv) & torch.isnan(gv.double())) | (gv.double() == wv)).all()
    if Q is not None:
        assert torch.isnan(gq[n:].float()).all(), "rows behind the last sequence"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,r3,rt3", SHAPES)
@pytest.mark.parametrize("new,rows,page", [(NEW, ROWS, 16), ([5, 0, 33, 1], [5, 9, 300, 64], 7), ([200], [200], 1)])
def test_append(new, rows, page, heads, r3, rt3, dtype):
    b = Batch(new, rows, page, r3, rt3, heads, DT[dtype], seed=heads, padding=2)
    g = torch.Generator().manual_seed(1)
    latent = torch.randn(b.T, r3 + rt3, generator=g).to(b.dtype).cuda()
    K, V = latent[:, :r3], latent[:, r3:]
    with Context(heads, r3, rt3, dtype) as c:
        check_appended(b, appended(c, b, K, V, b.Q), K, V, b.Q)
        check_appended(b, appended(c, b, K, V, None), K, V, None)
        check_appended(b, appended(c, b, K, V, None, rotate=False), K, V, None, rotate=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("offset", [0, 1, 3])
def test_append_rows_that_start_anywhere(offset, dtype):
    b = Batch([3, 1, 20], [40, 9, 64], 16, 48, 32, 5, DT[dtype], seed=1)
    g = torch.Generator().manual_seed(2)
    wide = torch.randn(b.T, 48 + 32 + 5, generator=g).to(b.dtype).cuda()
    K, V = wide[:, offset:offset + 48], wide[:, offset + 48:offset + 80]
    with Context(5, 48, 32, dtype) as c:
        check_appended(b, appended(c, b, K, V, b.Q), K, V, b.Q)


@pytest.mark.parametrize("rope", [True, False])
def test_append_shared_latent_and_no_rotation(rope):
    for shared in (True, False):
        b = Batch([3, 1], [40, 9], 16, 64, 64, 12, torch.bfloat16, shared=shared, seed=1)
        K = torch.randn(b.T, 64).to(b.dtype).cuda()
        V = None if shared else K + 1
        with Context(12, 64, 64, "bf16", shared=shared, base=1e4 if rope else None) as c:
            check_appended(b, appended(c, b, K, V, b.Q), K, V, b.Q, rope=rope)


def test_append_in_place_many_sequences_and_missing_pages():
    B = 2500                                                      # more batch bounds than are looked through at a time
    new = [i % 3 for i in range(B)]
    b = Batch(new, [q + (i * 11) % 40 for i, q in enumerate(new)], 16, 32, 32, 4, torch.bfloat16, seed=1)
    K = torch.randn(b.T, 32).to(b.dtype).cuda()
    with Context(4, 32, 32, "bf16") as c:
        got = appended(c, b, K, K, b.Q, inplace=True)
        check_appended(b, got, K, K, b.Q)
    b = Batch([2, 3, 1], [20, 2, 33], 16, 32, 32, 4, torch.bfloat16, seed=1)      # a token before the first row
    K = torch.randn(b.T, 32).to(b.dtype).cuda()
    with Context(4, 32, 32, "bf16") as c:
        check_appended(b, appended(c, b, K, K, b.Q), K, K, b.Q)
        for bad in (-1, len(b.K), 2 ** 31 - 1):                   # no page: its rows are stored nowhere
            lost = b.table.clone()
            lost[0, 1] = bad
            pages, _ = on_gpu(b)
            batch = ta.tucker_attn_batch.of(b.q_start.cuda(), b.kv_len.cuda(), lost.cuda(), tokens=b.T, max_new=3, max_len=33)
            ta.tucker_attn_append_paged(c.ctx, pages, batch, K, K)
            have, was = pages.tensors[0].cpu().view(-1, 32), b.K.view(-1, 32)
            at = b.rows_of(0)[18:]
            assert torch.equal(have[at], was[at])
            assert not torch.equal(have[b.rows_of(2)[32]], was[b.rows_of(2)[32]])
