"""The layer over a paged cache: append, attention and heads in one call, step after step as a serving program makes them, against
the fp64 oracle's forward of the whole sequences.

Tolerances: the library's 1e-5 in fp32 and 2e-2 in bf16 (relative L2).  In bf16 the rows of a call differ from the oracle by the
roundings of query, key and value latents, head queries, a probability (long steps), head outputs, merged latents and outputs, and of
the two head-mixed cores: nine or ten independent ones of 2^-8 / sqrt(3) in the mean square at most, 7.1e-3 together."""
import numpy as np
import pytest
import torch

from oracle import tucker_oracle as orc
from paper_2603_30033_amd import binding as ta
from paper_2603_30033_amd import workloads as wl
from paper_2603_30033_amd.device import Layer, to_device, to_host

pytestmark = pytest.mark.gpu

TOL = {"f32": 1e-5, "bf16": 2e-2}
tiny = wl.WORKLOADS["tiny_f32"]
CASES = {
    "f32": wl.scaled(tiny, seed=41),
    "bf16": wl.scaled(tiny, dtype="bf16", seed=42),
    "gpt2": wl.scaled(wl.WORKLOADS["gpt2_small"], seed=43),
    "unequal": wl.scaled(tiny, dtype="bf16", d_model=264, n_heads=5, r1=3, r2=40, r3=48, rt1=2, rt2=72, rt3=32, seed=44),
    "unequal_f32": wl.scaled(tiny, d_model=264, n_heads=5, r1=3, r2=40, r3=48, rt1=2, rt2=72, rt3=100, seed=45),
    "wide": wl.scaled(tiny, dtype="bf16", d_model=512, n_heads=32, r2=128, r3=128, seed=46),
    "wide_shared": wl.scaled(tiny, dtype="bf16", d_model=512, n_heads=32, r2=128, r3=128, shared_kv=True, seed=47),
    "shared_f32": wl.scaled(tiny, shared_kv=True, seed=48),
    "no_rope": wl.scaled(tiny, dtype="bf16", rope_base=None, seed=49),
}


class Server:
    """Sequences in one pool: pages are handed out in a random order, rows of nobody hold NaN."""

    def __init__(self, w, layer, B, page, pages, seed=0):
        self.layer, self.page, self.B = layer, page, B
        self.free = list(np.random.default_rng(seed).permutation(pages))
        rt3 = w.ranks_post()[2]
        dt = layer.weights["C"].dtype
        self.K = torch.full((pages, page, w.r3), float("nan"), dtype=dt, device="cuda")
        self.V = None if w.shared_kv else torch.full((pages, page, rt3), float("nan"), dtype=dt, device="cuda")
        self.pools = ta.tucker_attn_pages.of(self.K, self.V)
        self.tables = [[] for _ in range(B)]
        self.rows = [0] * B

    def batch(self, new, padding=0):
        for b, n in enumerate(new):
            self.rows[b] += n
            while len(self.tables[b]) * self.page < self.rows[b]:
                self.tables[b].append(int(self.free.pop()))
        width = max(map(len, self.tables))
        table = torch.tensor([t + [-1] * (width - len(t)) for t in self.tables], dtype=torch.int32)
        starts = torch.tensor([0] + list(np.cumsum(new)), dtype=torch.int32)
        return ta.tucker_attn_batch.of(starts.cuda(), torch.tensor(self.rows, dtype=torch.int32).cuda(), table.cuda(),
                                       tokens=sum(new) + padding, max_new=max(new), max_len=max(self.rows))

    def step(self, X, new, padding=0, **prefix):
        """X: per sequence all its tokens; the next new[b] of them go through the layer."""
        first = list(self.rows)
        batch = self.batch(new, padding)
        parts = [X[b][first[b]:first[b] + n] for b, n in enumerate(new)]
        rows = torch.cat(parts + [torch.full_like(X[0][:1], float("nan")).expand(padding, -1)]).contiguous()
        Y = self.layer.forward_paged(rows, self.pools, batch, **prefix)
        torch.cuda.synchronize()
        return np.split(to_host(Y)[:sum(new)], np.cumsum(new)[:-1])

    def cached(self, b):
        n = torch.arange(self.rows[b])
        at = (torch.tensor(self.tables[b])[n // self.page], n % self.page)
        return to_host(self.K[at]), None if self.V is None else to_host(self.V[at])


def inputs(w, B, N):
    w = wl.scaled(w, B=B, N=N)
    inp = wl.make_inputs(w)
    wts = wl.weights_of(inp)
    if w.shared_kv:
        wts = dict(wts, Ut3=wts["U3"])
    return w, inp, wts


def oracle(w, X, wts, rows=None):
    return orc.per_head_forward(X[None], wts, w.d_head, w.causal, w.rope_base, rows=rows)[0]


def check(y, ref, dtype, what):
    assert np.all(np.isfinite(y)), what
    err = orc.relative_l2(y, ref)
    assert err <= TOL[dtype], f"{what}: relative L2 {err:.3e}"


@pytest.mark.parametrize("page", [16, 7, 128])
@pytest.mark.parametrize("case", sorted(CASES))
def test_prompts_in_pieces_then_single_tokens(case, page):
    w, inp, wts = inputs(CASES[case], B=4, N=180)
    lengths = [180, 40, 3, 97]
    steps = [[130, 39, 0, 1], [47, 0, 1, 95], [1, 1, 1, 1], [2, 0, 1, 0]]     # whole prompts, pieces, decode, proposed tokens
    with Layer(w, inp, max_positions=200) as layer:
        s = Server(w, layer, 4, page, pages=sum(-(-n // page) for n in lengths) + 3)
        X = [to_device(inp["X"][b, :n], w.dtype) for b, n in enumerate(lengths)]
        out = [[] for _ in lengths]
        for new in steps:
            for b, y in enumerate(s.step(X, new)):
                out[b].append(y)
        for b, n in enumerate(lengths):
            assert s.rows[b] == n
            check(np.concatenate(out[b]), oracle(w, inp["X"][b, :n], wts), w.dtype, f"sequence {b}")
            K, V = s.cached(b)
            Kr, Vr = orc.latent_kv(inp["X"][b:b + 1, :n], wts, None if w.shared_kv else w.rope_base)
            check(K, Kr[0], w.dtype, f"cached keys of sequence {b}")
            if V is not None:
                check(V, Vr[0], w.dtype, f"cached values of sequence {b}")
        taken = sum(map(len, s.tables)) * page - sum(lengths)
        left = torch.isnan(s.K.float()).all(-1).sum().item() - len(s.free) * page
        assert left == taken                                      # rows of nobody were not written


@pytest.mark.parametrize("case", ["f32", "bf16", "wide", "wide_shared", "unequal"])
@pytest.mark.parametrize("prefix,page", [(64, 16), (70, 16), (5, 32)])
def test_a_common_prefix(case, prefix, page):
    B, own = 3, [40, 1, 17]
    w, inp, wts = inputs(CASES[case], B=B, N=prefix + 40)
    inp["X"][1:, :prefix] = inp["X"][0, :prefix]
    with Layer(w, inp, max_positions=prefix + 40) as layer:
        X = [to_device(inp["X"][b], w.dtype) for b in range(B)]
        s = Server(w, layer, B, page, pages=60)
        head = Server(w, layer, 1, page, pages=60)
        head.K, head.V, head.pools, head.free = s.K, s.V, s.pools, s.free          # the same pool
        head.step(X[:1], [prefix])
        table = torch.tensor(head.tables[0], dtype=torch.int32).cuda()
        # sequences begin behind the prefix: its whole pages are not in their tables, the rows of a part of one are copied
        for b in range(B):
            s.tables[b] = [-1] * (prefix // page)
            s.rows[b] = prefix
            if prefix % page:
                last = int(s.free.pop())
                s.tables[b].append(last)
                for pool in (s.K, s.V):
                    if pool is not None:
                        pool[last] = pool[head.tables[0][-1]]
        out = [[] for _ in range(B)]
        for new in [[n - (n > 1) for n in own], [1, 0, 1]]:
            for b, y in enumerate(s.step(X, new, prefix_table=table, prefix_len=prefix)):
                out[b].append(y)
        for b, n in enumerate(own):
            rows = list(range(prefix, prefix + n))
            check(np.concatenate(out[b]), oracle(w, inp["X"][b, :prefix + n], wts, rows), w.dtype, f"sequence {b}")


@pytest.mark.parametrize("case", ["gpt2", "llama"])
def test_long_prompts_in_pieces(case):
    # thousands of tokens a step: the product kernels' large tiles, keys dealt to many workgroups
    w = CASES["gpt2"] if case == "gpt2" else wl.scaled(wl.WORKLOADS["llama7b_n4096"], seed=51)
    w, inp, wts = inputs(w, B=2, N=4100)
    rows = [0, 1, 1500, 2047, 2048, 4097, 4099]
    with Layer(w, inp, max_positions=4100) as layer:
        s = Server(w, layer, 2, 64, pages=140)
        X = [to_device(inp["X"][b], w.dtype) for b in range(2)]
        out = [s.step(X, new) for new in ([2048, 1000], [2051, 3000], [1, 100])]
    for b in range(2):
        y = np.concatenate([o[b] for o in out])
        check(y[rows], oracle(w, inp["X"][b], wts, rows), w.dtype, f"sequence {b}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_tokens_that_see_their_whole_sequence(dtype):
    w, inp, wts = inputs(wl.scaled(tiny, dtype=dtype, causal=False, rope_base=None, seed=52), B=3, N=70)
    lengths = [70, 1, 33]
    with Layer(w, inp, max_positions=70) as layer:
        s = Server(w, layer, 3, 16, pages=12)
        out = s.step([to_device(inp["X"][b], dtype) for b in range(3)], lengths)
    for b, n in enumerate(lengths):
        check(out[b], oracle(w, inp["X"][b, :n], wts), dtype, f"sequence {b}")


def test_padding_rows_and_prepared_weights_change_nothing():
    w, inp, _ = inputs(CASES["bf16"], B=2, N=60)
    with Layer(w, inp, max_positions=60) as layer:
        X = [to_device(inp["X"][b], w.dtype) for b in range(2)]
        out = []
        for padding, prepared in ((0, False), (9, False), (0, True)):
            if prepared:
                layer.freeze_weights()
            s = Server(w, layer, 2, 16, pages=9)
            out.append([np.concatenate(s.step(X, new, padding)) for new in ([50, 20], [1, 1])])
        ta.tucker_attn_profile_enable(layer.ctx, True)
        s.step(X, [1, 1])
        names = [n for n, _ in ta.tucker_attn_profile_read(layer.ctx)]
        ta.tucker_attn_profile_enable(layer.ctx, False)
    for other in out[1:]:
        for a, b in zip(out[0], other):
            assert np.array_equal(a, b)
    assert names == ["factor_projection", "head_queries", "paged_append", "paged_attention", "latent_merge", "output_projection"]


def test_captured_steps_serve_other_lengths_and_pages():
    w, inp, wts = inputs(CASES["bf16"], B=3, N=80)
    with Layer(w, inp, max_positions=80) as layer:
        s = Server(w, layer, 3, 16, pages=20)
        X = [to_device(inp["X"][b], w.dtype) for b in range(3)]
        s.step(X, [30, 5, 75])
        starts = torch.arange(4, dtype=torch.int32, device="cuda")
        lens, table = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.full((3, 5), -1, dtype=torch.int32, device="cuda")
        batch = ta.tucker_attn_batch.of(starts, lens, table, tokens=3, max_new=1, max_len=80)
        x = torch.zeros_like(X[0][:3])
        y = torch.zeros_like(x)
        layer.forward_paged(x, s.pools, batch, Y=y)               # (lengths of zero: nothing is stored)
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            layer.forward_paged(x, s.pools, batch, Y=y)
        for _ in range(4):
            first = list(s.rows)
            s.batch([1, 1, 1])                                    # hands out pages
            x.copy_(torch.stack([X[b][first[b]] for b in range(3)]))
            lens.copy_(torch.tensor(s.rows, dtype=torch.int32))
            for b, t in enumerate(s.tables):
                table[b, :len(t)] = torch.tensor(t, dtype=torch.int32)
            graph.replay()
            torch.cuda.synchronize()
            got = to_host(y)
            eager = to_host(layer.forward_paged(x, s.pools, batch))
            assert np.array_equal(got, eager)
            for b in range(3):
                check(got[b], oracle(w, inp["X"][b, :s.rows[b]], wts, [s.rows[b] - 1])[0], w.dtype, f"sequence {b}")


def test_equals_the_contiguous_cache():
    # the pages of one sequence in order are a contiguous cache: decode on it and the call over pages agree
    w, inp, _ = inputs(CASES["gpt2"], B=2, N=65)
    with Layer(w, inp, max_positions=80) as layer:
        X = to_device(inp["X"], w.dtype)
        Kc = torch.zeros((2, 80, w.r3), dtype=X.dtype, device="cuda")
        Vc = torch.zeros_like(Kc)
        layer.forward(X[:, :64].contiguous(), Kc=Kc, Vc=Vc)
        pools = ta.tucker_attn_pages.of(Kc.clone().view(10, 16, w.r3), Vc.clone().view(10, 16, w.r3))
        i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
        batch = ta.tucker_attn_batch.of(i32([0, 1, 2]), i32([65, 65]), i32([[0, 1, 2, 3, 4], [5, 6, 7, 8, 9]]), tokens=2, max_new=1, max_len=65)
        last = X[:, 64].contiguous()
        y = to_host(layer.forward_paged(last, pools, batch))
        check(y, to_host(layer.decode(last, Kc, Vc, [65, 65])), w.dtype, "against decode")


def test_profiled_calls_name_their_own_kernels():
    w, inp, _ = inputs(CASES["bf16"], B=2, N=64)
    with Layer(w, inp, max_positions=64) as layer:
        X = to_device(inp["X"], w.dtype)
        ta.tucker_attn_profile_enable(layer.ctx, True)
        layer.forward(X)
        assert "attention_kernel" in dict(ta.tucker_attn_profile_read(layer.ctx))
        s = Server(w, layer, 2, 16, pages=8)
        s.step([X[0], X[1]], [64, 3])
        names = [n for n, _ in ta.tucker_attn_profile_read(layer.ctx)]
    assert names == ["prep_weights", "factor_projection", "head_queries", "paged_append", "paged_attention", "latent_merge", "output_projection"]
