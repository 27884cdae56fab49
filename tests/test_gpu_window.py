"""Attention with a window and sinks over bf16 and block-scaled caches, of chunks, single tokens and draft trees, against the 64-bit definition.

Tolerance, element by element: the output is rounded to bf16 (2^-8 of it) and every probability before it is multiplied with its value, to
bf16 (2^-8 of sum p |v|, which the oracle returns) or, over codes, to fp16 (2^-11); scores, exponentials (one pair in a few is a cubic good to
1.2e-4) and sums are fp32, for which 5e-4 of the same sum is ample: a score of 128 products of unit-variance inputs is good to about 1e-5, with the
rounding of a query row to fp16 (2^-25 of its largest magnitude for the small elements) to less than twice that."""
import numpy as np
import pytest
import torch

from oracle import serving as S

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


@pytest.fixture(scope="module")
def E():
    from paper_2401_15077_b200 import binding, build
    build.build()
    binding.load()
    assert torch.cuda.is_available()
    return binding


def _ints(v):
    return torch.tensor(v, dtype=torch.int32)


class Case:
    """Keys and values only where some token of the call sees them: every other slot is NaN, as are the scales of blocks that nothing sees, and
    pages that hold nothing to see are not in the table."""

    def __init__(self, n, lens, hq, hkv, d=128, page=0, block=0, window=0, sinks=0, tree=False, seed=0, pad=37, spare=3, scales=(0.005, 0.015)):
        g = torch.Generator().manual_seed(seed)
        self.n, self.lens, self.page, self.block, self.tree = n, lens, page, block, tree
        self.kw = {"window": window, "sinks": sinks}
        B, need = len(n), [a + b for a, b in zip(n, lens)]
        rows = (B, max(n)) if tree else (sum(n) + spare,)
        self.q = torch.randn(*rows, hq, d, generator=g).bfloat16()
        if tree:
            self.order = torch.zeros(B, max(n), dtype=torch.int32)
            for b, m in enumerate(n):
                for i in range(m):
                    self.order[b, i] = int(torch.randint(-1, i, (1,), generator=g)) if i else -1
        else:
            self.order = _ints(np.concatenate([[0], np.cumsum(n)]).tolist())
        seen = []
        for m, L in zip(n, lens):
            at = torch.arange(L + m)
            seen.append((at >= L - window + 1) | (at < sinks) if window else torch.ones(L + m, dtype=torch.bool))
            if m == 0:
                seen[-1][:] = False
        if page:
            used = [-(-x // page) for x in need]
            order = torch.randperm(sum(used) + 2, generator=g).tolist()
            self.table = torch.full((B, max(max(used), 1) + 1), -1, dtype=torch.int32)
            for b, u in enumerate(used):
                for i in range(u):
                    if seen[b][i * page:(i + 1) * page].any():
                        self.table[b, i] = order.pop()
            shape = (sum(used) + 2, hkv, page, d)
        else:
            cap = max(need) + pad
            self.table, shape = None, (B, hkv, -(-cap // block) * block if block else cap, d)
        if block:
            self.k, self.v = (torch.full(shape, 0x7f, dtype=torch.uint8) for _ in range(2))
            blocks = (*shape[:2], shape[2] // block)
            self.ks, self.vs = (torch.full(blocks, float("nan")) for _ in range(2))
        else:
            self.k, self.v = (torch.full(shape, float("nan"), dtype=torch.bfloat16) for _ in range(2))
            self.ks = self.vs = None
        lo, hi = scales
        for b in range(B):
            slots = seen[b].nonzero().flatten()
            if page:
                first, row = self.table[b].long()[slots // page], slots % page
            else:
                first, row = torch.full_like(slots, b), slots
            for h in range(hkv):
                for t, s in ((self.k, self.ks), (self.v, self.vs)):
                    if block:
                        x = torch.randint(0, 120, (len(slots), d), generator=g, dtype=torch.uint8)
                        t[first, h, row] = x + 128 * torch.randint(0, 2, x.shape, generator=g, dtype=torch.uint8)
                        new = torch.exp(np.log(lo) + (np.log(hi) - np.log(lo)) * torch.rand(s.shape[0], s.shape[2], generator=g))
                        s[first, h, row // block] = new[first, row // block]
                    else:
                        t[first, h, row] = torch.randn(len(slots), d, generator=g).bfloat16()

    def store(self, E):
        up = lambda t: None if t is None else t.to(DEV)  # noqa: E731
        return E.KVStore(up(self.k), up(self.v), block_table=up(self.table), k_scale=up(self.ks), v_scale=up(self.vs), block_size=self.block)

    def run(self, E, store=None, **kw):
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        out = torch.full(self.q.shape, 7.0, dtype=torch.bfloat16, device=DEV)
        fn = E.eagle_tree_window_attn if self.tree else E.eagle_window_attn
        if self.tree and "tree_sizes" not in kw:
            kw["tree_sizes"] = _ints(self.n).to(DEV)
        fn(self.q.to(DEV), store or self.store(E), _ints(self.lens).to(DEV), self.order.to(DEV), out, status=status, **{**self.kw, **kw})
        torch.cuda.synchronize()
        return out.cpu(), int(status.item())

    def want(self, **kw):
        order = {"tree_parent": self.order, "tree_sizes": _ints(self.n)} if self.tree else {"token_start": self.order}
        return S.window_attn(self.q, self.k, self.v, self.lens, block_table=self.table, k_scale=self.ks, v_scale=self.vs, block=self.block, **order,
                             **{**self.kw, **kw})

    def check(self, E, **kw):
        out, status = self.run(E)
        assert status == 0
        want, spread = self.want(**kw)
        got = out.double().numpy()
        rows = ~np.isnan(want[..., 0, 0])
        assert (got[~rows] == (0.0 if self.tree else 7.0)).all(), "rows outside of the sequences"
        assert np.isfinite(got).all()
        err = np.abs(got - want)[rows]
        tol = (2.0 ** -8 * np.abs(want) + (2.0 ** (-11 if self.block else -8) + 5e-4) * spread)[rows]
        assert (err <= tol).all(), (err.max(), (err / tol).max())
        return out


CHUNKS = {
    "one_token": dict(n=[1], lens=[70], hq=4, hkv=4, window=16, sinks=2),
    "one_token_nothing_before": dict(n=[1], lens=[0], hq=4, hkv=1, window=1),
    "window_of_one": dict(n=[40, 3], lens=[300, 0], hq=4, hkv=2, window=1),
    "window_of_one_and_a_sink": dict(n=[300], lens=[5], hq=2, hkv=2, window=1, sinks=1),
    "no_window": dict(n=[70, 1, 0, 33], lens=[100, 511, 3, 0], hq=8, hkv=2),
    "far": dict(n=[130], lens=[3000], hq=8, hkv=2, window=200, sinks=3, page=64),
    "sinks_past_the_window": dict(n=[60, 20], lens=[200, 10], hq=4, hkv=4, window=30, sinks=500),
    "sinks_into_a_second_tile": dict(n=[20], lens=[900], hq=4, hkv=4, window=100, sinks=130, page=16),
    "gap_inside_a_tile": dict(n=[3, 5], lens=[100, 230], hq=4, hkv=4, window=40, sinks=5, page=16),
    "wider_than_all": dict(n=[100, 9], lens=[50, 700], hq=6, hkv=3, window=4096, sinks=4),
    "window_of_a_tile": dict(n=[257], lens=[383], hq=2, hkv=1, window=128, page=128),
    "groups_of_16": dict(n=[33, 7], lens=[400, 90], hq=16, hkv=1, window=77, sinks=9, page=32),
    "groups_of_3": dict(n=[90, 1], lens=[700, 90], hq=9, hkv=3, window=129, sinks=1),
    "small_heads": dict(n=[150, 0, 31, 5], lens=[0, 40, 500, 260], hq=8, hkv=2, d=64, window=100, sinks=4, page=16),
    "long_chunk": dict(n=[700], lens=[64], hq=4, hkv=1, window=333, sinks=2, page=256),
}
SINGLES = {
    "batch": dict(n=[1] * 9, lens=[0, 1, 15, 16, 31, 127, 128, 700, 2049], hq=8, hkv=2, window=100, sinks=4, page=16),
    "some_empty": dict(n=[1, 0, 1, 0, 1], lens=[900, 4, 33, 0, 65], hq=4, hkv=4, window=64),
    "long": dict(n=[1], lens=[9000], hq=16, hkv=1, window=7001, sinks=100, page=64),
    "no_window": dict(n=[1, 1, 1], lens=[3000, 5, 1000], hq=6, hkv=3),
    "two_of_one": dict(n=[2, 0, 0], lens=[500, 9, 9], hq=8, hkv=1, window=60, sinks=1),
    "sinks_alone_and_itself": dict(n=[1, 1], lens=[1000, 40], hq=8, hkv=2, window=1, sinks=7),
    "small_heads": dict(n=[1] * 4, lens=[10, 300, 1500, 0], hq=4, hkv=4, d=64, window=200, sinks=2, page=32),
}


@pytest.mark.parametrize("block", [0, 16, 128])
@pytest.mark.parametrize("name", CHUNKS)
def test_chunks_match_the_definition(E, name, block):
    kw = dict(CHUNKS[name])
    if block and (kw.get("d") == 64 or kw.get("page", block) % block):
        kw.pop("d", None)
        kw["page"] = block
    Case(**kw, block=block, seed=len(name)).check(E)


@pytest.mark.parametrize("block", [0, 16, 64])
@pytest.mark.parametrize("name", SINGLES)
def test_single_tokens_match_the_definition(E, name, block):
    kw = dict(SINGLES[name])
    if block and (kw.get("d") == 64 or kw.get("page", block) % block):
        kw.pop("d", None)
        kw["page"] = block
    Case(**kw, block=block, seed=len(name), spare=0).check(E)


TREES = {
    "one_node_each": dict(n=[1, 1, 1], lens=[0, 100, 513], hq=4, hkv=4),
    "mixed": dict(n=[9, 64, 0, 1, 33], lens=[3, 700, 9, 250, 0], hq=8, hkv=2, page=32),
    "window": dict(n=[30, 64, 17], lens=[1000, 300, 40], hq=8, hkv=2, window=100, sinks=4, page=32),
    "smallest_window": dict(n=[64, 64], lens=[500, 63], hq=4, hkv=1, window=64, sinks=0),
    "groups_of_16": dict(n=[64, 20], lens=[333, 90], hq=16, hkv=1, window=200, sinks=150, page=128),
    "groups_of_3": dict(n=[50, 3], lens=[127, 1], hq=3, hkv=1),
    "no_groups": dict(n=[60], lens=[129], hq=2, hkv=2, page=128),
    "small_heads": dict(n=[40, 11], lens=[300, 0], hq=8, hkv=4, d=64, window=128, sinks=1),
}


@pytest.mark.parametrize("block", [0, 32])
@pytest.mark.parametrize("name", TREES)
def test_trees_match_the_definition(E, name, block):
    kw = dict(TREES[name])
    if block and kw.get("d") == 64:
        kw.pop("d")
    Case(**kw, block=block, tree=True, seed=len(name)).check(E)


@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("page", [0, 128, 256])
def test_block_sizes(E, block, page):
    Case(n=[45, 1, 130], lens=[300, 17, 128], hq=8, hkv=2, page=page, block=block, seed=block).check(E)
    Case(n=[1] * 3, lens=[300, 17, 128], hq=8, hkv=2, page=page, block=block, seed=block, spare=0).check(E)


def test_scales_far_apart(E):
    """Blocks whose scales differ by 2^30, small and large ones: weights keep their precision."""
    for seed, n in ((1, [40, 33]), (2, [1, 1])):
        c = Case(n=n, lens=[500, 700], hq=8, hkv=2, block=16, seed=seed, spare=0)
        g = torch.Generator().manual_seed(seed)
        c.vs = torch.exp2(torch.randint(-30, 1, c.vs.shape, generator=g).float()) * 3
        c.check(E)
        c.vs = torch.full_like(c.vs, 2.0 ** -60)
        c.vs[..., ::2] = 2.0 ** 60
        c.check(E)


def test_queries_of_any_size(E):
    """Query rows from 2^-100 to 2^100 (with scales that make up for it): fp16 holds neither."""
    for n in ([30, 9], [1, 1]):
        for power in (-100, 20, 100):
            c = Case(n=n, lens=[200, 300], hq=8, hkv=2, block=32, seed=3, spare=0)
            c.q = (c.q.float() * 2.0 ** power).bfloat16()
            c.ks = c.ks * 2.0 ** -power
            c.check(E)


def test_a_visible_score_that_is_no_number(E):
    """A NaN code in a visible key, a query that is infinite, a key scale of NaN: rows that see it are NaN, the others are as before."""
    for n, spare in (([40, 33], 3), ([1, 1], 0)):
        c = Case(n=n, lens=[100, 300], hq=4, hkv=2, block=16, seed=4, spare=spare)
        whole, _ = c.run(E)
        c.k[0, 0, 50, 3] = 0x7f
        out, _ = c.run(E)
        first = c.n[0]
        assert torch.isnan(out[:first, :2]).all() and torch.equal(out[:first, 2:], whole[:first, 2:]) and torch.equal(out[first:], whole[first:])
        c = Case(n=n, lens=[100, 300], hq=4, hkv=2, block=16, seed=4, spare=spare)
        c.q[0, 1, 5] = float("inf")
        out, _ = c.run(E)
        assert torch.isnan(out[0, 1]).all() and torch.equal(out[0, 2:], whole[0, 2:]) and torch.equal(out[1:], whole[1:])
        c = Case(n=n, lens=[100, 300], hq=4, hkv=2, block=0, window=40, seed=4, spare=spare)
        whole, _ = c.run(E)
        c.k[1, 1, 290, 3] = float("nan")
        out, _ = c.run(E)
        rows = slice(first, first + c.n[1])
        sees = torch.tensor([300 + i - 40 < 290 for i in range(c.n[1])])
        assert torch.isnan(out[rows][sees, 2:]).all() and torch.equal(out[rows][~sees], whole[rows][~sees]) and torch.equal(out[:first], whole[:first])


def test_equals_the_attention_without_a_window(E):
    """Same inputs, no limit: close to eagle_chunk_attn and eagle_tree_verify_attn (the same arithmetic; the work may be cut elsewhere)."""
    c = Case(n=[200, 1, 50], lens=[100, 700, 0], hq=8, hkv=2, page=64, seed=5)
    out, _ = c.run(E)
    ref = torch.full(c.q.shape, 7.0, dtype=torch.bfloat16, device=DEV)
    E.eagle_chunk_attn(c.q.to(DEV), c.store(E), _ints(c.lens).to(DEV), c.order.to(DEV), ref)
    assert torch.equal(ref.cpu(), out)
    t = Case(n=[30, 64], lens=[100, 700], hq=8, hkv=2, tree=True, seed=6)
    out, _ = t.run(E)
    ref = E.eagle_tree_verify_attn(t.q.to(DEV), t.k.to(DEV), t.v.to(DEV), _ints(t.lens).to(DEV), t.order.to(DEV), tree_sizes=_ints(t.n).to(DEV))
    want, spread = t.want()
    assert (np.abs(out.double().numpy() - ref.cpu().double().numpy())[~np.isnan(want)] <= 2.0 ** -6 * np.nan_to_num(spread)[~np.isnan(want)] + 1e-30).all()


def test_one_tree_for_every_sequence(E):
    c = Case(n=[20, 20, 20], lens=[10, 300, 77], hq=8, hkv=2, block=32, tree=True, seed=7)
    c.order[:] = c.order[0].clone()
    out = c.check(E)
    c.order = c.order[0].contiguous()
    shared, status = c.run(E, shared_tree=True, tree_sizes=_ints([20]).to(DEV))
    assert status == 0 and torch.equal(shared, out)


def test_refused_sequences_trees_and_pages(E):
    for block in (0, 16):
        c = Case(n=[40, 5, 6], lens=[10, 300, 2], hq=4, hkv=2, page=16, block=block, seed=8)
        whole, _ = c.run(E)
        c.lens = [10, -1, 2]
        out, status = c.run(E)
        assert status == -6 and (out[40:45] == 0).all() and torch.equal(out[:40], whole[:40]) and torch.equal(out[45:], whole[45:])
        c.lens = [10, 100000, 2]
        out, status = c.run(E)
        assert status == -6 and (out[40:45] == 0).all() and torch.equal(out[:40], whole[:40])
        c.lens = [10, 300, 2]
        for bad in (-1, 1 << 20):
            old = int(c.table[1, 7])
            c.table[1, 7] = bad
            out, status = c.run(E)
            assert status == -11 and (out[40:45] == 0).all() and torch.equal(out[:40], whole[:40]) and torch.equal(out[45:], whole[45:])
            c.table[1, 7] = old
        c.order = _ints([0, 45, 40, 51])
        out, status = c.run(E)
        assert status == -6 and ((out == 0) | (out == 7)).all()      # no row is computed
        s = Case(n=[1, 1, 1], lens=[10, 300, 2], hq=4, hkv=2, page=16, block=block, seed=8, spare=0)
        whole, _ = s.run(E)
        s.table[1, 7] = -5
        out, status = s.run(E)
        assert status == -11 and (out[1] == 0).all() and torch.equal(out[0], whole[0]) and torch.equal(out[2], whole[2])
        t = Case(n=[40, 5, 6], lens=[10, 300, 2], hq=4, hkv=2, page=16, block=block, tree=True, seed=8)
        whole, _ = t.run(E)
        t.order[1, 3] = 3
        out, status = t.run(E)
        assert status == -5 and (out[1] == 0).all() and torch.equal(out[0], whole[0]) and torch.equal(out[2], whole[2])
        t.order[1, 3] = 0
        t.lens = [10, 100000, 2]
        out, status = t.run(E)
        assert status == -6 and (out[1] == 0).all() and torch.equal(out[0], whole[0])
        t.lens = [10, 300, 2]
        out, status = t.run(E, tree_sizes=_ints([40, 41, 6]).to(DEV))
        assert status == -5 and (out[1] == 0).all() and torch.equal(out[0], whole[0])
        t.table[1, 7] = -1
        out, status = t.run(E)
        assert status == -11 and (out[1] == 0).all() and torch.equal(out[0], whole[0]) and torch.equal(out[2], whole[2])


def test_replayed_from_graphs_and_on_two_streams(E):
    """Two captured calls with a workspace each and eager calls on another stream, interleaved."""
    cases = [Case(n=[130, 40], lens=[300, 700], hq=8, hkv=2, block=32, page=64, window=200, sinks=4, seed=9), Case(n=[1] * 5, lens=[300, 700, 0, 64, 2000], hq=8, hkv=2, block=64, seed=10, spare=0),
             Case(n=[33, 64], lens=[100, 900], hq=8, hkv=2, window=500, tree=True, seed=11)]
    want, held = [], []
    for c in cases:
        want.append(c.run(E)[0])
        size = _ints(c.n).to(DEV)
        held.append((c.q.to(DEV), c.store(E), _ints(c.lens).to(DEV), c.order.to(DEV), torch.full(c.q.shape, 7.0, dtype=torch.bfloat16, device=DEV),
                     {"tree_sizes": size} if c.tree else {},
                     torch.empty(E.eagle_window_attn_workspace(len(c.n), 0 if c.tree else c.q.shape[0], 8, 2, 128, max_tree=max(c.n) if c.tree else 0), dtype=torch.uint8, device=DEV)))
    graphs = []
    torch.cuda.synchronize()
    for c, (q, store, lens, order, out, more, ws) in zip(cases, held):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            (E.eagle_tree_window_attn if c.tree else E.eagle_window_attn)(q, store, lens, order, out, workspace=ws, **c.kw, **more)
        graphs.append(graph)
    side = torch.cuda.Stream()
    for _ in range(3):
        for h in held:
            h[4].fill_(7.0)
        torch.cuda.synchronize()
        for graph in graphs:
            graph.replay()
        with torch.cuda.stream(side):
            again = [c.run(E)[0] for c in cases]
        torch.cuda.synchronize()
        for h, w, a in zip(held, want, again):
            assert torch.equal(h[4].cpu(), w) and torch.equal(a, w)


def test_a_workspace_for_more_tokens_serves_fewer(E):
    ws = torch.empty(E.eagle_window_attn_workspace(3, 500, 8, 2, 128), dtype=torch.uint8, device=DEV)
    for n in ([300, 100, 100], [3, 0, 0], [1, 1, 1], [2, 1, 0]):
        c = Case(n=n, lens=[100, 30, 700], hq=8, hkv=2, block=32, seed=12, spare=0)
        out, _ = c.run(E)
        got, _ = c.run(E, workspace=ws)
        assert torch.equal(out, got)


@pytest.mark.parametrize("form", ["chunk", "singles", "tree"])
@pytest.mark.parametrize("block", [0, 32])
def test_waits_that_run_out(E, form, block):
    """The copies stop after some tiles: every wait ends, the call reports it and the next one is as ever."""
    n = {"chunk": [300, 200] * 16, "singles": [1, 1] * 100, "tree": [64, 50] * 30}[form]      # more than ten tiles to a worker
    c = Case(n=n, lens=[900, 2000] * (len(n) // 2), hq=8, hkv=2, block=block, page=64, tree=form == "tree", seed=13, spare=0)
    good, status = c.run(E)
    assert status == 0
    lib = E.load()
    for tiles in (0, 2, 9):
        lib.eagle_set_wait_limit_ns(20_000_000)
        lib.eagle_test_stall_kv_producer(tiles)
        try:
            _, status = c.run(E)
        finally:
            lib.eagle_test_stall_kv_producer(-1)
            lib.eagle_set_wait_limit_ns(0)
        assert status == -8
        out, status = c.run(E)
        assert status == 0 and torch.equal(out, good)


def test_thousands_of_single_tokens_and_many_items(E):
    g = torch.Generator().manual_seed(14)
    B = 3000
    lens = torch.randint(0, 200, (B,), generator=g).tolist()
    c = Case(n=[1] * B, lens=lens, hq=2, hkv=1, block=16, page=16, window=90, sinks=3, seed=14, spare=0)
    c.check(E)
    t = Case(n=[(i * 7) % 20 for i in range(400)], lens=lens[:400], hq=4, hkv=2, block=16, page=16, window=90, sinks=3, tree=True, seed=15)
    t.check(E)


def test_random_shapes(E):
    g = np.random.default_rng(16)
    for seed in range(60):
        form = ["chunk", "singles", "tree"][seed % 3]
        block = [0, 16, 32, 64, 128][int(g.integers(5))]
        d = 128 if block else [64, 128][int(g.integers(2))]
        page = [0, 16, 64, 256][int(g.integers(4))]
        if block and page and page < block:
            page = block
        hkv = int(g.integers(1, 4))
        hq = hkv * int(g.integers(1, 17))
        B = int(g.integers(1, 6))
        n = {"chunk": g.integers(0, 180, B), "singles": np.ones(B, int), "tree": g.integers(0, 65, B)}[form].tolist()
        n[0] = max(n[0], 1)
        window = int(g.integers(64 if form == "tree" else 1, 600)) if g.random() < 0.7 else 0
        Case(n=n, lens=g.integers(0, 900, B).tolist(), hq=hq, hkv=hkv, d=d, page=page, block=block, window=window, sinks=int(g.integers(0, 200)) if g.random() < 0.5 else 0,
             tree=form == "tree", seed=seed, spare=int(g.integers(0, 2)) if form == "chunk" else 0).check(E)


@pytest.mark.parametrize("block", [0, 16])
@pytest.mark.parametrize("form", ["chunk", "singles", "tree"])
def test_pages_at_the_far_end_of_a_large_pool(E, form, block):
    """Offsets that pass 32 bits (elements and bytes): the same sequences in the last pages of a large pool give the same bits."""
    n = {"chunk": [60, 0, 200], "singles": [1, 1, 1], "tree": [33, 1, 64]}[form]
    case = Case(n, [700, 30, 90], 8, 4, page=128, block=block, window=300, sinks=5, tree=form == "tree", spare=0)
    want = case.check(E)
    pages = 36000 if block else 70000                        # of 64 KB of codes or 128 KB of bf16: more than 2^31 elements
    far = pages - case.k.shape[0]
    assert far * case.k[0].numel() > 2 ** 31 and (block or far * case.k[0].numel() * 2 > 2 ** 32)
    k, v = (torch.empty(pages, *t.shape[1:], dtype=t.dtype, device=DEV) for t in (case.k, case.v))
    k[far:], v[far:] = case.k.to(DEV), case.v.to(DEV)
    scales = {}
    if block:
        ks, vs = (torch.empty(pages, *t.shape[1:], device=DEV) for t in (case.ks, case.vs))
        ks[far:], vs[far:] = case.ks.to(DEV), case.vs.to(DEV)
        scales = {"k_scale": ks, "v_scale": vs}
    table = torch.where(case.table >= 0, case.table + far, case.table).to(DEV)
    got, status = case.run(E, E.KVStore(k, v, block_table=table, block_size=block, **scales))
    assert status == 0 and torch.equal(got, want)


@pytest.mark.parametrize("block", [0, 32])
@pytest.mark.parametrize("form", ["chunk", "singles", "tree"])
def test_a_window_far_into_a_long_sequence(E, form, block):
    """What a window sees does not depend on how much lies in front of it: a sequence moved back by 2^24 slots."""
    n = {"chunk": [150], "singles": [1], "tree": [40]}[form]
    case = Case(n, [1000], 8, 2, block=block, window=500, tree=form == "tree", spare=0)
    want = case.check(E)
    move = 1 << 24
    lens = _ints([1000 + move]).to(DEV)
    k, v = (torch.empty(1, 2, move + t.shape[2], 128, dtype=t.dtype, device=DEV) for t in (case.k, case.v))
    k[:, :, move:], v[:, :, move:] = case.k.to(DEV), case.v.to(DEV)
    scales = {}
    if block:
        ks, vs = (torch.empty(1, 2, k.shape[2] // block, device=DEV) for _ in range(2))
        ks[:, :, move // block:], vs[:, :, move // block:] = case.ks.to(DEV), case.vs.to(DEV)
        scales = {"k_scale": ks, "v_scale": vs}
    store = E.KVStore(k, v, block_size=block, **scales)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    if form == "tree":
        got = E.eagle_tree_window_attn(case.q.to(DEV), store, lens, case.order.to(DEV), tree_sizes=_ints(n).to(DEV), status=status, **case.kw)
    else:
        got = E.eagle_window_attn(case.q.to(DEV), store, lens, case.order.to(DEV), status=status, **case.kw)
    # (2^24 is a multiple of a K/V tile, so the steps are the same; how the work is cut is a matter of its cost, which is the same, too)
    assert int(status.item()) == 0 and torch.equal(got.cpu(), want)


@pytest.mark.parametrize("form", ["chunk", "tree"])
def test_tiles_over_codes_whose_copies_land_in_any_order(E, form):
    """The same call many times, its pages spread over a large pool of which a part is in the L2 cache, another one busy reading beside it: the same bits."""
    n = {"chunk": [300, 77], "tree": [64, 20] * 8}[form]
    case = Case(n, [4000, 2500] * (len(n) // 2), 8, 4, page=16, block=16, tree=form == "tree", spare=0, seed=17)
    want = case.check(E)
    pages, g = 20000, torch.Generator().manual_seed(18)      # of 8 KB each for keys and values: more than the L2 cache holds
    to = torch.randperm(pages, generator=g)[:case.k.shape[0]]
    moved = []
    for t in (case.k, case.v, case.ks, case.vs):
        moved.append(torch.zeros(pages, *t.shape[1:], dtype=t.dtype, device=DEV))
        moved[-1][to.to(DEV)] = t.to(DEV)
    store = E.KVStore(moved[0], moved[1], k_scale=moved[2], v_scale=moved[3], block_size=16,
                      block_table=torch.where(case.table >= 0, to.int()[case.table.clamp(min=0).long()], case.table).to(DEV))
    q, lens, order, sizes = case.q.to(DEV), _ints(case.lens).to(DEV), case.order.to(DEV), _ints(n).to(DEV)
    other, side, differ = torch.empty(1 << 26, device=DEV), torch.cuda.Stream(), torch.zeros((), dtype=torch.int64, device=DEV)
    outs = [torch.full(q.shape, 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    want = want.to(DEV)
    torch.cuda.synchronize()
    for i in range(300):
        with torch.cuda.stream(side):
            if i % 3:
                other.add_(1.0)
        out = outs[i % 2]
        if form == "tree":
            E.eagle_tree_window_attn(q, store, lens, order, out, tree_sizes=sizes)
        else:
            E.eagle_window_attn(q, store, lens, order, out)
        differ += (out.view(torch.int16) != want.view(torch.int16)).any()
    torch.cuda.synchronize()
    assert int(differ.item()) == 0


@pytest.mark.parametrize("form", ["chunk", "tree", "singles", "singles_of_16_heads"])
def test_small_queries_over_small_scales(E, form):
    """Query rows down to the smallest numbers over blocks of zeros, whose scales are 2^-40 as the append leaves them, and over scales at the bottom of
    their range: every score is next to 0, and a key that a row does not see has no weight all the same."""
    n = [1, 1] if form.startswith("singles") else [40, 33]
    hq = 16 if form == "singles_of_16_heads" else 8
    for scale, power in ((2.0 ** -40, -100), (2.0 ** -40, -110), (2.0 ** -40, -120), (2.0 ** -40, -133), (2.0 ** -126, -21), (2.0 ** -126, -60), (2.0 ** -126, -126)):
        c = Case(n=n, lens=[200, 333], hq=hq, hkv=1 if hq == 16 else 2, block=16, window=90, sinks=3, tree=form == "tree", seed=19, spare=0)
        c.q = (c.q.float() * 2.0 ** power).bfloat16()
        c.ks = torch.where(torch.isnan(c.ks), c.ks, torch.full_like(c.ks, scale))
        c.check(E)
        c.k = torch.where(c.k == 0x7f, c.k, torch.zeros_like(c.k))      # (what is not visible stays NaN)
        c.check(E)


@pytest.mark.parametrize("form", ["chunk", "tree", "singles"])
def test_small_queries_over_appended_zeros(E, form):
    """Keys of zeros and ordinary values through the library's own append, then queries of 2^-120: the mean of the values that a row sees."""
    tree, hq, hkv, B = form == "tree", 8, 2, 2
    g, lens = torch.Generator().manual_seed(20), [50, 0]
    shape = (B, hkv, 192, 128)
    k, v = (torch.zeros(shape, dtype=torch.uint8, device=DEV) for _ in range(2))
    scales = [torch.ones(B, hkv, 12, device=DEV) for _ in range(2)]
    store = E.KVStore(k, v, k_scale=scales[0], v_scale=scales[1], block_size=16)
    freqs, _ = E.eagle_rope_frequencies(128, device=DEV)
    for step, n in enumerate(([50, 0], [1, 1] if form == "singles" else [40, 33])):
        last = step == 1
        rows = (B, max(n)) if tree and last else (sum(n),)
        q = (torch.randn(*rows, hq, 128, generator=g) * 2.0 ** -120).bfloat16().to(DEV)
        kk, vv = torch.zeros(*rows, hkv, 128, dtype=torch.bfloat16, device=DEV), torch.randn(*rows, hkv, 128, generator=g).bfloat16().to(DEV)
        at = _ints(lens if last else [0, 0])
        if tree and last:
            order = torch.zeros(B, max(n), dtype=torch.int32)
            for i in range(max(n)):
                order[:, i] = i // 2 - 1
            q = E.eagle_tree_block_append(q, kk, vv, store, at.to(DEV), order.to(DEV), freqs, tree_sizes=_ints(n).to(DEV))
        else:
            order = _ints(np.concatenate([[0], np.cumsum(n)]).tolist())
            q = E.eagle_block_append(q, kk, vv, store, at.to(DEV), order.to(DEV), freqs)
    assert (scales[0][0, :, :4] == 2.0 ** -40).all()
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    kw = {"tree_parent": order, "tree_sizes": _ints(n)} if tree else {"token_start": order}
    fn = E.eagle_tree_window_attn if tree else E.eagle_window_attn
    got = fn(q, store, _ints(lens).to(DEV), order.to(DEV), status=status, window=70, sinks=2, **({"tree_sizes": _ints(n).to(DEV)} if tree else {}))
    want, spread = S.window_attn(q.cpu(), k.cpu(), v.cpu(), lens, k_scale=scales[0].cpu(), v_scale=scales[1].cpu(), block=16, window=70, sinks=2, **kw)
    rows = ~np.isnan(want[..., 0, 0])
    err = np.abs(got.cpu().double().numpy() - want)[rows]
    assert int(status.item()) == 0 and (err <= (2.0 ** -8 * np.abs(want) + (2.0 ** -11 + 5e-4) * spread)[rows]).all()


@pytest.mark.parametrize("form", ["chunk", "tree", "singles", "singles_of_16_heads"])
def test_value_scales_outside_of_their_range(E, form):
    """A visible one is reported, and the rows of other sequences are as ever; one that nothing sees may be anything."""
    n = [1, 1, 1] if form.startswith("singles") else [40, 33, 20]
    hq, hkv = (16, 1) if form == "singles_of_16_heads" else (4, 2)
    for page in (0, 32):
        c = Case(n=n, lens=[200, 333, 60], hq=hq, hkv=hkv, block=16, page=page, window=120, sinks=3, tree=form == "tree", seed=21, spare=0)
        whole, status = c.run(E)
        assert status == 0
        own = slice(1, 2) if form == "tree" else slice(n[0], n[0] + n[1])
        others = torch.ones(whole.shape[0], dtype=torch.bool)
        others[own] = False
        for slot, seen in ((300, True), (2, True), (100, False), (340, form != "singles" and form != "singles_of_16_heads")):
            at, block = (int(c.table[1, slot // page]), slot % page // 16) if page else (1, slot // 16)
            if at < 0:
                continue                                     # (a page that nothing sees)
            old = c.vs[at, -1, block].item()
            for scale in (2.0 ** -60.5, 2.0 ** 60.5, 2.0 ** 120, 0.0, -1.0, float("inf"), float("nan"), 2.0 ** -60, 2.0 ** 60):
                wrong = seen and not 2.0 ** -60 <= scale <= 2.0 ** 60
                c.vs[at, -1, block] = scale
                out, status = c.run(E)
                assert status == (-13 if wrong else 0), (slot, scale, status)
                assert torch.equal(out[others], whole[others]) and (seen or torch.equal(out, whole))
            c.vs[at, -1, block] = old


def test_the_largest_values_that_can_be_attended_to(E):
    """Through the library's own append: values up to 448 * 2^60 next to zeros; a larger one is stored and reported when it is seen."""
    g, n = torch.Generator().manual_seed(22), 80
    for factor, want_status in ((1.0, 0), (1.1, -13)):
        for singles in (False, True):
            k, v = (torch.zeros(1, 1, 96, 128, dtype=torch.uint8, device=DEV) for _ in range(2))
            ks, vs = (torch.ones(1, 1, 6, device=DEV) for _ in range(2))
            store = E.KVStore(k, v, k_scale=ks, v_scale=vs, block_size=16)
            freqs, _ = E.eagle_rope_frequencies(128, device=DEV)
            q, kk, vv = torch.randn(n, 4, 128, generator=g), torch.randn(n, 1, 128, generator=g), torch.randn(n, 1, 128, generator=g)
            vv[:16] = 0.0
            vv[16:32] *= 2.0 ** 58
            vv[20, 0, 5] = 448.0 * 2.0 ** 60 * factor
            status = torch.zeros(1, dtype=torch.int32, device=DEV)
            start = _ints([0, n]).to(DEV)
            q = E.eagle_block_append(q.bfloat16().to(DEV), kk.bfloat16().to(DEV), vv.bfloat16().to(DEV), store, _ints([0]).to(DEV), start, freqs, status=status)
            assert int(status.item()) == 0 and float(vs[0, 0, 0]) == 2.0 ** -40 and float(vs[0, 0, 1]) == 2.0 ** (60 if factor == 1.0 else 61)
            lens = [0]
            if singles:
                q, lens, start = q[-1:].contiguous(), [n - 1], _ints([0, 1]).to(DEV)
            got = E.eagle_window_attn(q, store, _ints(lens).to(DEV), start, status=status)
            assert int(status.item()) == want_status
            if want_status == 0:
                want, spread = S.window_attn(q.cpu(), k.cpu(), v.cpu(), lens, token_start=start.cpu(), k_scale=ks.cpu(), v_scale=vs.cpu(), block=16)
                assert (np.abs(got.cpu().double().numpy() - want) <= 2.0 ** -8 * np.abs(want) + (2.0 ** -11 + 5e-4) * spread).all()


@pytest.mark.parametrize("block", [0, 16])
@pytest.mark.parametrize("form", ["chunk", "tree", "singles"])
def test_sequences_that_end_where_32_bits_do(E, form, block):
    """A window at the far end of a sequence of almost 2^31 slots (of whose pages the table holds the last few): up to 2^31 - 256 the same as anywhere else, past it refused."""
    n = {"chunk": [150], "singles": [1], "tree": [40]}[form]
    most, page = 2 ** 31 - 256, 256
    near = 1024 - n[0]                                       # ends with a tile, as the far one does
    case = Case(n, [near], 8, 2, page=page, block=block, window=300, tree=form == "tree", seed=24, spare=0)
    want = case.check(E)
    table = torch.full((1, 2 ** 31 // page), -1, dtype=torch.int32)
    shift = (most - 1024) // page
    table[0, shift:shift + 4] = case.table[0, :4]
    table[0, shift + 4] = case.table[0, 3]
    case.table = table
    store = case.store(E)
    case.lens = [most - n[0]]
    out, status = case.run(E, store)
    assert status == 0 and torch.equal(out, want)
    for more in (1, 100, 255):
        case.lens = [most - n[0] + more]
        out, status = case.run(E, store)
        assert status == -6 and (out == 0).all()
