"""Attention of packed chunks over the cache, against the 64-bit definition.

Tolerance, element by element: the output is rounded to bf16 (2^-8 of it) and every probability before it is multiplied
with its value (2^-8 of sum p |v|, which the oracle returns); scores, exponentials (one pair in a few is a cubic good to 1.2e-4) and sums are
fp32, for which 5e-4 of the same sum is ample: a score of 128 products of unit-variance inputs is good to about 1e-5 and its
exponential relatively to the same."""
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
    """Keys and values only where the sequences are: every other slot is NaN."""

    def __init__(self, n, lens, hq, hkv, d, page=0, seed=0, pad=37, spare=3):
        g = torch.Generator().manual_seed(seed)
        self.n, self.lens, self.page = n, lens, page
        B, need = len(n), [a + b for a, b in zip(n, lens)]
        self.start = _ints(np.concatenate([[0], np.cumsum(n)]).tolist())
        self.q = torch.randn(sum(n) + spare, hq, d, generator=g).bfloat16()
        if page:
            used = [-(-x // page) for x in need]
            order = torch.randperm(sum(used) + 2, generator=g).tolist()
            self.table = torch.full((B, max(max(used), 1) + 1), -1, dtype=torch.int32)
            for b, u in enumerate(used):
                self.table[b, :u] = _ints([order.pop() for _ in range(u)])
            shape = (sum(used) + 2, hkv, page, d)
        else:
            self.table, shape = None, (B, hkv, max(need) + pad, d)
        self.k, self.v = (torch.full(shape, float("nan"), dtype=torch.bfloat16) for _ in range(2))
        for b, m in enumerate(need):
            kk, vv = (torch.randn(hkv, m, d, generator=g).bfloat16() for _ in range(2))
            if page:
                for i in range(-(-m // page)):
                    w = min(page, m - i * page)
                    self.k[self.table[b, i], :, :w], self.v[self.table[b, i], :, :w] = kk[:, i * page:i * page + w], vv[:, i * page:i * page + w]
            else:
                self.k[b, :, :m], self.v[b, :, :m] = kk, vv

    def run(self, E, **kw):
        up = lambda t: None if t is None else t.to(DEV)  # noqa: E731
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        out = torch.full(self.q.shape, 7.0, dtype=torch.bfloat16, device=DEV)
        E.eagle_chunk_attn(up(self.q), E.KVStore(up(self.k), up(self.v), block_table=up(self.table)), up(_ints(self.lens)), up(self.start), out,
                           status=status, **kw)
        torch.cuda.synchronize()
        return out.cpu(), int(status.item())

    def want(self, **kw):
        return S.chunk_attn(self.q, self.k, self.v, self.lens, self.start, block_table=self.table, **kw)


def _check(out, want, spread):
    got = out.double().numpy()
    rows = ~np.isnan(want[:, 0, 0])
    assert (got[~rows] == 7.0).all(), "rows outside the sequences have changed"
    assert np.isfinite(got).all()
    err, tol = np.abs(got - want)[rows], (2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 5e-4) * spread)[rows]
    assert (err <= tol).all(), (err.max(), (err / tol).max())


CASES = {
    "one_token_empty_cache": dict(n=[1], lens=[0], hq=1, hkv=1, d=64),
    "one_token": dict(n=[1], lens=[300], hq=8, hkv=2, d=128),
    "two_tokens_at_a_tile_edge": dict(n=[2, 2, 2, 1], lens=[126, 127, 128, 127], hq=4, hkv=4, d=128),
    "single_tokens_lone_head": dict(n=[1, 1, 1], lens=[5, 1000, 255], hq=4, hkv=1, d=64),
    "three_heads": dict(n=[40, 1, 0, 130], lens=[0, 700, 9, 60], hq=12, hkv=3, d=128),
    "group_of_five": dict(n=[61, 26], lens=[10, 0], hq=10, hkv=2, d=64),
    "group_of_seven": dict(n=[100], lens=[33], hq=7, hkv=1, d=128),
    "group_of_sixteen": dict(n=[19, 8, 1], lens=[0, 200, 4000], hq=16, hkv=1, d=128),
    "no_group": dict(n=[257, 3], lens=[0, 127], hq=3, hkv=3, d=64),
    "prompt_in_tiles": dict(n=[512], lens=[0], hq=2, hkv=1, d=128),
    "prompt_behind_a_prefix": dict(n=[300], lens=[1000], hq=4, hkv=1, d=128),
    "ragged_many": dict(n=[(i * 7) % 23 for i in range(40)], lens=[(i * 53) % 411 for i in range(40)], hq=4, hkv=2, d=64),
    "all_empty": dict(n=[0, 0], lens=[3, 0], hq=4, hkv=2, d=64),
}


@pytest.mark.parametrize("page", [0, 16, 64, 256])
@pytest.mark.parametrize("name", list(CASES))
def test_matches_the_definition(E, name, page):
    c = Case(**CASES[name], page=page, seed=len(name))
    out, status = c.run(E)
    assert status == 0
    _check(out, *c.want())


def test_one_long_context_is_split_and_merged(E):
    """One token over a long context: every CTA takes a piece (even and odd numbers of KV heads: twins and lone tiles)."""
    for hq, hkv in ((4, 2), (3, 1), (6, 3)):
        c = Case([1], [30011], hq, hkv, 64, page=128, seed=hq)
        out, status = c.run(E)
        assert status == 0
        _check(out, *c.want())


def test_many_single_tokens_are_whole_units_and_pieces(E):
    """More units than CTAs, of very different lengths: whole ones are dealt out, the rest is cut."""
    lens = [(i * 977) % 2600 for i in range(90)]
    c = Case([1] * 90, lens, 8, 4, 64, page=32, seed=3)
    out, status = c.run(E)
    assert status == 0
    _check(out, *c.want())


def test_the_softmax_scale_and_growing_scores(E):
    c = Case([130], [200], 2, 1, 64, seed=4)
    for scale in (0.01, 1.0):
        out, status = c.run(E, sm_scale=scale)
        want, spread = c.want(sm_scale=scale)
        # a score's fp32 error grows with the scale: 64 products of up to ~16 each, 2^-24 apiece, times the scale
        assert status == 0
        _check(out, want, spread)
    # keys that grow along the sequence move the running maximum again and again
    c.k *= torch.linspace(0.01, 6.0, c.k.shape[2]).bfloat16()[:, None]
    out, status = c.run(E)
    assert status == 0
    _check(out, *c.want())


def test_masked_slots_may_hold_anything(E):
    """Keys that a row does not see may be infinite or NaN; past the chunk, values too (the cases above have NaN there)."""
    c = Case([140], [20], 4, 2, 128, seed=6)
    c.k[0, :, 159] = float("nan")
    c.k[0, :, 158] = float("inf")
    out, status = c.run(E)
    want, spread = c.want()
    assert status == 0
    got = out.double().numpy()
    err = np.abs(got - want)[:138]
    assert (err <= (2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 5e-4) * spread)[:138]).all()
    assert np.isnan(got[139]).all()


def test_paged_equals_contiguous_bit_for_bit_and_repeats(E):
    kw = dict(n=[70, 1, 200, 0, 1], lens=[300, 2000, 5, 8, 61], hq=8, hkv=2, d=128, seed=7)
    a = Case(**kw)
    want = a.run(E)[0]
    for page in (16, 128):
        c = Case(**kw, page=page)
        for b, m in enumerate([x + y for x, y in zip(c.n, c.lens)]):
            for j in range(m):
                at = int(c.table[b, j // page]), slice(None), j % page
                c.k[at], c.v[at] = a.k[b, :, j], a.v[b, :, j]
        c.q = a.q
        for _ in range(3):
            same = torch.equal(want.view(torch.int16), c.run(E)[0].view(torch.int16))
            assert same


def test_a_workspace_full_of_leftovers(E):
    c = Case([33, 1, 5], [100, 900, 0], 6, 3, 64, seed=8)
    ws = torch.full((E.eagle_chunk_attn_workspace(3, c.q.shape[0], 6, 3, 64),), 255, dtype=torch.uint8, device=DEV)
    out, status = c.run(E, workspace=ws)
    _check(out, *c.want())
    other = Case([1, 1, 1], [3000, 10, 10], 6, 3, 64, seed=9)
    other.q = other.q[:c.q.shape[0]]
    out, status = other.run(E, workspace=ws)
    assert status == 0
    _check(out, *other.want())


# ---------------------------------------------------------------------------------------------------------------- bad inputs
def test_a_sequence_that_does_not_fit_is_zeroed(E):
    c = Case([5, 6, 3], [10, 20, 30], 4, 2, 64, seed=10)
    want, spread = c.want()
    for bad in (-2, c.k.shape[2] - 5):
        c.lens = [10, bad, 30]
        out, status = c.run(E)
        assert status == -6 and (out[5:11] == 0).all()
        w, sp = want.copy(), spread.copy()
        w[5:11], sp[5:11] = 0, 0
        _check(out, w, sp)


def test_a_page_outside_the_pool_is_reported_and_the_sequence_zeroed(E):
    c = Case([5, 6, 3], [10, 200, 30], 4, 2, 64, page=16, seed=11)
    want, spread = c.want()
    for bad in (-1, c.k.shape[0], 2 ** 31 - 1, -(2 ** 31)):
        c.table[1, 12] = bad                 # the last page in use
        out, status = c.run(E)
        assert status == -11 and (out[5:11] == 0).all()
        w, sp = want.copy(), spread.copy()
        w[5:11], sp[5:11] = 0, 0
        _check(out, w, sp)
    assert c.table[1, 13] == -1              # an entry past the pages in use is never looked at


def test_starts_that_descend_or_leave_the_rows_are_refused(E):
    c = Case([5, 6, 3], [10, 20, 30], 4, 2, 64, seed=12)
    good = c.start.clone()
    for i, v in ((1, 12), (3, 18), (0, -1), (2, 4)):
        c.start = good.clone()
        c.start[i] = v
        assert c.run(E)[1] == -6
    c.start = good
    out, status = c.run(E)
    assert status == 0
    _check(out, *c.want())


def test_a_limit_on_waits_that_none_needs_changes_nothing(E):
    c = Case([64, 1], [500, 700], 4, 2, 128, seed=13)
    E.set_wait_limit_ns(200_000_000)
    try:
        out, status = c.run(E)
    finally:
        E.set_wait_limit_ns(0)
    assert status == 0
    _check(out, *c.want())


def test_replayed_from_a_graph_with_other_lengths(E):
    """The plan is made on the device: a captured call follows the lengths it finds when it is replayed."""
    a, b = Case([20, 1, 30], [100, 50, 0], 4, 2, 128, page=16, seed=14), Case([1, 49, 1], [3, 60, 400], 4, 2, 128, page=16, seed=15)
    pages, per = max(a.k.shape[0], b.k.shape[0]), max(a.table.shape[1], b.table.shape[1])
    dev = dict(q=torch.empty_like(a.q, device=DEV), k=torch.empty(pages, 2, 16, 128, dtype=torch.bfloat16, device=DEV),
               v=torch.empty(pages, 2, 16, 128, dtype=torch.bfloat16, device=DEV), table=torch.full((3, per), -1, dtype=torch.int32, device=DEV),
               lens=torch.zeros(3, dtype=torch.int32, device=DEV), start=torch.zeros(4, dtype=torch.int32, device=DEV))
    out, status = torch.full(a.q.shape, 7.0, dtype=torch.bfloat16, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    kv = E.KVStore(dev["k"], dev["v"], block_table=dev["table"])
    ws = torch.empty(E.eagle_chunk_attn_workspace(3, a.q.shape[0], 4, 2, 128), dtype=torch.uint8, device=DEV)
    graph = torch.cuda.CUDAGraph()
    E.eagle_chunk_attn(dev["q"], kv, dev["lens"], dev["start"], out, workspace=ws, status=status)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        E.eagle_chunk_attn(dev["q"], kv, dev["lens"], dev["start"], out, workspace=ws, status=status)
    for c in (a, b, a):
        out.fill_(7.0)
        dev["q"].copy_(c.q)
        dev["k"][:c.k.shape[0]].copy_(c.k)
        dev["v"][:c.v.shape[0]].copy_(c.v)
        dev["table"][:, :c.table.shape[1]].copy_(c.table)
        dev["lens"].copy_(_ints(c.lens))
        dev["start"].copy_(c.start)
        graph.replay()
        torch.cuda.synchronize()
        assert int(status.item()) == 0
        _check(out.cpu(), *c.want())


@pytest.mark.parametrize("seed", range(12))
def test_random_shapes(E, seed):
    r = np.random.default_rng(seed)
    hkv, G, d = int(r.integers(1, 5)), int(r.integers(1, 17)), int(r.choice([64, 128]))
    B = int(r.integers(1, 12))
    n = [int(x) for x in r.integers(0, int(r.choice([2, 40, 200])), B)]
    lens = [int(x) for x in r.integers(0, int(r.choice([5, 300, 3001])), B)]
    c = Case(n, lens, G * hkv, hkv, d, page=int(r.choice([0, 16, 32, 64, 128])), seed=seed + 100)
    out, status = c.run(E)
    assert status == 0
    _check(out, *c.want())


# ---- no more rows than sequences: the kernel for single tokens (it takes several tokens of a sequence too, 16 / G at a time)
ROWS = {
    "lone": dict(n=[1], lens=[0], hq=1, hkv=1, d=64),
    "tile_edges": dict(n=[1] * 8, lens=[62, 63, 64, 126, 127, 128, 191, 255], hq=4, hkv=2, d=128),
    "group_of_three": dict(n=[1, 1, 1], lens=[700, 1, 90], hq=12, hkv=4, d=128),
    "group_of_seven": dict(n=[1, 0, 1, 0], lens=[33, 8, 1500, 0], hq=7, hkv=1, d=64),
    "group_of_sixteen": dict(n=[1, 1], lens=[4000, 64], hq=32, hkv=2, d=128),
    "no_group": dict(n=[1] * 5, lens=[0, 1, 2, 300, 500], hq=3, hkv=3, d=64),
    "sixteen_tokens_in_a_tile": dict(n=[16, 0, 1] + [0] * 20, lens=[50, 3, 700] + [1] * 20, hq=2, hkv=2, d=128),
    "more_tokens_than_a_tile": dict(n=[20] + [0] * 21 + [2], lens=[117] + [9] * 21 + [0], hq=10, hkv=2, d=64),
    "a_tile_for_each_token": dict(n=[0, 9, 1, 3] + [0] * 12, lens=[0, 60, 127, 126] + [40] * 12, hq=16, hkv=1, d=128),
    "one_long": dict(n=[1], lens=[30011], hq=6, hkv=3, d=128),
    "long_and_short": dict(n=[1] * 90, lens=[(i * 977) % 2600 for i in range(90)], hq=8, hkv=4, d=64),
    "all_empty": dict(n=[0, 0], lens=[3, 0], hq=4, hkv=2, d=64),
}


@pytest.mark.parametrize("page", [0, 16, 32, 64, 256])
@pytest.mark.parametrize("name", list(ROWS))
def test_single_tokens_match_the_definition(E, name, page):
    c = Case(**ROWS[name], page=page, seed=len(name), spare=0)
    assert c.q.shape[0] <= len(c.n)
    out, status = c.run(E)
    assert status == 0
    _check(out, *c.want())


def test_single_tokens_with_a_row_behind_the_last_sequence(E):
    c = Case([1, 0, 0, 1, 0], [200, 5, 0, 77, 1], 8, 2, 128, page=16, seed=21, spare=2)
    out, status = c.run(E)
    assert status == 0
    _check(out, *c.want())


def test_single_tokens_and_what_they_cannot_see(E):
    """Infinite and NaN keys of later tokens, growing scores, a NaN that is seen: as for chunks."""
    c = Case([3, 0, 0, 0], [200, 0, 0, 0], 4, 2, 128, seed=22, spare=0)
    c.k[0, :, 202] = float("nan")
    c.k[0, :, 201] = float("inf")
    out, status = c.run(E)
    want, spread = c.want()
    assert status == 0
    got = out.double().numpy()
    err = np.abs(got - want)[:1]
    assert (err <= (2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 5e-4) * spread)[:1]).all()
    assert np.isnan(got[2]).all()
    c = Case([1, 1], [900, 310], 4, 1, 64, seed=23, spare=0)
    c.k *= torch.linspace(0.01, 6.0, c.k.shape[2]).bfloat16()[:, None]
    out, status = c.run(E)
    assert status == 0
    _check(out, *c.want())


def test_single_tokens_repeat_bit_for_bit_over_any_cache(E):
    kw = dict(n=[1] * 9, lens=[300, 2000, 5, 8, 61, 64, 63, 4000, 0], hq=8, hkv=2, d=128, seed=24, spare=0)
    a = Case(**kw)
    want = a.run(E)[0]
    for page in (16, 128):
        c = Case(**kw, page=page)
        for b, m in enumerate([x + y for x, y in zip(c.n, c.lens)]):
            for j in range(m):
                at = int(c.table[b, j // page]), slice(None), j % page
                c.k[at], c.v[at] = a.k[b, :, j], a.v[b, :, j]
        c.q = a.q
        for _ in range(3):
            assert torch.equal(want.view(torch.int16), c.run(E)[0].view(torch.int16))


def test_single_tokens_of_bad_sequences_are_zeroed(E):
    c = Case([1, 1, 1], [40, 70, 20], 4, 2, 64, page=16, seed=25, spare=0)
    want = c.want()[0]
    c.table[1, 2] = c.k.shape[0]
    out, status = c.run(E)
    assert status == -11 and (out[1] == 0).all()
    for b in (0, 2):
        assert np.abs(out[b].double().numpy() - want[b]).max() < 0.05
    c.table[1, 2] = 0
    c.lens[1] = c.table.shape[1] * 16
    out, status = c.run(E)
    assert status == -6 and (out[1] == 0).all()
    for b in (0, 2):
        assert np.abs(out[b].double().numpy() - want[b]).max() < 0.05


@pytest.mark.parametrize("spare", [0, 3])
def test_more_sequences_and_units_than_the_planner_keeps_at_hand(E, spare):
    n = [i % 3 % 2 for i in range(300)] if spare == 0 else [(i * 5) % 4 for i in range(300)]
    for hq, hkv in ((4, 2), (16, 16)):
        c = Case(n, [(i * 37) % 90 for i in range(300)], hq, hkv, 64, page=16 if hq == 4 else 0, seed=26, spare=spare)
        out, status = c.run(E)
        assert status == 0
        _check(out, *c.want())
    # (5000 units and more)
    c = Case([1] * 320 if spare == 0 else [2] * 320, [(i * 11) % 30 for i in range(320)], 16, 16, 64, seed=27, spare=spare)
    out, status = c.run(E)
    assert status == 0
    _check(out, *c.want())


@pytest.mark.parametrize("spare", [0, 3])
@pytest.mark.parametrize("page", [0, 256])
def test_caches_of_more_than_2_31_elements(E, page, spare):
    """The same sequences at the far end of a large cache: the outputs agree bit for bit."""
    c = Case([1, 1, 1] if spare == 0 else [1, 40, 130], [500, 3, 777], 16, 8, 128, page=page, seed=28, spare=spare)
    want, status = c.run(E)
    assert status == 0
    k, v = c.k, c.v
    if page:
        shape = (9000, 8, page, 128)                     # 2.4e9 elements
        far = 9000 - k.shape[0]
        c.k, c.v = (torch.empty(shape, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        c.k[far:], c.v[far:] = k.to(DEV), v.to(DEV)
        c.table = torch.where(c.table >= 0, c.table + far, c.table)
    else:
        c.k, c.v = (torch.empty(3, 8, 1000000, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        c.k[:, :, :k.shape[2]], c.v[:, :, :k.shape[2]] = k.to(DEV), v.to(DEV)
    out, status = c.run(E)
    assert status == 0 and torch.equal(out.view(torch.int16), want.view(torch.int16))
    del c
    torch.cuda.empty_cache()


def test_single_tokens_of_long_streams(E):
    """Every SM streams megabytes through its ring, call after call: the same bits each time, and the tile kernel's answer (which
    it takes when rows behind the last sequence make them more than the sequences).  The tolerance is twice the one above;
    sum p |v| is the tile kernel's too, of absolute values, 1% up for its own error."""
    g = torch.Generator(device=DEV).manual_seed(29)
    lens = [512 + (i * 2311) % 7600 for i in range(48)]
    for d, hq, hkv, page in ((128, 32, 8, 64), (64, 16, 8, 16), (128, 16, 16, 0)):
        per = 8192 // page if page else 0
        shape = (48 * per, hkv, page, d) if page else (48, hkv, 8192, d)
        q = torch.randn(51, hq, d, generator=g, device=DEV).bfloat16()
        k, v = (torch.randn(shape, generator=g, device=DEV, dtype=torch.bfloat16) for _ in range(2))
        table = torch.randperm(48 * per, generator=g, device=DEV).int().view(48, per) if page else None
        sl, start = _ints(lens).to(DEV), torch.arange(49, dtype=torch.int32, device=DEV)
        runs = [E.eagle_chunk_attn(q[:48], E.KVStore(k, v, block_table=table), sl, start) for _ in range(6)]
        tile = E.eagle_chunk_attn(q, E.KVStore(k, v, block_table=table), sl, start)[:48].double()
        spread = 1.01 * E.eagle_chunk_attn(q, E.KVStore(k, v.abs(), block_table=table), sl, start)[:48].double()
        torch.cuda.synchronize()
        assert all(torch.equal(runs[0].view(torch.int16), r.view(torch.int16)) for r in runs[1:])
        err = (runs[0].double() - tile).abs()
        assert bool((err <= 2 * (2.0 ** -8 * tile.abs() + (2.0 ** -8 + 5e-4) * spread)).all())


def test_calls_on_two_streams_at_once(E):
    """Both kernels, back to back on two streams with workspaces of their own: each gives what it gives alone."""
    cases = [Case([1] * 40, [(i * 331) % 3000 for i in range(40)], 8, 2, 128, page=32, seed=41, spare=0),
             Case([150, 1, 77], [300, 4000, 0], 8, 2, 128, page=16, seed=42),
             Case([1, 0, 1], [9000, 5, 20], 16, 4, 64, seed=43, spare=0)]
    want = [c.run(E)[0] for c in cases]
    args = [(c.q.to(DEV), E.KVStore(c.k.to(DEV), c.v.to(DEV), block_table=None if c.table is None else c.table.to(DEV)), _ints(c.lens).to(DEV), c.start.to(DEV))
            for c in cases]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    outs = []
    for rep in range(12):
        for i, s in enumerate(streams):
            which = (rep + i) % 3
            with torch.cuda.stream(s):
                out = torch.full(cases[which].q.shape, 7.0, dtype=torch.bfloat16, device=DEV)
                E.eagle_chunk_attn(*args[which], out)
            outs.append((which, out))
    torch.cuda.synchronize()
    assert all(torch.equal(o.cpu().view(torch.int16), want[w].view(torch.int16)) for w, o in outs)


def test_thousands_of_single_tokens(E):
    c = Case([1] * 3000, [(i * 7) % 50 for i in range(3000)], 2, 1, 64, page=16, seed=44, spare=0)
    out, status = c.run(E)
    assert status == 0
    _check(out, *c.want())


def test_single_tokens_replayed_from_a_graph_with_other_lengths(E):
    """A serving loop's decode graph: a fixed number of rows, sequences that grow, end (their rows stay as they are) and begin."""
    steps = [Case([1, 1, 0, 1], [40, 700, 3, 0], 8, 2, 128, page=16, seed=45, spare=1), Case([0, 1, 1, 1], [9, 701, 333, 1], 8, 2, 128, page=16, seed=46, spare=1),
             Case([0, 0, 0, 0], [1, 2, 3, 4], 8, 2, 128, page=16, seed=47, spare=4)]
    pages, per = max(c.k.shape[0] for c in steps), max(c.table.shape[1] for c in steps)
    k, v = (torch.empty(pages, 2, 16, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    table, lens, start = torch.full((4, per), -1, dtype=torch.int32, device=DEV), torch.zeros(4, dtype=torch.int32, device=DEV), torch.zeros(5, dtype=torch.int32, device=DEV)
    q, out, status = torch.zeros(4, 8, 128, dtype=torch.bfloat16, device=DEV), torch.empty(4, 8, 128, dtype=torch.bfloat16, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    kv, ws = E.KVStore(k, v, block_table=table), torch.empty(E.eagle_chunk_attn_workspace(4, 4, 8, 2, 128), dtype=torch.uint8, device=DEV)
    E.eagle_chunk_attn(q, kv, lens, start, out, workspace=ws, status=status)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        E.eagle_chunk_attn(q, kv, lens, start, out, workspace=ws, status=status)
    for c in steps + steps[:1]:
        out.fill_(7.0)
        q.copy_(c.q)
        k[:c.k.shape[0]].copy_(c.k)
        v[:c.v.shape[0]].copy_(c.v)
        table.fill_(-1)
        table[:, :c.table.shape[1]].copy_(c.table)
        lens.copy_(_ints(c.lens))
        start.copy_(c.start)
        graph.replay()
        torch.cuda.synchronize()
        assert int(status.item()) == 0
        _check(out.cpu(), *c.want())


@pytest.mark.parametrize("single", [False, True])
@pytest.mark.parametrize("what", ["nan", "inf"])
def test_a_visible_nan_or_infinite_score_makes_its_row_nan_wherever_it_is(E, what, single):
    """At every place of a tile's first 32 columns and some later ones: rows that see the key, and only those (a key with one infinite
    component scores +inf or -inf by the query's sign; -inf is a weight of 0)."""
    for at in list(range(33)) + [63, 64, 97, 127, 130]:
        c = Case([1, 1] if single else [3, 1, 40], [131, 50] if single else [131, 50, 100], 4, 2, 128, seed=51, spare=0 if single else 3)
        c.k[0, :, at] = float("nan") if what == "nan" else 0.0
        if what == "inf":
            c.k[0, :, at, 5] = float("inf")
        out, status = c.run(E)
        assert status == 0
        got = out.double().numpy()
        hit = np.zeros(got.shape[:2], bool)
        n0 = c.n[0]
        hit[:n0] = True if what == "nan" else (c.q[:n0, :, 5].double().numpy() > 0)
        if what == "inf":
            c.k[0, :, at] = 0.0                        # score 0 in place of -inf: one weight more, so those rows are only looked at for NaN
        want, spread = c.want() if what == "inf" else (None, None)
        assert np.isnan(got[hit]).all()
        rest = ~hit
        rest[sum(c.n):] = False
        assert np.isfinite(got[rest]).all()
        if what == "inf":
            err, tol = np.abs(got - want), 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 5e-4) * spread
            rest[:n0] = False
            assert (err <= tol)[rest].all()


# ---------------------------------------------------------------------------------- cut units of bad sequences, extreme values
@pytest.mark.parametrize("where", ["first", "middle", "last"])
@pytest.mark.parametrize("single", [False, True])
def test_a_page_outside_the_pool_in_a_sequence_whose_units_are_cut(E, single, where):
    """Its rows are zeros although pieces of them come to be merged, and the other sequences' are what they are without it."""
    c = Case(*(([1, 1], [30011, 500], 6, 3) if single else ([140, 1, 9], [30000, 40, 300], 4, 2)), 128, page=16, seed=61, spare=0 if single else 3)
    want, spread = c.want()
    used = -(-(c.n[0] + c.lens[0]) // 16)
    c.table[0, {"first": 0, "middle": used // 2, "last": used - 1}[where]] = c.k.shape[0]
    want[:c.n[0]], spread[:c.n[0]] = 0, 0
    q, kv, lens, start = c.q.to(DEV), E.KVStore(c.k.to(DEV), c.v.to(DEV), block_table=c.table.to(DEV)), _ints(c.lens).to(DEV), c.start.to(DEV)
    outs, status = [torch.full(c.q.shape, 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(20)], torch.zeros(1, dtype=torch.int32, device=DEV)
    for out in outs:
        E.eagle_chunk_attn(q, kv, lens, start, out, status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == -11
    for out in outs:
        assert (out[:c.n[0]] == 0).all()
        _check(out.cpu(), want, spread)


def test_short_calls_one_right_behind_another(E):
    """A CTA takes the shared and tensor memory that the call before has just left: thousands of calls of one to a few steps, both
    head sizes and both kernels in turn, give the same bits every time."""
    cases = [Case([2, 1], [3, 0], 4, 2, 64, seed=71), Case([60, 9], [0, 131], 8, 8, 128, page=16, seed=72), Case([1, 1], [50, 5], 8, 8, 128, seed=73, spare=0),
             Case([300], [100], 2, 2, 64, page=64, seed=74)]
    args = []
    for c in cases:
        kv = E.KVStore(c.k.to(DEV), c.v.to(DEV), block_table=None if c.table is None else c.table.to(DEV))
        args.append((c.q.to(DEV), kv, _ints(c.lens).to(DEV), c.start.to(DEV)))
    outs = [[torch.full(c.q.shape, 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2)] for c in cases]
    spaces = [[torch.empty(E.eagle_chunk_attn_workspace(len(c.n), c.q.shape[0], c.q.shape[1], c.k.shape[1], c.q.shape[2]), dtype=torch.uint8, device=DEV)
               for _ in range(2)] for c in cases]
    status, graph = torch.zeros(1, dtype=torch.int32, device=DEV), torch.cuda.CUDAGraph()
    for i, c in enumerate(cases):
        E.eagle_chunk_attn(*args[i], outs[i][0], workspace=spaces[i][0], status=status)
        _check(outs[i][0].cpu(), *c.want())
    want = [o[0].clone() for o in outs]
    with torch.cuda.graph(graph):
        for k in range(2):
            for i in range(len(cases)):
                E.eagle_chunk_attn(*args[i], outs[i][k], workspace=spaces[i][k], status=status)
    differ = torch.zeros((), dtype=torch.int64, device=DEV)
    for _ in range(300):
        for o in outs:
            o[0].fill_(7.0), o[1].fill_(7.0)
        graph.replay()
        for o, w in zip(outs, want):
            differ += sum((x.view(torch.int16) != w.view(torch.int16)).sum() for x in o)
    torch.cuda.synchronize()
    assert int(status.item()) == 0 and int(differ.item()) == 0


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("single", [False, True])
def test_scores_of_large_magnitude(E, single, sign):
    """Every score is a multiple of 2048 between 2^22 and 2^24 (or its negative) plus a whole number of at most 5, all of them exact
    in fp32, so the weights are exact as well up to the errors of any other row: what the large part adds to all of a row cancels."""
    g = torch.Generator().manual_seed(62)
    c = Case(*(([1, 1], [900, 301]) if single else ([40, 3, 1], [200, 700, 2000])), 16, 1, 128, seed=62, spare=0 if single else 3)
    for t in (c.q, c.k):
        t[:] = torch.where(t.isnan(), t, 0)
    i = torch.arange(c.q.shape[0] * 16).view(-1, 16)
    c.q[..., 0], c.q[..., 1] = 2048.0 * (1 + (i % 128) / 128) * (1 + i // 128 % 2), 1.0
    for b, m in enumerate([x + y for x, y in zip(c.n, c.lens)]):
        c.k[b, :, :m, 0] = 2048.0 * sign
        c.k[b, :, :m, 1] = torch.randint(-5, 6, (m,), generator=g).bfloat16()
    out, status = c.run(E, sm_scale=1.0)
    assert status == 0
    _check(out, *c.want(sm_scale=1.0))


def test_row_sums_change_hands_between_items_of_a_few_steps(E):
    """Each item of two or more steps has its row sums in both softmax groups: hundreds of items of two to five steps in every CTA pair,
    call after call with the same bits, and values of 1 come out as 1 (within the roundings of the probabilities: 2^-8, and 5e-4)."""
    c = Case([70 + i % 5 for i in range(60)], [130 + (i * 67) % 400 for i in range(60)], 16, 16, 64, seed=75)
    c.v = torch.where(c.v.isnan(), c.v, 1).bfloat16()
    q, kv, lens, start = c.q.to(DEV), E.KVStore(c.k.to(DEV), c.v.to(DEV)), _ints(c.lens).to(DEV), c.start.to(DEV)
    outs = [E.eagle_chunk_attn(q, kv, lens, start)[:sum(c.n)] for _ in range(10)]
    torch.cuda.synchronize()
    assert all(torch.equal(outs[0].view(torch.int16), o.view(torch.int16)) for o in outs[1:])
    assert float((outs[0].float() - 1).abs().max()) <= 2.0 ** -8 + 2.0 ** -8 + 5e-4


@pytest.mark.parametrize("prefix", [20, 6000])
@pytest.mark.parametrize("single", [False, True])
def test_the_largest_values_in_slots_that_a_row_does_not_see(E, single, prefix):
    """The weight of a slot that a row does not see is 0, whatever finite value stands there."""
    c = Case([6] + [0] * 7 if single else [140], [prefix] + [5] * 7 if single else [prefix], 4, 2, 128, seed=63, spare=0 if single else 3)
    first, end = prefix + (2 if single else 110), prefix + c.n[0]
    c.v[0, :, first:end] = 3e38
    c.v[0, :, first:end:3] = -3e38
    out, status = c.run(E)
    want, spread = c.want()
    assert status == 0
    n = first - prefix
    err, tol = np.abs(out.double().numpy() - want)[:n], (2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 5e-4) * spread)[:n]
    assert (err <= tol).all(), (err.max(), (err / tol).max())


@pytest.mark.parametrize("tiles", [0, 2, 9])
@pytest.mark.parametrize("d,page", [(128, 0), (128, 16), (64, 0), (64, 64)])
@pytest.mark.parametrize("single", [False, True])
def test_a_wait_that_runs_out_is_reported_and_the_next_call_is_right(E, single, d, page, tiles):
    """The copies of every CTA fall silent after some tiles (test hook) and the limit is 2 ms: the call returns by itself with the status
    of a time-out, rows outside the sequences are as they were, and an ordinary call right after gives the same bits as one before."""
    c = Case(*(([1, 1], [60000, 31000]) if single else ([70, 0, 5], [40000, 3, 31000])), 8, 4, d, page=page, seed=81, spare=0 if single else 3)
    q, kv = c.q.to(DEV), E.KVStore(c.k.to(DEV), c.v.to(DEV), block_table=None if c.table is None else c.table.to(DEV))
    lens, start, used = _ints(c.lens).to(DEV), c.start.to(DEV), sum(c.n)

    def call():
        out, status = torch.full(c.q.shape, 7.0, dtype=torch.bfloat16, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
        E.eagle_chunk_attn(q, kv, lens, start, out, status=status)
        torch.cuda.synchronize()
        return out, int(status.item())

    want, status = call()
    assert status == 0
    E.set_wait_limit_ns(2_000_000)
    E.test_stall_kv_producer(tiles)
    try:
        out, status = call()
    finally:
        E.test_stall_kv_producer(-1)
        E.set_wait_limit_ns(0)
    assert status == -8 and (out[used:] == 7.0).all()
    out, status = call()
    assert status == 0 and torch.equal(out.view(torch.int16), want.view(torch.int16))


@pytest.mark.parametrize("n", [1, 2])
def test_as_many_slots_as_a_length_can_name(E, n):
    """2^31 - 1 slots, the same page of 2^20 over and over: all scores are 0 and all values 1, so every partial sum is a whole number and
    the output is 1."""
    k, v = (torch.full((1, 1, 1 << 20, 64), x, dtype=torch.bfloat16, device=DEV) for x in (0.0, 1.0))
    kv, status = E.KVStore(k, v, block_table=torch.zeros(1, 1 << 11, dtype=torch.int32, device=DEV)), torch.zeros(1, dtype=torch.int32, device=DEV)
    q = torch.ones(n, 1, 64, dtype=torch.bfloat16, device=DEV)
    for slots, want in ((2 ** 31 - 1, 0), (2 ** 31 - 1 - 300, 0)):
        status.zero_()
        out = E.eagle_chunk_attn(q, kv, _ints([slots - n]).to(DEV), _ints([0, n]).to(DEV), status=status)
        torch.cuda.synchronize()
        assert int(status.item()) == want and (out == 1).all()
    E.eagle_chunk_attn(q, kv, _ints([2 ** 31 - n]).to(DEV), _ints([0, n]).to(DEV), out, status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == -6 and (out == 0).all()
