"""Rotary positions with the write into the cache, against the 64-bit definition.

Tolerances.  bf16 results are rounded once: half a step is 2^-8 of the value.  Before that the angle is exact to 2^-25 of a turn
(2e-7 rad), sine and cosine to a few fp32 ulps and the rotation is two products and a sum in fp32: 8e-7 of amplitude * (|x| + |y|) covers
them.  e4m3 codes are half a step off at the most, 2^-4 of the value or 2^-10 below 2^-6, on top of the same fp32 error over the scale."""
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
    """Inputs on the host: one projection's rows, lengths, an empty cache (poisoned) of the asked kind."""

    def __init__(self, n, lens, hq, hkv, d, page=0, fp8=False, rotary=None, seed=0, tree=None, spare=3, rows=None):
        g = torch.Generator().manual_seed(seed)
        self.n, self.lens, self.hq, self.hkv, self.d, self.page, self.fp8, self.tree = n, lens, hq, hkv, d, page, fp8, tree
        B = len(lens)
        start = np.concatenate([[0], np.cumsum(n)])
        self.start = _ints(start.tolist())
        rows = rows if rows is not None else int(start[-1]) + 2          # two rows behind the last sequence
        lead = (B, tree) if tree else (rows,)
        self.qkv = torch.randn(*lead, hq + 2 * hkv, d, generator=g).bfloat16()
        self.q, self.k, self.v = self.qkv.split((hq, hkv, hkv), dim=-2)
        R = rotary or d
        self.freqs = torch.tensor(S.rope_frequencies(R)[0])
        need = [a + b for a, b in zip(n, lens)]
        if page:
            used = [-(-x // page) for x in need]
            pages, per = sum(used) + spare, max(max(used), 1)
            order = torch.randperm(pages, generator=g).tolist()
            self.table = torch.full((B, per), -1, dtype=torch.int32)
            for b, u in enumerate(used):
                self.table[b, :u] = _ints([order.pop() for _ in range(u)])
            shape = (pages, hkv, page, d)
        else:
            self.table, shape = None, (B, hkv, max(need) + 3, d)
        if fp8:
            self.kc, self.vc = (torch.full(shape, 0x7f, dtype=torch.uint8) for _ in range(2))
            self.ks, self.vs = (torch.rand(B, hkv, generator=g) * 0.02 + 0.002 for _ in range(2))
        else:
            self.kc, self.vc = (torch.full(shape, float("nan"), dtype=torch.bfloat16) for _ in range(2))
            self.ks = self.vs = None

    def store(self, E):
        up = lambda t: None if t is None else t.to(DEV)  # noqa: E731
        return E.KVStore(up(self.kc), up(self.vc), block_table=up(self.table), k_scale=up(self.ks), v_scale=up(self.vs))


def _values(c, t):
    return S.e4m3(t.numpy()) if c.fp8 else t.double().numpy()


def _check(c, q_out, kv, want_q, stored, amplitude, q_before, live_rows):
    got = q_out.cpu().double().numpy()
    pair = 2 * float(c.qkv.double().abs().max()) * abs(amplitude)
    for at in np.ndindex(got.shape[:-2]):
        if at in live_rows:
            err = np.abs(got[at] - want_q[at])
            assert (err <= 2.0 ** -8 * np.abs(want_q[at]) + 8e-7 * pair).all(), (at, err.max())
        else:
            assert np.array_equal(got[at], q_before[at], equal_nan=True), at
    kc, vc = c.kc.clone(), c.vc.clone()
    got_k, got_v = kv.k.cpu(), kv.v.cpu()
    for b, slot, key, value in stored:
        first, row = S.place_of(b, slot, None if c.table is None else c.table.numpy(), c.page)
        for new, whole, kept, scale in ((key, got_k, kc, c.ks), (value, got_v, vc, c.vs)):
            have = _values(c, whole[first, :, row])
            if c.fp8:
                e = np.clip(new / scale[b].double().numpy()[:, None], -448, 448)
                tol = np.maximum(2.0 ** -4 * np.abs(e), 2.0 ** -10) + 8e-7 * pair / scale[b].double().numpy()[:, None] + 2e-7 * np.abs(e)
            else:
                e, tol = new, 2.0 ** -8 * np.abs(new) + 8e-7 * pair
            assert (np.abs(have - e) <= tol).all(), (b, slot, np.abs(have - e).max())
            kept[first, :, row] = whole[first, :, row]
    # nothing else has changed
    bits = lambda t: t.view(torch.uint8)  # noqa: E731
    assert torch.equal(bits(kc), bits(got_k)) and torch.equal(bits(vc), bits(got_v))


def _run_chunk(E, c, interleaved=False, amplitude=1.0, positions=None, dense=False, q_out=None, kv=None):
    kv = kv or c.store(E)
    qkv = c.qkv.to(DEV)
    q, k, v = qkv.split((c.hq, c.hkv, c.hkv), dim=-2)
    if dense:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    if q_out is None:
        q_out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device=DEV)
    before = q_out.cpu().double().numpy()
    E.eagle_rope_append(q, k, v, kv, _ints(c.lens).to(DEV), c.start.to(DEV), c.freqs.to(DEV), q_out, interleaved=interleaved, amplitude=amplitude,
                        positions=None if positions is None else positions.to(DEV), status=status)
    torch.cuda.synchronize()
    return q_out, kv, int(status.item()), before


CHUNKS = {
    "one_token": dict(n=[1], lens=[0], hq=4, hkv=4, d=64),
    "one_far": dict(n=[3], lens=[1000003 - 3], hq=2, hkv=1, d=128, page=1 << 16),
    "ragged_paged": dict(n=[5, 0, 1, 17, 0], lens=[0, 9, 100, 31, 4], hq=12, hkv=3, d=128, page=16),
    "ragged_contiguous": dict(n=[0, 33, 2], lens=[7, 0, 250], hq=7, hkv=1, d=64),
    "part_of_the_head": dict(n=[9, 4], lens=[5, 60], hq=4, hkv=2, d=128, rotary=48, page=32),
    "smallest_part": dict(n=[6], lens=[11], hq=3, hkv=3, d=64, rotary=16),
    "fp8_paged": dict(n=[13, 1, 40], lens=[3, 77, 0], hq=8, hkv=2, d=128, fp8=True, page=32),
    "fp8_contiguous": dict(n=[2, 5], lens=[0, 12], hq=4, hkv=4, d=128, fp8=True, rotary=64),
    "many_sequences": dict(n=[i % 3 for i in range(70)], lens=[i * 5 % 40 for i in range(70)], hq=2, hkv=1, d=64, page=16),
    "wide_group": dict(n=[70], lens=[2], hq=64, hkv=8, d=128),
    "no_queries": dict(n=[4, 3], lens=[1, 2], hq=0, hkv=2, d=64),
}


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("name", list(CHUNKS))
def test_chunk_form_matches_the_definition(E, name, interleaved):
    c = Case(**CHUNKS[name], seed=len(name))
    amplitude = 1.25 if name in ("ragged_paged", "fp8_contiguous") else 1.0
    want, stored = S.rope_append(c.q, c.k, c.v, c.lens, c.freqs.numpy(), token_start=c.start, interleaved=interleaved, amplitude=amplitude)
    q_out, kv, status, before = _run_chunk(E, c, interleaved, amplitude)
    assert status == 0
    _check(c, q_out, kv, want, stored, amplitude, before, {(t,) for t in range(sum(c.n))})


def test_positions_of_their_own_and_dense_rows(E):
    c = Case([4, 7], [3, 0], 4, 2, 128, seed=5)
    positions = _ints([-5, 0, 2 ** 30, 11, 1, 1, 1, 99, 12345678, 5, 6, 0, 0])
    want, stored = S.rope_append(c.q, c.k, c.v, c.lens, c.freqs.numpy(), token_start=c.start, positions=positions)
    for dense in (False, True):
        q_out, kv, status, before = _run_chunk(E, c, positions=positions, dense=dense)
        assert status == 0
        _check(c, q_out, kv, want, stored, 1.0, before, {(t,) for t in range(11)})


def test_queries_in_place(E):
    c = Case([6, 5], [3, 0], 4, 2, 64, seed=6)
    want, stored = S.rope_append(c.q, c.k, c.v, c.lens, c.freqs.numpy(), token_start=c.start)
    q, kv = c.q.to(DEV).contiguous(), c.store(E)
    before = q.cpu().double().numpy()
    E.eagle_rope_append(q, c.k.to(DEV), c.v.to(DEV), kv, _ints(c.lens).to(DEV), c.start.to(DEV), c.freqs.to(DEV), q)
    _check(c, q, kv, want, stored, 1.0, before, {(t,) for t in range(11)})


TREES = {
    "one_node": dict(n=[1], lens=[4], tree=1, hq=2, hkv=2, d=64),
    "ragged": dict(n=[7, 0, 64, 33], lens=[0, 5, 100, 31], tree=64, hq=8, hkv=2, d=128, page=16),
    "odd": dict(n=[5, 3], lens=[2, 40], tree=5, hq=6, hkv=3, d=64),
    "fp8": dict(n=[9, 26], lens=[50, 1], tree=26, hq=8, hkv=8, d=128, fp8=True, page=32, rotary=64),
}


def _parents(n, T, seed, chain=False):
    g = np.random.default_rng(seed)
    p = np.full((len(n), T), 2 ** 30, dtype=np.int32)
    for b, m in enumerate(n):
        for i in range(m):
            p[b, i] = i - 1 if chain else g.integers(-1, i)
    return torch.tensor(p)


def _run_tree(E, c, parents, sizes, shared=False, interleaved=False):
    kv, qkv = c.store(E), c.qkv.to(DEV)
    q, k, v = qkv.split((c.hq, c.hkv, c.hkv), dim=-2)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    q_out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device=DEV)
    before = q_out.cpu().double().numpy()
    E.eagle_tree_rope_append(q, k, v, kv, _ints(c.lens).to(DEV), parents.to(DEV), c.freqs.to(DEV), q_out,
                             tree_sizes=None if sizes is None else sizes.to(DEV), shared_tree=shared, interleaved=interleaved, status=status)
    torch.cuda.synchronize()
    return q_out, kv, int(status.item()), before


@pytest.mark.parametrize("chain", [False, True])
@pytest.mark.parametrize("name", list(TREES))
def test_tree_form_matches_the_definition(E, name, chain):
    c = Case(**TREES[name], seed=len(name))
    parents, sizes = _parents(c.n, c.tree, 3, chain), _ints(c.n)
    want, stored = S.rope_append(c.q, c.k, c.v, c.lens, c.freqs.numpy(), tree_parent=parents, tree_sizes=sizes, interleaved=chain)
    q_out, kv, status, before = _run_tree(E, c, parents, sizes, interleaved=chain)
    assert status == 0
    _check(c, q_out, kv, want, stored, 1.0, before, {(b, i) for b, m in enumerate(c.n) for i in range(m)})


def test_one_tree_for_every_sequence(E):
    c = Case([9, 9, 9], [4, 0, 77], 4, 2, 64, tree=9, page=16, seed=8)
    one = _parents([9], 9, 4)
    a = _run_tree(E, c, one[0], None, shared=True)
    b = _run_tree(E, c, one.repeat(3, 1), None)
    assert a[2] == b[2] == 0 and torch.equal(a[0], b[0])
    assert torch.equal(a[1].k.view(torch.int16), b[1].k.view(torch.int16)) and torch.equal(a[1].v.view(torch.int16), b[1].v.view(torch.int16))


def test_fp8_extremes_and_not_a_number(E):
    c = Case([1], [0], 1, 1, 128, fp8=True, seed=1, rotary=16)
    c.ks.fill_(0.5)
    c.vs.fill_(0.5)
    row = torch.zeros(128)
    row[:6] = torch.tensor([1e4, -1e4, float("nan"), float("inf"), 2.0 ** -11, 1.0625])
    c.qkv[0, 2] = row.bfloat16()
    _, kv, status, _ = _run_chunk(E, c)
    got = S.e4m3(kv.v.cpu().numpy())[0, 0, 0, :6]
    # 2^-11 / 0.5 = 2^-10 lies halfway between 0 and the smallest code, 1.0625 / 0.5 = 2.125 halfway between 2 and 2.25: to even
    assert status == 0 and np.isnan(got[2]) and got[[0, 1, 3, 4, 5]].tolist() == [448.0, -448.0, 448.0, 0.0, 2.0]


# ---------------------------------------------------------------------------------------------------------------- bad inputs
def test_a_sequence_without_room_is_left_out(E):
    c = Case([3, 4, 2], [5, 6, 1], 2, 2, 64, seed=9)
    cap = c.kc.shape[2]
    for bad_len in (-1, cap - 3):
        lens = [5, bad_len, 1]
        keep = Case([3, 4, 2], [5, 6, 1], 2, 2, 64, seed=9)
        keep.lens = lens
        q_out, kv, status, before = _run_chunk(E, keep)
        assert status == -6
        got = q_out.cpu().double().numpy()
        assert (got[3:7] == 0).all()
        want, stored = S.rope_append(c.q, c.k, c.v, [5, 6, 1], c.freqs.numpy(), token_start=c.start)
        before[3:7] = 0
        _check(keep, q_out, kv, want, [s for s in stored if s[0] != 1], 1.0, before, {(t,) for t in (0, 1, 2, 7, 8)})


def test_a_page_outside_the_pool_is_not_written(E):
    c = Case([20, 2], [0, 3], 2, 2, 64, page=16, seed=10)
    for bad in (-1, c.kc.shape[0], 2 ** 31 - 1):
        c.table[0, 1] = bad
        want, stored = S.rope_append(c.q, c.k, c.v, c.lens, c.freqs.numpy(), token_start=c.start)
        q_out, kv, status, before = _run_chunk(E, c)
        assert status == -11
        _check(c, q_out, kv, want, [s for s in stored if not (s[0] == 0 and s[1] >= 16)], 1.0, before, {(t,) for t in range(22)})


def test_starts_that_descend_are_reported(E):
    c = Case([4, 4], [0, 0], 2, 2, 64, seed=11)
    c.start = _ints([0, 6, 4])
    q_out, kv, status, before = _run_chunk(E, c)
    assert status == -6
    c.start = _ints([0, 4, 99])
    assert _run_chunk(E, c)[2] == -6


@pytest.mark.parametrize("what", ["parent", "size"])
def test_an_invalid_tree_is_reported_and_zeroed(E, what):
    c = Case([5, 6], [3, 2], 2, 2, 64, tree=6, seed=12)
    parents, sizes = _parents(c.n, 6, 5), _ints(c.n)
    want, stored = S.rope_append(c.q, c.k, c.v, c.lens, c.freqs.numpy(), tree_parent=parents, tree_sizes=sizes)
    if what == "parent":
        parents[0, 3] = 3
    else:
        sizes[0] = 7
    q_out, kv, status, before = _run_tree(E, c, parents, sizes)
    assert status == -5
    before[0, :5 if what == "parent" else 6] = 0
    _check(c, q_out, kv, want, [s for s in stored if s[0] == 1], 1.0, before, {(1, i) for i in range(6)})


def test_replayed_from_a_graph_on_another_stream(E):
    c = Case([5, 9], [0, 30], 4, 2, 128, page=16, seed=13)
    kv, qkv, lens, start, freqs = c.store(E), c.qkv.to(DEV), _ints(c.lens).to(DEV), c.start.to(DEV), c.freqs.to(DEV)
    q, k, v = qkv.split((c.hq, c.hkv, c.hkv), dim=-2)
    q_out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device=DEV)
    before = q_out.cpu().double().numpy()
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        E.eagle_rope_append(q, k, v, kv, lens, start, freqs, q_out)
    fresh = torch.randn(c.qkv.shape, generator=torch.Generator().manual_seed(99)).bfloat16()
    qkv.copy_(fresh)
    graph.replay()
    torch.cuda.synchronize()
    c.qkv = fresh
    c.q, c.k, c.v = fresh.split((c.hq, c.hkv, c.hkv), dim=-2)
    want, stored = S.rope_append(c.q, c.k, c.v, c.lens, c.freqs.numpy(), token_start=c.start)
    _check(c, q_out, kv, want, stored, 1.0, before, {(t,) for t in range(14)})


def test_rows_of_their_own_are_asked_for(E):
    c = Case([3, 2], [1, 4], 4, 2, 64, seed=14, rows=5)
    q, k, v, kv, lens, start, freqs = c.q.to(DEV), c.k.to(DEV), c.v.to(DEV), c.store(E), _ints(c.lens).to(DEV), c.start.to(DEV), c.freqs.to(DEV)
    for bad in (q[:1].expand(5, -1, -1), q.transpose(0, 1).contiguous().transpose(0, 1), q[:, :, ::2], q.float(), q[:4]):
        with pytest.raises(E.EagleError):
            E.eagle_rope_append(bad, k, v, kv, lens, start, freqs)
    with pytest.raises(E.EagleError):
        E.eagle_rope_append(q, k, v[:, :1], kv, lens, start, freqs)
    with pytest.raises(E.EagleError):
        E.eagle_rope_append(q, k, v, kv, lens, start, freqs.float())
    # every other row of a larger tensor is a constant stride
    wide = torch.randn(10, 4, 64, device=DEV).bfloat16()
    wide[::2] = q
    a = E.eagle_rope_append(wide[::2], k, v, kv, lens, start, freqs)
    assert torch.equal(a, E.eagle_rope_append(q.contiguous(), k, v, kv, lens, start, freqs))


def test_thousands_of_sequences(E):
    """(The search for a token's sequence takes a third round beyond 1024 of them.)"""
    c = Case([(i * 7 + i // 900) % 3 for i in range(2500)], [(i * 13) % 29 for i in range(2500)], 1, 1, 64, page=16, seed=31)
    want, stored = S.rope_append(c.q, c.k, c.v, c.lens, c.freqs.numpy(), token_start=c.start)
    q_out, kv, status, before = _run_chunk(E, c)
    assert status == 0
    _check(c, q_out, kv, want, stored, 1.0, before, {(t,) for t in range(sum(c.n))})


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("page", [0, 256])
def test_caches_of_more_than_2_31_elements(E, page, fp8):
    """The same tokens at the far end of a large cache: the same bits there."""
    c = Case([2, 40, 3], [300, 7, 511], 4, 8, 128, page=page, fp8=fp8, seed=32)
    q_small, kv, status, _ = _run_chunk(E, c)
    assert status == 0
    up = lambda t: None if t is None else t.to(DEV)  # noqa: E731
    if page:
        far, shape = 9000 - c.kc.shape[0], (9000, 8, page, 128)          # 2.4e9 elements
    else:
        far, shape = 0, (3, 8, 1000000, 128)
    big_k, big_v = (torch.zeros(shape, dtype=c.kc.dtype, device=DEV) for _ in range(2))
    part = (slice(far, None),) if page else (slice(None), slice(None), slice(0, c.kc.shape[2]))
    big_k[part], big_v[part] = up(c.kc), up(c.vc)
    table = up(torch.where(c.table >= 0, c.table + far, c.table)) if page else None
    big = E.KVStore(big_k, big_v, block_table=table, k_scale=up(c.ks), v_scale=up(c.vs))
    q_big, _, status, _ = _run_chunk(E, c, kv=big)
    bits = lambda t: t.contiguous().view(torch.uint8)  # noqa: E731
    assert status == 0 and torch.equal(bits(q_small), bits(q_big))
    assert torch.equal(bits(kv.k), bits(big_k[part])) and torch.equal(bits(kv.v), bits(big_v[part]))
    rest = (slice(0, far),) if page else (slice(None), slice(None), slice(c.kc.shape[2], None))
    assert not bool(big_k[rest].any()) and not bool(big_v[rest].any())


def _nearest_codes(x):
    """The e4m3 code nearest to each fp32 value (a tie goes to the even code), by search in the table of values."""
    table = S.e4m3(np.arange(127))
    x = np.asarray(x, dtype=np.float64)
    lo = np.clip(np.searchsorted(table, np.abs(x), side="right") - 1, 0, 125)
    d_lo, d_hi = np.abs(x) - table[lo], table[lo + 1] - np.abs(x)
    code = np.where((d_hi < d_lo) | ((d_hi == d_lo) & (lo % 2 == 1)), lo + 1, lo)
    return (code | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def test_fp8_codes_are_the_nearest_to_the_fp32_quotient(E):
    """Values at the middle between two codes, times scales that are no powers of two (products exact in bf16), and others; position 0 turns
    by nothing, so keys are compared too."""
    B = 24
    c = Case([1] * B, [0] * B, 1, 4, 128, fp8=True, seed=33, rows=B)
    c.qkv[:, 1:] *= 3
    ties = np.array([(2 * m + 1) / 16 * 2.0 ** e for m in range(8, 16) for e in range(-6, 8)] + [(2 * m + 1) * 2.0 ** -10 for m in range(8)] + [-1.0625, -2.125] * 4)
    assert len(ties) == 128
    for b in range(12):
        for h, odd in enumerate((3, 5, 7, 3 * 2.0 ** -40)):
            scale = odd * 2.0 ** -(b + 2)
            c.ks[b, h] = c.vs[b, h] = scale
            for row in (1 + h, 5 + h):
                c.qkv[b, row] = torch.tensor(ties * scale).bfloat16()
                assert (c.qkv[b, row].double().numpy() == ties * scale).all()
    _, kv, status, _ = _run_chunk(E, c)
    assert status == 0
    for rows, cache, scale in ((slice(1, 5), kv.k, c.ks), (slice(5, 9), kv.v, c.vs)):
        x = c.qkv[:, rows].float().numpy() / scale.numpy()[:, :, None]
        assert x.dtype == np.float32 and np.abs(x).max() > 448
        want, got = _nearest_codes(x), cache.cpu().numpy()[:, :, 0]
        assert (got == want).all(), (got != want).sum()


@pytest.mark.parametrize("tree", [False, True])
def test_a_lone_row_may_have_any_stride(E, tree):
    """Heads first, tokens second, as attention layers often keep them: with one token its heads are dense, and there is no second row."""
    c = Case([1], [5], 4, 2, 64, seed=34, rows=1, tree=1 if tree else None)
    lens, freqs = _ints(c.lens).to(DEV), c.freqs.to(DEV)
    rest = (lens, _ints([[-1]]).to(DEV) if tree else c.start.to(DEV), freqs)
    call = E.eagle_tree_rope_append if tree else E.eagle_rope_append
    dense = [t.to(DEV).contiguous() for t in (c.q, c.k, c.v)]

    def by_heads(t):
        t = t.transpose(-3, -2)
        return torch.empty(t.shape, dtype=t.dtype, device=DEV).copy_(t).transpose(-3, -2)

    heads_first = [by_heads(t) for t in dense]
    assert all(t.stride(-3) == 64 for t in heads_first)
    a, b = c.store(E), c.store(E)
    out_a, out_b = call(*dense, a, *rest), call(*heads_first, b, *rest)
    assert torch.equal(out_a, out_b) and all(torch.equal(x.view(torch.int16), y.view(torch.int16)) for x, y in ((a.k, b.k), (a.v, b.v)))
    # the queries turned in place, a lone row of a projection's output among them
    for q in (heads_first[0], c.qkv.to(DEV)[..., :4, :]):
        assert q.is_contiguous() and torch.equal(call(q, dense[1], dense[2], c.store(E), *rest, q_out=q), out_a)
    if not tree:
        none = [by_heads(t)[:0] for t in dense]
        assert call(*none, c.store(E), lens, _ints([0, 0]).to(DEV), freqs).shape == (0, 4, 64)


@pytest.mark.parametrize("scale", [2.0 ** -126, 2.0 ** -100, 1.0, 3.0, 2.0 ** 100])
def test_fp8_codes_of_zeros_infinities_and_extreme_scales(E, scale):
    """The sign of a zero, values whose quotient leaves fp32's range, scales at the edge of the normal numbers."""
    c = Case([1] * 3, [0] * 3, 1, 2, 128, fp8=True, seed=35, rows=3)
    c.ks.fill_(scale), c.vs.fill_(scale)
    c.qkv[:, 1:] = (c.qkv[:, 1:].double() * 100 * scale).bfloat16()
    c.qkv[:, 3, :6] = torch.tensor([float("inf"), -float("inf"), 0.0, -0.0, 3e38, -3e38]).bfloat16()
    _, kv, status, _ = _run_chunk(E, c)
    assert status == 0
    for rows, cache in ((slice(1, 3), kv.k), (slice(3, 5), kv.v)):
        with np.errstate(over="ignore"):
            x = c.qkv[:, rows].float().numpy() / np.float32(scale)
        assert (_nearest_codes(x) == cache.cpu().numpy()[:, :, 0]).all()
