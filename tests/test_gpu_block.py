"""Appends into a block-scaled cache against the 64-bit definition.

Scales have to be equal: powers of two of a maximum that is taken in fp32 (2^-24), far from a border with these seeds.  A code has to be the
nearest one to x / scale, up to the fp32 terms of x: a rotation is two products and a sum of terms of at most sqrt(2) amplitude |x|, sines and
cosines good to 2^-22, so 1e-6 of the pair's magnitude is ample.  Queries are rounded to bf16 once (2^-8 relative) on top of that."""
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
    def __init__(self, n, lens, hq, hkv, block, page=0, tree=None, rotary=128, interleaved=False, amplitude=1.0, seed=0, spare=3, positions=False,
                 strided=False, scale=(-3, 3)):
        g = torch.Generator().manual_seed(seed)
        self.n, self.lens, self.block, self.page, self.tree, B = n, lens, block, page, tree, len(n)
        self.kw = {"interleaved": interleaved, "amplitude": amplitude}
        need = [a + b for a, b in zip(n, lens)]
        if page:
            used = [-(-x // page) for x in need]
            order = torch.randperm(sum(used) + 2, generator=g).tolist()
            self.table = torch.full((B, max(max(used), 1) + 1), -1, dtype=torch.int32)
            for b, u in enumerate(used):
                self.table[b, :u] = _ints([order.pop() for _ in range(u)])
            shape = (sum(used) + 2, hkv, page, 128)
        else:
            self.table, shape = None, (B, hkv, -(-(max(need) + 1) // block) * block, 128)
        self.k, self.v = (torch.randint(0, 256, shape, generator=g, dtype=torch.uint8) for _ in range(2))
        blocks = (*shape[:2], shape[2] // block)
        self.ks, self.vs = (torch.exp2(torch.randint(-11, -5, blocks, generator=g).float()) for _ in range(2))
        T = max(n) if tree else 0
        rows = (B, T) if tree else (sum(n) + spare,)
        # magnitudes that differ from head to head and token to token, so that scales do
        size = torch.exp2(torch.randint(*scale, (*rows, hq + 2 * hkv, 1), generator=g).float())
        self.qkv = (torch.randn(*rows, hq + 2 * hkv, 128, generator=g) * size).bfloat16()
        self.split, self.strided = (hq, hkv, hkv), strided
        self.freqs = torch.pow(torch.tensor(10000.0, dtype=torch.float64), -2.0 * torch.arange(rotary // 2, dtype=torch.float64) / rotary)
        if tree:
            self.order = torch.zeros(B, T, dtype=torch.int32)
            for b, m in enumerate(n):
                for i in range(m):
                    self.order[b, i] = int(torch.randint(-1, i, (1,), generator=g)) if tree == "random" or i == 0 else i - 1
            self.extra = {"tree_sizes": _ints(n)}
        else:
            self.order = _ints(np.concatenate([[0], np.cumsum(n)]).tolist())
            self.extra = {"positions": torch.randint(0, 1 << 20, rows, generator=g, dtype=torch.int32)} if positions else {}

    def run(self, E):
        up = lambda t: None if t is None else t.to(DEV)  # noqa: E731
        self.got = [up(t).clone() for t in (self.k, self.v, self.ks, self.vs)]
        k, v, ks, vs = self.got
        store = E.KVStore(k, v, block_table=up(self.table), k_scale=ks, v_scale=vs, block_size=self.block)
        qkv = up(self.qkv)
        q, kk, vv = qkv.split(self.split, dim=-2)
        if not self.strided:
            q, kk, vv = q.contiguous(), kk.contiguous(), vv.contiguous()
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        q_out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device=DEV)
        fn = E.eagle_tree_block_append if self.tree else E.eagle_block_append
        fn(q, kk, vv, store, up(_ints(self.lens)), up(self.order), up(self.freqs), q_out, status=status, **{n: up(t) for n, t in self.extra.items()}, **self.kw)
        torch.cuda.synchronize()
        return q_out.cpu(), int(status.item())

    def want(self):
        q, k, v = self.qkv.split(self.split, dim=-2)
        cache = [t.numpy() for t in (self.k, self.v, self.ks, self.vs)]
        order = {"tree_parent": self.order} if self.tree else {"token_start": self.order}
        return S.block_append(q, k, v, cache, self.lens, self.freqs.numpy(), self.block, block_table=self.table, **order, **self.extra, **self.kw)

    def check(self, E):
        q, status = self.run(E)
        assert status == 0
        rows, res = self.want()
        gone = np.isnan(rows)
        got = q.double().numpy()
        assert (got[gone] == 7.0).all(), "rows outside the sequences have changed"
        pair = np.abs(rows).max(-1, keepdims=True)
        assert (np.abs(got - rows) <= 2.0 ** -8 * np.abs(rows) + 1e-6 * pair)[~gone].all()
        for (values, codes, scales), c, s in zip(res, self.got[:2], self.got[2:]):
            c, s = c.cpu().numpy(), s.cpu().double().numpy()
            assert np.array_equal(s, scales), "scales"
            new = ~np.isnan(values)
            assert np.array_equal(c[~new], codes[~new]), "codes that should not change, or older ones by a larger scale"
            y, best = values[new], S.e4m3(S.nearest_code(values[new]))
            here = S.e4m3(c[new])
            slack = 1e-6 * np.broadcast_to(np.nanmax(np.abs(np.where(new, values, 0)), -1, keepdims=True), values.shape)[new]
            assert (np.abs(here - np.clip(y, -448, 448)) <= np.abs(best - np.clip(y, -448, 448)) + 2 * slack).all(), "codes that are not the nearest"


CHUNKS = {
    "one_token": dict(n=[1], lens=[70], hq=4, hkv=4, block=64, spare=0),
    "one_token_first": dict(n=[1], lens=[0], hq=1, hkv=1, block=16, spare=0),
    "block_edges": dict(n=[1, 1, 1, 2, 3, 16, 17], lens=[15, 16, 17, 15, 31, 16, 15], hq=8, hkv=2, block=16),
    "odd": dict(n=[0, 5, 1, 0, 77, 33], lens=[9, 3, 64, 0, 131, 0], hq=6, hkv=3, block=32, page=64, strided=True),
    "long": dict(n=[700, 301], lens=[45, 0], hq=8, hkv=8, block=128, page=128, interleaved=True, amplitude=1.2),
    "part_turned": dict(n=[130, 7], lens=[3, 60], hq=4, hkv=1, block=64, page=256, rotary=48, strided=True),
    "part_turned_neighbours": dict(n=[40, 7], lens=[3, 60], hq=2, hkv=2, block=16, page=16, rotary=16, interleaved=True),
    "positions": dict(n=[20, 40], lens=[8, 0], hq=4, hkv=2, block=32, positions=True),
    "many_singles": dict(n=[1] * 300, lens=[(i * 37) % 200 for i in range(300)], hq=2, hkv=1, block=32, page=32, spare=0),
    "many_singles_and_spare_rows": dict(n=[1] * 300, lens=[(i * 37) % 200 for i in range(300)], hq=2, hkv=1, block=32, page=32),
    "chunks_among_empty_sequences": dict(n=[37, 0, 3, 1, 20] + [0] * 60, lens=[5, 9, 30, 0, 64] + [7] * 60, hq=4, hkv=3, block=16, page=32, spare=0, strided=True),
    "singles_with_positions": dict(n=[1, 1, 1, 2], lens=[15, 16, 200, 63], hq=2, hkv=5, block=64, positions=True, interleaved=True, rotary=64, spare=0),
    "many_heads": dict(n=[9, 80], lens=[5, 64], hq=64, hkv=32, block=64),
    "no_queries": dict(n=[9, 80], lens=[5, 64], hq=0, hkv=2, block=64),
    "ragged": dict(n=[(i * 29) % 90 for i in range(40)], lens=[(i * 53) % 150 for i in range(40)], hq=4, hkv=2, block=64, page=64, strided=True),
    "small_and_large": dict(n=[300, 20], lens=[7, 100], hq=1, hkv=2, block=16, scale=(-60, 100)),
}


@pytest.mark.parametrize("name", CHUNKS)
def test_chunks_match_the_definition(E, name):
    Case(**CHUNKS[name], seed=len(name)).check(E)


TREES = {
    "one_node": dict(n=[1, 1], lens=[0, 33], hq=4, hkv=4, block=16),
    "mixed": dict(n=[5, 64, 0, 17, 33], lens=[3, 60, 9, 0, 16], hq=8, hkv=2, block=16, page=32, strided=True),
    "wide_blocks": dict(n=[64, 30, 1], lens=[127, 100, 5], hq=4, hkv=4, block=128, page=128, interleaved=True),
    "chains": dict(n=[64, 12], lens=[1, 63], hq=6, hkv=3, block=64, rotary=64, amplitude=1.3),
    "many": dict(n=[(i * 13) % 40 for i in range(120)], lens=[(i * 31) % 300 for i in range(120)], hq=4, hkv=1, block=32, page=64),
}


@pytest.mark.parametrize("name", TREES)
def test_trees_match_the_definition(E, name):
    Case(**TREES[name], tree="chain" if name == "chains" else "random", seed=len(name)).check(E)


def test_one_tree_for_every_sequence(E):
    c = Case([12, 12, 12], [0, 20, 61], 4, 2, 32, page=32, tree="random", seed=3)
    c.order[:] = c.order[0].clone()
    c.check(E)
    per_sequence = [t.clone() for t in c.got]
    c.order, c.extra = c.order[0].contiguous(), {"tree_sizes": _ints([12])}
    c.kw["shared_tree"] = True
    _, status = c.run(E)
    assert status == 0 and all(torch.equal(a, b) for a, b in zip(c.got, per_sequence))


def test_infinities_nan_and_zeros(E):
    """Only finite magnitudes count for a scale; infinite ones become 448, NaN stays NaN, a block of zeros takes 2^-40."""
    c = Case([64], [0], 1, 2, 16, seed=4)
    q, k, v = c.qkv.split(c.split, dim=-2)
    v[0, 0, 3], v[1, 0, 4], v[2, 0, 5] = float("inf"), float("-inf"), float("nan")
    v[16:32], k[16:32] = 0.0, 0.0
    v[32:48] = float("nan")
    v[48:, 0] = torch.finfo(torch.bfloat16).max
    c.run(E)
    codes, scales = c.got[1].cpu(), c.got[3].cpu()
    assert codes[0, 0, 0, 3] == 0x7e and codes[0, 0, 1, 4] == 0xfe and codes[0, 0, 2, 5] & 0x7f == 0x7f
    assert scales[0, :, 1].eq(2.0 ** -40).all() and c.got[2].cpu()[0, :, 1].eq(2.0 ** -40).all() and codes[0, :, 16:32].eq(0).all()
    assert scales[0, :, 2].eq(2.0 ** -40).all() and (codes[0, :, 32:48] & 0x7f).eq(0x7f).all()
    finite = v[:16, 0].float()[torch.isfinite(v[:16, 0].float())].abs().max().item()
    assert scales[0, 0, 0] == S.block_scale(finite) and scales[0, 0, 3] == 2.0 ** 120


def test_a_scale_that_is_no_power_of_two_stays_while_it_is_large_enough(E):
    c = Case([10], [20], 1, 1, 64, seed=5, scale=(0, 1))
    c.ks[:], c.vs[:] = 0.3, 1e-4
    q, status = c.run(E)
    rows, res = c.want()
    assert status == 0 and c.got[2][0, 0, 0] == c.ks[0, 0, 0] and c.got[3][0, 0, 0] > 1e-4
    values, codes, scales = res[0]
    new = ~np.isnan(values)
    y = np.where(new, values * np.float64(0.3) / np.float64(np.float32(0.3)), 0)[new]      # the scale is the fp32 number
    got = S.e4m3(c.got[0].cpu().numpy()[new])
    assert (np.abs(got - y) <= np.abs(S.e4m3(S.nearest_code(y)) - y) + 1e-5).all()
    older = S.e4m3(c.got[1].cpu().numpy()[0, 0, :20]) * float(c.got[3][0, 0, 0])
    was = S.e4m3(c.v.numpy()[0, 0, :20]) * np.float64(np.float32(1e-4))
    ok = ~np.isnan(was)
    # half a step of the new code (2^-4 of it), or of the smallest one (2^-10)
    assert (np.abs(older - was)[ok] <= 2.0 ** -4 * np.abs(was[ok]) + 2.0 ** -10 * float(c.got[3][0, 0, 0]) + 1e-9).all()


def test_token_by_token_is_like_at_once(E):
    """A block filled by single tokens ends with the scale that the whole block would get, and codes within one more rounding of the value."""
    n, block = 64, 32
    whole = Case([n], [0], 1, 2, block, seed=6, spare=0)
    whole.run(E)
    step = Case([1], [0], 1, 2, block, seed=6, spare=0)
    k, v = whole.k, whole.v
    step.k, step.v, step.ks, step.vs = k.clone(), v.clone(), whole.ks.clone(), whole.vs.clone()
    for i in range(n):
        step.qkv, step.lens = whole.qkv[i:i + 1].contiguous(), [i]
        step.run(E)
        step.k, step.v, step.ks, step.vs = (t.cpu() for t in step.got)
    for a, b, sa, sb in ((whole.got[0], step.got[0], whole.got[2], step.got[2]), (whole.got[1], step.got[1], whole.got[3], step.got[3])):
        assert torch.equal(sa[:, :, :n // block], sb[:, :, :n // block])
        x, y = S.e4m3(a.cpu().numpy())[0, :, :n], S.e4m3(b.cpu().numpy())[0, :, :n]
        # halving a code loses bits only below 2^-6 of the code's range: half a step there is 2^-10, twice that with several steps
        assert np.abs(x - y).max() <= 2.0 ** -9


def test_refused_sequences_and_pages(E):
    c = Case([4, 5, 6], [10, 30, 2], 4, 2, 16, page=16, seed=7)
    c.lens = [10, -1, 2]
    q, status = c.run(E)
    assert status == -6 and (q[4:9] == 0).all() and not (q[:4] == 0).all()
    assert (q[15:] == 7).all()
    c = Case([4, 5, 6], [10, 30, 2], 4, 2, 16, page=16, seed=7)
    c.lens = [10, c.table.shape[1] * 16 - 4, 2]
    q, status = c.run(E)
    assert status == -6 and (q[4:9] == 0).all()
    c = Case([4, 5, 6], [10, 30, 2], 4, 2, 16, page=16, seed=7)
    bad = int(c.table[1, 2])
    c.table[1, 2] = 1 << 20                                  # slots 32 .. 34 of sequence 1
    before = [t.clone() for t in (c.k, c.ks)]
    q, status = c.run(E)
    assert status == -11 and torch.equal(c.got[0][bad].cpu(), before[0][bad]) and torch.equal(c.got[2][bad].cpu(), before[1][bad])
    c = Case([4, 5, 6], [10, 30, 2], 4, 2, 16, page=16, tree="random", seed=7)
    c.order[1, 2] = 2
    q, status = c.run(E)
    assert status == -5 and (q[1, :5] == 0).all() and (q[1, 5:] == 7).all() and (q[0, 4:] == 7).all()
    c = Case([4, 5, 6], [10, 30, 2], 4, 2, 16, page=16, tree="random", seed=7)
    c.lens = [10, 1000, 2]
    q, status = c.run(E)
    assert status == -6 and (q[1, :5] == 0).all()
    c = Case([1, 1, 1], [10, 32, 2], 4, 2, 16, page=16, seed=7, spare=0)
    bad = int(c.table[1, 2])
    c.table[1, 2] = -3
    before = [t.clone() for t in (c.k, c.ks)]
    q, status = c.run(E)
    assert status == -11 and torch.equal(c.got[0][bad].cpu(), before[0][bad]) and torch.equal(c.got[2][bad].cpu(), before[1][bad])
    c.lens = [10, -1, 2]
    q, status = c.run(E)
    assert status == -6 and (q[1] == 0).all() and not (q[0] == 0).all()
    c = Case([4, 5, 6], [10, 30, 2], 4, 2, 16, seed=7)
    c.order = _ints([0, 9, 4, 15])                           # starts that descend
    q, status = c.run(E)
    assert status == -6


def test_commit_moves_codes_between_a_trees_blocks(E):
    """After a tree's append its blocks share a scale: the accepted path is committed as bytes and stands for the same values."""
    c = Case([40, 33], [30, 9], 4, 2, 16, page=32, tree="chain", seed=8)
    c.run(E)
    k, v, ks, vs = c.got
    path = torch.full((2, 40), -1, dtype=torch.int32)
    path[0, :5], path[1, :3] = _ints([0, 3, 17, 30, 39]), _ints([2, 20, 32])
    was = [S.e4m3(x.cpu().numpy()) * s.cpu().double().numpy().repeat(16, -1)[..., None] for x, s in ((k, ks), (v, vs))]
    new, _ = E.eagle_tree_commit_paged(k.view(torch.bfloat16), v.view(torch.bfloat16), c.table.to(DEV), _ints(c.lens).to(DEV), path.to(DEV), 40)
    torch.cuda.synchronize()
    now = [S.e4m3(x.cpu().numpy()) * s.cpu().double().numpy().repeat(16, -1)[..., None] for x, s in ((k, ks), (v, vs))]
    at = lambda x, b, slot: x[int(c.table[b, slot // 32]), :, slot % 32]  # noqa: E731
    for b, p in enumerate(([0, 3, 17, 30, 39], [2, 20, 32])):
        assert int(new[b]) == c.lens[b] + len(p)
        for j, m in enumerate(p):
            for x, y in zip(was, now):
                assert np.array_equal(at(x, b, c.lens[b] + m), at(y, b, c.lens[b] + j), equal_nan=True)


def test_replayed_from_a_graph(E):
    c = Case([3, 70, 1], [5, 64, 31], 4, 2, 32, page=32, seed=9)
    c.run(E)
    want = [t.clone() for t in c.got]
    k, v, ks, vs = (t.to(DEV) for t in (c.k, c.v, c.ks, c.vs))
    store = E.KVStore(k, v, block_table=c.table.to(DEV), k_scale=ks, v_scale=vs, block_size=32)
    q, kk, vv = (t.contiguous() for t in c.qkv.to(DEV).split(c.split, dim=-2))
    lens, order, freqs, out = _ints(c.lens).to(DEV), c.order.to(DEV), c.freqs.to(DEV), torch.empty_like(q)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        E.eagle_block_append(q, kk, vv, store, lens, order, freqs, out)
    for _ in range(2):                                       # (the second replay finds the scales grown already)
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((ks, vs), want[2:])) and torch.equal(k, want[0]) and torch.equal(v, want[1])


@pytest.mark.parametrize("tree", [None, "random"])
def test_pages_at_the_far_end_of_a_large_pool(E, tree):
    """Offsets that pass 32 bits: the same sequences in the last pages of a large pool give the same codes and scales."""
    case = Case([20, 1, 50], [70, 5, 130], 4, 4, 16, page=128, tree=tree)
    q, status = case.run(E)
    assert status == 0
    near = [t.cpu() for t in case.got]
    pages = 70000                                            # of 64 KB: more than 2^32 bytes
    far = pages - case.k.shape[0]
    assert far * case.k[0].numel() > 2 ** 32
    big = []
    for t in (case.k, case.v, case.ks, case.vs):
        big.append(torch.empty(pages, *t.shape[1:], dtype=t.dtype, device=DEV))
        big[-1][far:] = t.to(DEV)
    store = E.KVStore(big[0], big[1], block_table=torch.where(case.table >= 0, case.table + far, case.table).to(DEV), k_scale=big[2], v_scale=big[3], block_size=16)
    state = torch.zeros(1, dtype=torch.int32, device=DEV)
    a, b, c = (t.contiguous().to(DEV) for t in case.qkv.split(case.split, dim=-2))
    fn = E.eagle_tree_block_append if tree else E.eagle_block_append
    got = fn(a, b, c, store, _ints(case.lens).to(DEV), case.order.to(DEV), case.freqs.to(DEV), torch.full(a.shape, 7.0, dtype=torch.bfloat16, device=DEV), status=state,
             **{n: t.to(DEV) for n, t in case.extra.items()})
    assert int(state.item()) == 0 and torch.equal(got.cpu(), q)
    for t, want in zip(big, near):
        assert torch.equal(t[far:].cpu(), want)


@pytest.mark.parametrize("form", ["chunks", "singles", "trees"])
def test_older_codes_by_a_scale_that_is_no_power_of_two(E, form):
    """Stored again, an older code is the nearest one to value(code) * old / new, also where that product lies next to a middle between two codes: old scales are
    quotients of small numbers, rounded to fp32, so that products of codes with them do (1.7 times a code is off a middle by a rounding of 1.7)."""
    B = 40
    n, lens = [1 if form == "singles" else 9] * B, [37 + i % 20 for i in range(B)]
    c = Case(n, lens, 1, 3, 64, tree="random" if form == "trees" else None, seed=10, scale=(0, 1), spare=0)
    g = torch.Generator().manual_seed(23)
    for s in (c.ks, c.vs):
        num, den = (torch.randint(lo, hi, s.shape, generator=g).double() for lo, hi in ((17, 64), (8, 16)))
        s[:] = (num / den * torch.exp2(torch.randint(-14, -8, s.shape, generator=g).double())).float()
    c.check(E)
    assert (c.got[2].cpu() > c.ks).float().mean() > 0.2      # (they have grown)
