"""Sampling against the 64-bit definition.

Which tokens stay and which one is drawn have to be equal: weights are fp64 (2^-45) and sums are integers of 2^-43 or less of the largest weight, so
over 10^5 tokens a border is good to 1e-10 of the sum, and a draw closer to one than 1e-9 (none is, with these seeds) would not be compared.
Probabilities are fp32 roundings (2^-24 relative) of numbers good to 1e-10 relative."""
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


def _run(E, z, u=None, num_rows=None, probs=True, **kw):
    up = lambda t: None if t is None else t.to(DEV)  # noqa: E731
    B, R, V = z.shape
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    tokens = torch.full((B, R), -7, dtype=torch.int32, device=DEV) if u is not None else None
    out = torch.full((B, R, V), 7.0, device=DEV) if probs else None
    E.eagle_sample(up(z), up(u), tokens, out, num_rows=up(num_rows), status=status, **{n: up(t) for n, t in kw.items()})
    torch.cuda.synchronize()
    return None if tokens is None else tokens.cpu(), None if out is None else out.cpu(), int(status.item())


def _check(z, u, tokens, probs, num_rows=None, **kw):
    B, R, V = z.shape
    zz = z.float().numpy()
    for b in range(B):
        rows = R if num_rows is None else int(num_rows[b])
        for r in range(R):
            if r >= rows:
                assert tokens is None or int(tokens[b, r]) == -7
                assert probs is None or (probs[b, r] == 7.0).all()
                continue
            t, p, margin = S.sample(zz[b, r], None if u is None else float(u[b, r]), **{n: x[b].item() for n, x in kw.items()})
            if probs is not None:
                got = probs[b, r].double().numpy()
                assert ((got > 0) == (p > 1e-44)).all() or (np.abs(got - p) < 1e-40)[(got > 0) != (p > 1e-44)].all(), (b, r, "another set")
                assert (np.abs(got - p) <= (2.0 ** -24 + 1e-9) * p + 1e-44).all(), (b, r)
            if tokens is not None and margin > 1e-9:
                assert int(tokens[b, r]) == t, (b, r, int(tokens[b, r]), t, margin)


def _params(g, B, V):
    rand = lambda: torch.rand(B, generator=g)  # noqa: E731
    return {"temperature": torch.where(rand() < 0.2, 0.0, 0.3 + 1.2 * rand()), "top_k": torch.where(rand() < 0.3, 0.0, torch.exp(rand() * np.log(V))).int(),
            "top_p": torch.where(rand() < 0.3, 1.0, 0.2 + 0.8 * rand()), "min_p": torch.where(rand() < 0.5, 0.0, 0.2 * rand())}


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("B,R,V", [(8, 1, 1), (8, 2, 2), (9, 3, 37), (16, 2, 1000), (12, 3, 2047), (6, 2, 4099), (24, 2, 32000), (8, 1, 50257), (4, 1, 129537),
                                   (700, 1, 33)])
def test_matches_the_definition(E, B, R, V, bf16):
    g = torch.Generator().manual_seed(B * 131 + R * 17 + V)
    z = torch.randn(B, R, V, generator=g) * 3
    z = z.bfloat16() if bf16 else z
    u = torch.rand(B, R, generator=g)
    kw = _params(g, B, V)
    n = torch.randint(0, R + 1, (B,), generator=g, dtype=torch.int32)
    tokens, probs, status = _run(E, z, u, n, **kw)
    assert status == 0
    _check(z, u, tokens, probs, n, **kw)


@pytest.mark.parametrize("name", ["temperature", "top_k", "top_p", "min_p"])
def test_each_filter_alone(E, name):
    g = torch.Generator().manual_seed(5)
    B, V = 40, 5003
    z, u = torch.randn(B, 1, V, generator=g) * 2.5, torch.rand(B, 1, generator=g)
    values = {"temperature": torch.linspace(0.05, 8.0, B), "top_k": torch.arange(-1, B - 1).int() * 17, "top_p": torch.linspace(-0.1, 1.1, B),
              "min_p": torch.linspace(-0.1, 1.2, B)}[name]
    tokens, probs, status = _run(E, z, u, **{name: values})
    assert status == 0
    _check(z, u, tokens, probs, **{name: values})
    only, _, _ = _run(E, z, u, probs=False, **{name: values})
    _, alone, _ = _run(E, z, None, **{name: values})
    assert torch.equal(only, tokens) and torch.equal(alone, probs)


def test_ties_go_to_the_lowest_index(E):
    """Few values, many times each: the cut falls among equal ones."""
    g = torch.Generator().manual_seed(6)
    B, V = 48, 9001
    z = torch.randint(-3, 3, (B, 1, V), generator=g).float() * 0.5
    z[::3] = 1.25                                            # all equal
    u = torch.rand(B, 1, generator=g)
    kw = {"top_k": torch.randint(1, V, (B,), generator=g).int(), "top_p": torch.rand(B, generator=g), "temperature": torch.rand(B, generator=g) + 0.2}
    for names in (["top_k"], ["top_p"], ["top_k", "top_p", "temperature"], []):
        some = {n: kw[n] for n in names}
        tokens, probs, _ = _run(E, z, u, **some)
        _check(z, u, tokens, probs, **some)
    greedy = {"temperature": torch.zeros(B)}
    tokens, probs, _ = _run(E, z, u, **greedy)
    assert torch.equal(tokens[:, 0], z[:, 0].argmax(-1).int()) or all(z[b, 0, tokens[b, 0]] == z[b, 0].max() and not (z[b, 0, :tokens[b, 0]] == z[b, 0].max()).any() for b in range(B))
    _check(z, u, tokens, probs, **greedy)


def test_a_cut_among_thousands_of_close_values(E):
    """More values in the cut's bin than are ranked at once: it is cut finer, by counts and by masses."""
    g = torch.Generator().manual_seed(7)
    B, V = 8, 60001
    z = 5.0 + torch.rand(B, 1, V, generator=g) * 1e-3
    z[:, :, ::7] = 5.0005
    z[4:] *= -1.0
    u = torch.rand(B, 1, generator=g)
    for kw in ({"top_k": torch.tensor([1, 2, 5000, 30000, 45000, 59999, 60000, 60001]).int()}, {"top_p": torch.linspace(0.01, 0.99, B)},
               {"top_k": torch.full((B,), 20000).int(), "top_p": torch.linspace(0.3, 0.999, B)}):
        tokens, probs, _ = _run(E, z, u, **kw)
        _check(z, u, tokens, probs, **kw)


def test_values_that_are_no_ordinary_numbers(E):
    g = torch.Generator().manual_seed(8)
    V, inf, nan = 3001, float("inf"), float("nan")
    z = torch.randn(10, 1, V, generator=g)
    z[0, 0, ::2] = -inf
    z[1, 0, 1:] = -inf                                       # one token
    z[2, 0, 5] = z[2, 0, 77] = inf                           # two that share everything
    z[3, 0, ::3] = nan
    z[4] = -inf
    z[5] = nan
    z[6, 0, :] = torch.finfo(torch.float32).min
    z[7, 0, 100:] = torch.finfo(torch.float32).min           # a mask of the lowest value
    z[8, 0, ::2] = 0.0
    z[8, 0, 1::2] = -0.0                                     # zeros of either sign are equal
    z[9] = z[9] * 1e38
    u = torch.rand(10, 1, generator=g)
    for kw in ({}, {"top_k": torch.full((10,), 50).int()}, {"top_p": torch.full((10,), 0.7)}, {"top_k": torch.full((10,), 2900).int(), "top_p": torch.full((10,), 0.9)},
               {"temperature": torch.full((10,), 1e-38)}, {"temperature": torch.full((10,), inf)}, {"temperature": torch.full((10,), nan)},
               {"min_p": torch.full((10,), nan), "top_p": torch.full((10,), nan)}):
        tokens, probs, status = _run(E, z, u, **kw)
        assert status == -12
        assert tokens[4, 0] == -1 and tokens[5, 0] == -1 and (probs[4:6] == 0).all()
        if "temperature" in kw and not kw["temperature"][0] < 1e30:
            live = [b for b in range(10) if b not in (4, 5)]
            assert torch.isfinite(probs).all() and (probs[live].double().sum(-1) - 1).abs().max() < 1e-5
            if kw["temperature"][0] != kw["temperature"][0]:
                assert ((probs[live] > 0).sum(-1) == 1).all()   # NaN is greedy
            else:
                assert probs[0, 0, 1] == pytest.approx(1.0 / (V // 2), rel=1e-6) and probs[0, 0, 0] == 0
            continue
        _check(z, u, tokens, probs, **kw)


def test_uniforms_at_the_ends(E):
    z = torch.tensor([[[-1.0, 2.0, -float("inf"), 0.5, -float("inf")]]]).repeat(5, 1, 1)
    u = torch.tensor([0.0, 1.0 - 2.0 ** -24, 1.0, -1.0, float("nan")])[:, None]
    tokens, _, _ = _run(E, z, u)
    assert tokens[:, 0].tolist() == [0, 3, 3, 0, 3]


@pytest.mark.parametrize("V,bf16", [(400001, False), (1 << 20, False), (1 << 20, True)])
def test_vocabularies_that_do_not_fit_shared_memory(E, V, bf16):
    g = torch.Generator().manual_seed(9)
    z = torch.randn(3, 1, V, generator=g) * 3
    z = z.bfloat16() if bf16 else z
    u = torch.rand(3, 1, generator=g)
    kw = {"top_k": torch.tensor([0, 3000, 0]).int(), "top_p": torch.tensor([0.9, 1.0, 1.0]), "temperature": torch.tensor([0.8, 1.1, 1.0])}
    tokens, probs, _ = _run(E, z, u, **kw)
    _check(z, u, tokens, probs, **kw)


def test_the_split_of_a_row_changes_nothing(E):
    """The same row alone (a cluster of eight) and among many (one CTA each), at any alignment."""
    g = torch.Generator().manual_seed(10)
    V = 32003
    row = torch.randn(V, generator=g) * 3
    many = row[None, None].repeat(400, 1, 1)
    u, kw = torch.full((400, 1), 0.6180), {"top_p": torch.full((400,), 0.93), "top_k": torch.full((400,), 3000).int()}
    tokens, probs, _ = _run(E, many, u, **kw)
    one, p1, _ = _run(E, many[:1], u[:1], **{n: t[:1] for n, t in kw.items()})
    assert (tokens == one[0, 0]).all() and torch.equal(probs, p1.expand_as(probs))
    base = torch.zeros(V + 5, device=DEV)
    for off in range(1, 5):                                  # a first row that does not begin on 16 bytes
        view = base[off:off + V].view(1, 1, V)
        view.copy_(many[0])
        t, p = E.eagle_sample(view, u[:1].to(DEV), with_probs=True, **{n: x[:1].to(DEV) for n, x in kw.items()})
        assert torch.equal(t.cpu(), one) and torch.equal(p.cpu(), p1)


def test_replayed_from_a_graph_and_on_two_streams(E):
    g = torch.Generator().manual_seed(11)
    z, u = (torch.randn(6, 3, 20011, generator=g) * 3).to(DEV), torch.rand(6, 3, generator=g).to(DEV)
    kw = {"top_p": torch.full((6,), 0.9, device=DEV), "temperature": torch.full((6,), 0.8, device=DEV)}
    want = E.eagle_sample(z, u, with_probs=True, **kw)
    side = torch.cuda.Stream()
    tokens, probs = torch.zeros(6, 3, dtype=torch.int32, device=DEV), torch.zeros(6, 3, 20011, device=DEV)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        E.eagle_sample(z, u, tokens, probs, **kw)
    z2 = torch.randn_like(z) * 2
    want2 = E.eagle_sample(z2, u, with_probs=True, **kw)
    torch.cuda.synchronize()
    for _ in range(3):
        graph.replay()
        with torch.cuda.stream(side):
            got2 = E.eagle_sample(z2, u, with_probs=True, **kw)
    torch.cuda.synchronize()
    assert torch.equal(tokens, want[0]) and torch.equal(probs, want[1]) and torch.equal(got2[0], want2[0]) and torch.equal(got2[1], want2[1])


def test_adjusted_rows_to_distributions_to_acceptance(E):
    """logit adjustment -> filtered distributions of target and draft -> acceptance on probabilities: what the oracle decides on the
    definition's distributions (rounded to fp32, as the kernels hand them on)."""
    g = torch.Generator().manual_seed(12)
    B, T, V = 6, 9, 3001
    parent = torch.tensor([[-1, 0, 1, -1, 3, 0, 5, 2, 4]] * B, dtype=torch.int32)
    draft = torch.randint(0, V, (B, T), generator=g, dtype=torch.int32)
    z = torch.randn(B, T + 1, V, generator=g) * 3
    allowed = torch.randint(-(1 << 31), 1 << 31, (B, T + 1, (V + 31) // 32), generator=g, dtype=torch.int32)
    rows = E.eagle_tree_logits_adjust(z.to(DEV), draft.to(DEV), parent.to(DEV), allowed=allowed.to(DEV))
    kw = {"temperature": torch.full((B,), 0.8), "top_p": torch.full((B,), 0.9), "top_k": torch.full((B,), 200).int()}
    on = {n: t.to(DEV) for n, t in kw.items()}
    _, target = E.eagle_sample(rows, with_probs=True, **on)
    _, small = E.eagle_sample((z[:, :T] * 0.9).to(DEV), with_probs=True, **on)
    u = torch.rand(B, T + 1, generator=g)
    path, bonus, n = _accept(E, target, small, draft, parent, u)
    adjusted = S.logits_adjust(z, draft, parent, allowed=allowed)
    want = np.stack([[S.sample(adjusted[b, r].astype(np.float32), **{n: t[b].item() for n, t in kw.items()})[1] for r in range(T + 1)] for b in range(B)])
    assert np.abs(target.cpu().double().numpy() - want).max() <= 2.0 ** -24
    for b in range(B):                                        # the bonus token is one that the filters and the grammar left
        last = int(path[b, int(n[b]) - 1]) + 1 if int(n[b]) else 0
        assert want[b, last][int(bonus[b])] > 0


def _accept(E, target, small, draft, parent, u):
    B, T = draft.shape
    n = torch.zeros(B, dtype=torch.int32, device=DEV)
    path, bonus = E.eagle_tree_accept(target, small, draft.to(DEV), parent.to(DEV), u.to(DEV), accept_len=n)[:2]
    torch.cuda.synchronize()
    return path.cpu(), bonus.cpu(), n.cpu()


def test_top_p_next_to_one_over_the_largest_vocabulary(E):
    """The tail's weights are below a unit of the sums and are rounded up, so that what they sum to is more than 1 - p, the definition's less: either
    answer keeps the first two tokens, a prefix of the tail at the most, and their probabilities (the tail's sum is 1e-7)."""
    V = 1 << 20
    z = torch.full((1, 1, V), float(np.log(0.7 * 2.0 ** -43)))
    z[0, 0, 700000], z[0, 0, 3] = 0.0, float(np.log(0.5))
    for top_p in (1 - 2.0 ** -24, 1 - 2.0 ** -20):
        tokens, probs, status = _run(E, z, torch.full((1, 1), 0.9), top_p=torch.full((1,), top_p))
        assert status == 0 and int(tokens[0, 0]) == 700000
        got = probs[0, 0].double().numpy()
        assert abs(got[700000] - 2 / 3) < 4e-7 and abs(got[3] - 1 / 3) < 4e-7
        got[[3, 700000]] = 0
        kept = np.flatnonzero(got)
        assert got.max() < 1e-13 and (len(kept) == 0 or kept[-1] - kept[0] + 1 - len(kept) <= 2)
        assert top_p == 1 - 2.0 ** -24 or len(kept) == 0


def test_more_elements_than_32_bits_count(E):
    """The last rows of 33000 x 65537 logits (2^31 elements and more)."""
    R, V, last = 33000, 65537, 3
    z = torch.zeros(1, R, V, dtype=torch.bfloat16, device=DEV)
    g = torch.Generator().manual_seed(12)
    tail = (torch.randn(1, last, V, generator=g) * 3).bfloat16()
    z[:, R - last:] = tail.to(DEV)
    u = torch.rand(1, R, generator=g)
    kw = {"top_k": torch.full((1,), 50).int(), "top_p": torch.full((1,), 0.9)}
    probs = torch.full((1, R, V), 7.0, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    tokens, _ = E.eagle_sample(z, u.to(DEV), None, probs, status=status, **{n: t.to(DEV) for n, t in kw.items()})
    assert int(status.item()) == 0
    _check(tail, u[:, R - last:], tokens[:, R - last:].cpu(), probs[:, R - last:].cpu(), **kw)
    assert (tokens[:, :R - last] < 45).all() and (probs[:, R - last - 1].cpu() == torch.tensor([1 / 45] * 45 + [0.0] * (V - 45))).all()


def test_values_whose_differences_overflow(E):
    """Logits of either sign next to the largest number, and filters that look at differences of them."""
    g = torch.Generator().manual_seed(13)
    B, V = 12, 5000
    z = torch.randn(B, 1, V, generator=g)
    z[:6] = -1e38 - z[:6].abs() * 5e37                       # all negative
    z[6:9] = z[6:9] * 1e38
    z[9] = 3e38
    z[9, 0, ::2] = -3e38
    z[10, 0] = 4.6e36 + z[10, 0] * 1e35                      # about where 64 of them overflow
    z[11, 0] = -4.6e36 + z[11, 0] * 1e35
    u = torch.rand(B, 1, generator=g)
    t = torch.tensor([1.0, 1e37, float("inf"), 1e36, 3e38, 1.0, 1e38, float("inf"), 1e37, float("inf"), 1e35, 1e35])
    k = torch.tensor([3, 50, 200, 128, 129, 5000, 7, 4000, 100, 0, 60, 3000]).int()
    for kw in ({"temperature": t, "top_p": torch.full((B,), 0.6)}, {"temperature": t, "top_k": k}, {"temperature": t, "top_k": k, "top_p": torch.full((B,), 0.8)},
               {"temperature": t, "min_p": torch.full((B,), 0.3)}):
        tokens, probs, status = _run(E, z, u, **kw)
        assert status == 0
        _check(z, u, tokens, probs, **kw)


@pytest.mark.parametrize("bf16", [False, True])
def test_small_top_k(E, bf16):
    """Where the few tokens that can stay are looked for first: k up to and past the most that are taken that way, all the largest values side by side or
    under one thread, many equal ones, fewer tokens than k."""
    g = torch.Generator().manual_seed(14)
    B, V = 40, 20011
    z = torch.randn(B, 2, V, generator=g) * 2
    z[8:16, :, 5000:5600] += 20                              # neighbours
    z[16:24] = z[16:24].round()                              # thousands of equal values
    z[24:28] = -float("inf")
    for b in range(24, 28):
        z[b, :, torch.randperm(V, generator=g)[:10 * (b - 23)]] = torch.randn(10 * (b - 23), generator=g)
    z[28:32] = z[28:32].sort(-1).values
    z = z.bfloat16() if bf16 else z
    u = torch.rand(B, 2, generator=g)
    k = torch.tensor([1, 2, 7, 50, 255, 256, 257, 300] * 5).int()
    p, m = torch.tensor([0.3, 0.9, 0.99, 1.0, 0.05] * 8), torch.tensor([0.0, 0.1, 0.0, 0.02, 0.5, 0.0, 1.0] * 6)[:B]
    for kw in ({"top_k": k}, {"top_k": k, "top_p": p}, {"top_k": k, "top_p": p, "min_p": m, "temperature": torch.linspace(0.2, 3, B)}):
        tokens, probs, status = _run(E, z, u, **kw)
        assert status == 0
        _check(z, u, tokens, probs, **kw)


@pytest.mark.parametrize("bf16", [False, True])
def test_tiny_temperatures_with_filters(E, bf16):
    """Temperatures down to the smallest numbers of fp32: only values next to the largest one weigh anything, whatever the filters do with differences
    of values over the temperature.  Rows of ordinary values, of equal largest ones, and of values about as far apart as the temperature is small."""
    g = torch.Generator().manual_seed(15)
    temperatures = torch.tensor([1e-35, 1e-36, 4e-37, 1e-37, 1.2e-38, 1e-40, 1e-45] * 3)
    B, V = len(temperatures), 12007
    z = torch.randn(B, 1, V, generator=g) * 3
    z[7:14, 0, ::5] = z[7:14, 0].max(-1, keepdim=True).values   # (2402 equal ones)
    z[14:] = torch.randn(B - 14, 1, V, generator=g) * 3 * temperatures[14:, None, None]
    z = z.bfloat16() if bf16 else z
    u = torch.rand(B, 1, generator=g)
    t, p = {"temperature": temperatures}, torch.linspace(0.05, 0.999, B)
    for kw in ({"top_p": p}, {"top_k": torch.full((B,), 3000).int(), "top_p": p}, {"top_k": torch.full((B,), 300).int(), "top_p": p},
               {"top_k": torch.full((B,), 40).int(), "top_p": p}, {"top_p": p, "min_p": torch.full((B,), 0.05)}, {"top_k": torch.full((B,), 3000).int()}, {}):
        for R in (1, 30):                                       # clusters of eight CTAs, and a CTA or two to a row
            many, uu = z.expand(B, R, V).contiguous(), u.expand(B, R).contiguous()
            tokens, probs, status = _run(E, many, uu, **kw, **t)
            assert status == 0 and torch.equal(tokens, tokens[:, :1].expand(B, R)) and torch.equal(probs, probs[:, :1].expand(B, R, V))
            _check(z, u, tokens[:, :1], probs[:, :1], **kw, **t)
            only, _, _ = _run(E, many, uu, probs=False, **kw, **t)
            _, alone, _ = _run(E, many, None, **kw, **t)
            assert torch.equal(only, tokens) and torch.equal(alone, probs)
