"""Penalties, biases and masks on a tree's logit rows, against the 64-bit definition.

Tolerance: the work is fp32 (division, multiplication, a product and two subtractions, an addition), each within 2^-24 of its result, and the
sum of a token's biases adds as many; 1e-6 of the largest magnitude on the way (|z| rho + phi c + pi + sum |bias|) covers them."""
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


def make(B, T, V, seed, sizes=None, H=0, bias=0, grammar=False, bf16=False, penalties=True, chain=False, crowd=7):
    g, r = torch.Generator().manual_seed(seed), np.random.default_rng(seed)
    z = torch.randn(B, T + 1, V, generator=g) * 3
    kw = {}
    z = z.bfloat16() if bf16 else z
    parent = np.full((B, T), 2 ** 30, dtype=np.int32)
    sizes = sizes if sizes is not None else [T] * B
    for b in range(B):
        for i in range(sizes[b]):
            parent[b, i] = i - 1 if chain else r.integers(-1, i)
    # few different tokens, so that paths, history and bias lists meet
    pool = r.integers(0, V, crowd)
    some = lambda *s: torch.tensor(r.choice(pool, s), dtype=torch.int32)  # noqa: E731
    if T:
        kw.update(draft_tokens=some(B, T), tree_parent=torch.tensor(parent), tree_sizes=_ints(sizes))
    if penalties:
        kw.update(repetition=torch.rand(B, generator=g) + 0.6, presence=torch.randn(B, generator=g), frequency=torch.rand(B, generator=g))
    if H:
        kw.update(history=some(B, H), history_len=_ints([H] + [int(x) for x in r.integers(0, H + 1, B - 1)]), prompt_len=_ints([int(x) for x in r.integers(0, H, B)]))
    if bias:
        kw.update(bias_tokens=some(B, bias), bias_values=torch.randn(B, bias, generator=g), bias_len=_ints([int(x) for x in r.integers(0, bias + 1, B)]))
    if grammar:
        kw["allowed"] = torch.tensor(r.integers(-2 ** 31, 2 ** 31, (B, T + 1, (V + 31) // 32)), dtype=torch.int32)
    return z, kw


def run(E, z, kw, out=None, **more):
    up = {k: v.to(DEV) for k, v in kw.items()}
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    out = torch.full(z.shape, 7.0, device=DEV) if out is None else out
    E.eagle_tree_logits_adjust(z.to(DEV), out=out, status=status, **up, **more)
    torch.cuda.synchronize()
    return out.cpu(), int(status.item())


def check(got, z, kw):
    want = S.logits_adjust(z, **kw)
    got = got.double().numpy()
    live = ~np.isnan(want)
    assert (got[~live] == 7.0).all(), "rows past the tree have changed"
    masked = np.isinf(want) & live
    assert (got[masked] == want[masked]).all()
    live &= ~masked
    most = lambda k: float(kw[k].abs().max()) if k in kw else 0.0  # noqa: E731
    extra = most("frequency") * (kw["history"].shape[1] if "history" in kw else 0) + most("frequency") * 65 + most("presence")
    if "bias_values" in kw:
        extra += float(kw["bias_values"].abs().sum(1).max())
    size = np.abs(z.double().numpy()) * 2 + extra
    err = np.abs(got - want)
    assert (err[live] <= 1e-6 * size[live]).all(), (err[live] / size[live]).max()
    # what nothing applies to comes through bit for bit
    if not kw.get("history", torch.empty(0)).numel() and "draft_tokens" not in kw and "bias_tokens" not in kw:
        assert np.array_equal(got[live], z.double().numpy()[live])


CASES = {
    "plain_decoding": dict(B=3, T=0, V=1000, H=50),
    "one_of_everything": dict(B=1, T=1, V=1, H=3, bias=2, grammar=True),
    "odd_vocabulary": dict(B=4, T=9, V=2049, sizes=[9, 0, 5, 1], H=40, bias=11, grammar=True),
    "wide": dict(B=2, T=5, V=33333, H=300, bias=64, grammar=True),
    "bf16": dict(B=3, T=7, V=4097, sizes=[7, 2, 6], H=100, bias=5, grammar=True, bf16=True),
    "chain": dict(B=2, T=64, V=5000, sizes=[64, 33], H=20, chain=True),
    "no_history": dict(B=2, T=6, V=700, bias=3),
    "bias_only": dict(B=5, T=0, V=6000, bias=1024, penalties=False, crowd=40),
    "mask_only": dict(B=2, T=3, V=90, grammar=True, penalties=False),
    "nothing": dict(B=2, T=0, V=513, penalties=False, bf16=True),
    "long_history": dict(B=2, T=2, V=3000, H=20000, crowd=500),
}


@pytest.mark.parametrize("name", list(CASES))
def test_matches_the_definition(E, name):
    z, kw = make(**CASES[name], seed=len(name))
    got, status = run(E, z, kw)
    assert status == 0
    check(got, z, kw)


def test_in_place_and_twice_the_same(E):
    z, kw = make(4, 12, 5001, 3, sizes=[12, 3, 0, 7], H=60, bias=20, grammar=True)
    a, _ = run(E, z, kw)
    buf = z.to(DEV)
    up = {k: v.to(DEV) for k, v in kw.items()}
    E.eagle_tree_logits_adjust(buf, out=buf, **up)
    for b, n in enumerate([12, 3, 0, 7]):
        assert torch.equal(buf[b, :n + 1].cpu(), a[b, :n + 1]) and torch.equal(buf[b, n + 1:].cpu(), z[b, n + 1:])
    assert torch.equal(run(E, z, kw)[0], a)


def test_one_tree_for_every_sequence(E):
    z, kw = make(3, 8, 900, 4, H=10)
    kw["tree_parent"] = kw["tree_parent"][:1].repeat(3, 1)
    a, _ = run(E, z, kw)
    shared = dict(kw, tree_parent=kw["tree_parent"][0].contiguous(), tree_sizes=kw["tree_sizes"][:1].contiguous())
    b, status = run(E, z, shared, shared_tree=True)
    assert status == 0 and torch.equal(a, b)


def test_a_mask_that_allows_nothing_and_odd_values(E):
    z, kw = make(2, 0, 100, 5, H=8)
    kw["allowed"] = torch.zeros(2, 1, 4, dtype=torch.int32)
    got, status = run(E, z, kw)
    assert status == 0 and torch.isinf(got).all() and (got < 0).all()
    kw["allowed"] = torch.full((2, 1, 4), -1, dtype=torch.int32)
    z[0, 0, :4] = torch.tensor([float("inf"), float("-inf"), float("nan"), -0.0])
    kw["history"][0, :4] = _ints([0, 1, 2, 3])
    kw["history_len"][0] = 8
    got, status = run(E, z, kw)
    assert got[0, 0, 0] == float("inf") and got[0, 0, 1] == float("-inf") and torch.isnan(got[0, 0, 2])


def test_lengths_are_clamped_and_strange_tokens_ignored(E):
    z, kw = make(2, 3, 500, 6, H=10, bias=4)
    ok, status = run(E, z, dict(kw, history_len=_ints([10, 10]), bias_len=_ints([4, 4])))
    assert status == 0
    long, status = run(E, z, dict(kw, history_len=_ints([2 ** 31 - 1, 11]), bias_len=_ints([5, 99])))
    assert status == 0 and torch.equal(ok, long)
    none, _ = run(E, z, dict(kw, history_len=_ints([0, 0]), bias_len=_ints([0, 0])))
    minus, status = run(E, z, dict(kw, history_len=_ints([-1, -5]), bias_len=_ints([-1, -2 ** 31])))
    assert status == 0 and torch.equal(none, minus)
    for name in ("history", "bias_tokens", "draft_tokens"):
        for bad in (-1, 500, 2 ** 31 - 1):
            odd = dict(kw, **{name: kw[name].clone()}, history_len=_ints([10, 10]), bias_len=_ints([4, 4]))
            odd[name][1, 0] = bad
            got, status = run(E, z, odd)
            assert status == -7 and torch.equal(got[0], ok[0])
            if name == "history":
                less = dict(odd, history=odd["history"].clone())
                less["history"][1, 0] = int(kw["history"][1, 1]) if int(kw["prompt_len"][1]) > 1 else 0
    odd = dict(kw, history=kw["history"].clone(), history_len=_ints([10, 10]), bias_len=_ints([4, 4]))
    odd["history"][1, 9] = -3
    got, _ = run(E, z, odd)
    short, _ = run(E, z, dict(kw, history_len=_ints([10, 9]), bias_len=_ints([4, 4])))
    assert torch.equal(got, short)


@pytest.mark.parametrize("what", ["parent", "size"])
def test_an_invalid_tree_is_reported_and_zeroed(E, what):
    z, kw = make(3, 5, 3001, 7, sizes=[5, 4, 5], H=6)
    ok, _ = run(E, z, kw)
    if what == "parent":
        kw["tree_parent"][1, 2] = 2
    else:
        kw["tree_sizes"][1] = 6
    got, status = run(E, z, kw)
    assert status == -5 and (got[1] == 0).all()
    assert torch.equal(got[0], ok[0]) and torch.equal(got[2], ok[2])


def test_replayed_from_a_graph(E):
    z, kw = make(2, 6, 2500, 8, H=30, bias=4, grammar=True)
    up = {k: v.to(DEV) for k, v in kw.items()}
    dz, out = z.to(DEV), torch.full(z.shape, 7.0, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        E.eagle_tree_logits_adjust(dz, out=out, **up)
    z2, kw2 = make(2, 6, 2500, 9, H=30, bias=4, grammar=True)
    dz.copy_(z2)
    for k in up:
        up[k].copy_(kw2[k])
    graph.replay()
    torch.cuda.synchronize()
    check(out.cpu(), z2, kw2)


def test_the_largest_vocabulary(E):
    """Rows whose elements pass 2^31, in place: every untouched logit keeps its bits, the others are what the formula says."""
    V, B = (1 << 30) - 1, 3
    z = torch.empty(B, 1, V, device=DEV)
    for b in range(B):
        z[b, 0] = torch.arange(b, b + V, dtype=torch.int32, device=DEV).remainder_(8191).sub_(4000)
    at = _ints([[0, V - 1, V - 2047], [V - 1, 5, V // 2], [V - 1, V - 2, 2048]]).to(DEV)
    allowed = torch.full((B, 1, (V + 31) // 32), -1, dtype=torch.int32, device=DEV)
    allowed[2, 0, -1] = ~(1 << 3)                         # token V - 28
    rho, phi, pi = (torch.tensor(x, device=DEV) for x in ([1.5, 2.0, 0.5], [0.25, 0.5, 1.0], [0.125, 0.0, 2.0]))
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    want = z.clone()
    for b in range(B):
        for t in at[b].tolist():
            x = float(z[b, 0, t])
            want[b, 0, t] = (x / float(rho[b]) if x > 0 else x * float(rho[b])) - float(phi[b]) - float(pi[b])
    want[2, 0, (V // 32) * 32 + 3] = -float("inf")
    E.eagle_tree_logits_adjust(z, out=z, history=at, history_len=_ints([3, 3, 3]).to(DEV), repetition=rho, frequency=phi, presence=pi, allowed=allowed,
                               status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    wrong = (z != want).nonzero()
    assert all(abs(float(z[i, j, k]) - float(want[i, j, k])) <= 1e-6 * 16500 for i, j, k in wrong[:16].tolist()) and len(wrong) <= 9
    del z, want, allowed
    torch.cuda.empty_cache()
