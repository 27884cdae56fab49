"""The 64-bit definitions of block-scaled caches, windowed attention and sampling against independent ones, and what the entry points refuse
before anything is launched."""
import ctypes
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

from oracle import serving as S


@pytest.fixture(scope="module")
def lib():
    from paper_2401_15077_b200 import binding, build
    build.build()
    return binding.load()


# ------------------------------------------------------------------------------------------------------------- codes and scales
def test_nearest_code_is_the_conversion_to_e4m3():
    x = torch.cat([torch.linspace(-460, 460, 20001), torch.logspace(-12, 2.7, 5001), -torch.logspace(-12, 2.7, 5001),
                   torch.tensor([0.0, -0.0, 448.0, 464.0, 1e9, -1e9, 2.0 ** -10, 3 * 2.0 ** -10])])
    want = x.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(S.nearest_code(x.double().numpy()), want)
    assert S.nearest_code(np.array([np.nan]))[0] == 127
    # every middle between two codes goes to the even one
    v = S.e4m3(np.arange(127))
    mid = (v[1:] + v[:-1]) / 2
    assert np.array_equal(S.nearest_code(mid), np.where(np.arange(126) % 2 == 0, np.arange(126), np.arange(1, 127)))


def test_block_scale_is_the_least_power_of_two():
    for a in [0.0, 1e-30, 448.0 * 2.0 ** -40, 448.0 * 2.0 ** -40 * (1 + 2.0 ** -20), 0.875, 1.0, 447.9, 448.0, 448.1, 3e38]:
        s = S.block_scale(a)
        e = math.log2(s)
        assert e == int(e) and -40 <= e <= 120
        assert a <= 448.0 * s and (e == -40 or a > 448.0 * s / 2)


def _append_case(tree, seed):
    g = torch.Generator().manual_seed(seed)
    n, lens, hq, hkv, block = [5, 40, 0, 17], [3, 60, 9, 16], 2, 2, 16
    shape = (4, hkv, 112, 128)
    k, v = (torch.randint(0, 127, shape, generator=g, dtype=torch.uint8).numpy() for _ in range(2))
    ks, vs = (2.0 ** torch.randint(-12, -4, (*shape[:2], 7), generator=g).double().numpy() for _ in range(2))
    rows = (4, max(n)) if tree else (sum(n),)
    x = torch.randn(*rows, hq + 2 * hkv, 128, generator=g).bfloat16()
    freqs = np.array([10000.0 ** (-2 * m / 128) for m in range(64)])
    if tree:
        order = {"tree_parent": torch.tensor([[i - 1 if i % 3 else -1 for i in range(max(n))]] * 4), "tree_sizes": n}
    else:
        order = {"token_start": np.concatenate([[0], np.cumsum(n)])}
    return (k, v, ks, vs), x.split((hq, hkv, hkv), dim=-2), lens, n, freqs, block, order


@pytest.mark.parametrize("tree", [False, True])
def test_appended_values_are_within_half_a_step_and_older_ones_are_kept(tree):
    cache, (q, k, v), lens, n, freqs, block, order = _append_case(tree, 3)
    _, res = S.block_append(q, k, v, cache, lens, freqs, block, **order)
    _, stored = S.rope_append(q, k, v, lens, freqs, **order)
    for which in (0, 1):
        values, codes, scales = res[which]
        old = S.e4m3(cache[which]) * cache[2 + which].repeat(block, -1)[..., None]
        for b, slot, key, val in stored:
            x, s = (key, val)[which], scales[b, :, slot // block][:, None]
            assert np.allclose(values[b, :, slot] * s, x, rtol=1e-12, atol=0)
            assert (np.abs(values[b, :, slot]) <= 448).all()
            assert np.log2(s).tolist() == np.round(np.log2(s)).tolist()
        for b in range(4):
            if not n[b]:
                assert np.array_equal(codes[b], cache[which][b]) and np.array_equal(scales[b], cache[2 + which][b])
                continue
            now = S.e4m3(codes[b, :, :lens[b]]) * scales[b].repeat(block, -1)[:, :lens[b], None]
            step = 2.0 ** -4 * np.abs(old[b, :, :lens[b]]) + 2.0 ** -10 * scales[b].repeat(block, -1)[:, :lens[b], None]
            assert (np.abs(now - old[b, :, :lens[b]]) <= step).all()
            touched = range(lens[b] // block, (lens[b] + n[b] - 1) // block + 1)
            same = np.array([scales[b, :, t] for t in touched])
            assert not tree or (same == same[0]).all(), "a tree's blocks share a scale"
            others = [t for t in range(7) if t not in touched]
            assert np.array_equal(scales[b][:, others], cache[2 + which][b][:, others])


# ----------------------------------------------------------------------------------------------------------------- attention
def test_without_a_window_it_is_the_chunk_attention():
    g = torch.Generator().manual_seed(4)
    k, v = (torch.randn(3, 2, 70, 64, generator=g).bfloat16() for _ in range(2))
    q, lens, starts = torch.randn(29, 4, 64, generator=g).bfloat16(), [40, 0, 9], [0, 20, 28, 29]
    a, b = S.window_attn(q, k, v, lens, token_start=starts), S.chunk_attn(q, k, v, lens, starts)
    assert np.allclose(a[0], b[0], rtol=1e-12, atol=1e-14) and np.allclose(a[1], b[1], rtol=1e-12, atol=1e-14)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 3), (7, 0), (30, 2), (30, 50), (1000, 4)])
def test_a_window_is_a_mask(window, sinks):
    g = torch.Generator().manual_seed(5)
    L, n, d = 33, 25, 64
    k, v = (torch.randn(1, 1, L + n, d, generator=g).bfloat16() for _ in range(2))
    q = torch.randn(n, 2, d, generator=g).bfloat16()
    j, p = torch.arange(L + n)[None], (L + torch.arange(n))[:, None]
    mask = (j <= p) & ((j > p - window) | (j < sinks))
    want = torch.nn.functional.scaled_dot_product_attention(q.double().transpose(0, 1), k[0].double().expand(2, -1, -1), v[0].double().expand(2, -1, -1), mask)
    got, _ = S.window_attn(q, k, v, [L], token_start=[0, n], window=window, sinks=sinks)
    assert np.allclose(got, want.transpose(0, 1).numpy(), rtol=1e-11, atol=1e-13)
    # a chain of nodes sees what a chunk sees, as long as the path is inside of the window
    if window >= n:
        chain = torch.arange(-1, n - 1)[None]
        tree, _ = S.window_attn(q[None], k, v, [L], tree_parent=chain, window=window, sinks=sinks)
        assert np.allclose(tree[0], got, rtol=1e-12, atol=1e-14)


def test_blocks_stand_for_code_times_scale():
    g = torch.Generator().manual_seed(6)
    codes = [torch.randint(0, 120, (5, 2, 32, 128), generator=g, dtype=torch.uint8) for _ in range(2)]
    scales = [2.0 ** torch.randint(-9, -5, (5, 2, 2), generator=g).float() for _ in range(2)]
    plain = [torch.from_numpy(S.e4m3(c.numpy()) * s.double().numpy().repeat(16, -1)[..., None]).bfloat16() for c, s in zip(codes, scales)]      # exact
    q = torch.randn(14, 4, 128, generator=g).bfloat16()
    kw = dict(token_start=[0, 9, 14], block_table=torch.tensor([[3, 0], [4, 1]]), window=20, sinks=2)
    a = S.window_attn(q, *codes, [40, 11], k_scale=scales[0], v_scale=scales[1], block=16, **kw)
    b = S.window_attn(q, *plain, [40, 11], **kw)
    assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])


# ------------------------------------------------------------------------------------------------------------------ sampling
def test_sampling_by_hand():
    z = np.log([0.4, 0.1, 0.3, 0.15, 0.05])
    for u, t in ((0.0, 0), (0.39, 0), (0.41, 1), (0.51, 2), (0.79, 2), (0.81, 3), (0.96, 4)):
        assert S.sample(z, u)[0] == t
    assert np.allclose(S.sample(z, top_k=2)[1], [4 / 7, 0, 3 / 7, 0, 0])
    assert np.allclose(S.sample(z, top_p=0.69)[1], [4 / 7, 0, 3 / 7, 0, 0])
    assert np.allclose(S.sample(z, top_p=0.71)[1], np.array([0.4, 0, 0.3, 0.15, 0]) / 0.85)
    assert np.allclose(S.sample(z, min_p=0.3)[1], np.array([0.4, 0, 0.3, 0.15, 0]) / 0.85)
    assert np.allclose(S.sample(z, top_k=4, top_p=0.9)[1], np.array([0.4, 0.1, 0.3, 0.15, 0]) / 0.95)      # 0.85 of 0.95 is 0.894
    assert np.allclose(S.sample(z, top_k=4, top_p=0.89)[1], np.array([0.4, 0, 0.3, 0.15, 0]) / 0.85)
    assert S.sample(z, 0.99, temperature=0.0)[0] == 0 and S.sample(z, top_p=0.0)[1].tolist() == [1, 0, 0, 0, 0]
    p = S.sample(z, temperature=0.5)[1]
    assert np.allclose(p, np.array([16, 1, 9, 2.25, 0.25]) / 28.5)
    assert S.sample([2.0, 2.0, 2.0, 1.0], top_k=2)[1].tolist() == [0.5, 0.5, 0, 0]       # equal ones: the lowest ids
    assert S.sample([-np.inf, np.nan, 3.0], 0.5)[0] == 2 and S.sample([-np.inf, np.nan], 0.5)[0] == -1


def test_sampling_against_a_sorted_formulation():
    g = np.random.default_rng(7)
    for _ in range(60):
        V = int(g.integers(2, 60))
        z = np.round(g.normal(size=V) * 2, 1)                # (some are equal)
        T, k, p, m = float(g.uniform(0.3, 2)), int(g.integers(0, V + 3)), float(g.uniform(0.05, 1.1)), float(g.choice([0.0, 0.05, 0.3]))
        w = [Fraction(float(x)) for x in np.exp((z - z.max()) / T)]
        order = sorted(range(V), key=lambda i: (-z[i], i))
        if 0 < k < V:
            order = order[:k]
        if p < 1:
            total, run, kept = sum(w[i] for i in order), Fraction(0), []
            for i in order:
                if kept and run >= Fraction(p) * total:
                    break
                kept.append(i)
                run += w[i]
            order = kept
        order = [i for i in order if w[i] >= Fraction(m)]
        want = np.zeros(V)
        want[order] = [float(w[i] / sum(w[j] for j in order)) for i in order]
        u = float(g.random())
        t, got, margin = S.sample(z, u, T, k, p, m)
        assert np.allclose(got, want, rtol=1e-12, atol=0)
        if margin > 1e-9:
            assert t == int(np.searchsorted(np.cumsum(want), u, side="right"))


def test_drawn_tokens_follow_the_distribution():
    g = np.random.default_rng(8)
    z = g.normal(size=40) * 2
    _, p, _ = S.sample(z, None, 0.8, 12, 0.95, 0.01)
    n = 20000
    count = np.bincount([S.sample(z, u, 0.8, 12, 0.95, 0.01)[0] for u in g.random(n)], minlength=40)
    assert (count[p == 0] == 0).all()
    live = p > 0
    chi = ((count[live] - n * p[live]) ** 2 / (n * p[live])).sum()
    assert chi < live.sum() - 1 + 5 * math.sqrt(2 * (live.sum() - 1))


# ------------------------------------------------------------------------------------------------------------------ refusals
def test_host_checks_return_before_any_launch(lib):
    from paper_2401_15077_b200 import binding as E
    before, fake = E.launch_count(), 4096
    by, ref = ctypes.byref, lambda d, **kw: (d, [setattr(d, n, x) for n, x in kw.items()])[0]

    def store(**kw):
        return ref(E.KVStoreDesc(fake, fake, fake, fake, 256, None, 0, 0, 0), **kw)

    # ---- appends
    def block(**kw):
        return ref(E.BlockDesc(2, 10, 8, 4, 2, 128, 0, 32, 0.0, 0, 0, 0, fake, None, None, 0, None), **kw)

    for fn in (lib.eagle_block_append, lib.eagle_tree_block_append):
        call = lambda d, s, q=fake, k=fake, lens=fake: fn(by(d), q, k, fake, fake, by(s), lens, fake, None)  # noqa: E731, B023
        assert fn(None, fake, fake, fake, fake, by(store()), fake, fake, None) == -1
        assert fn(by(block()), fake, fake, fake, fake, None, fake, fake, None) == -1
        for bad in (dict(block_size=0), dict(block_size=8), dict(block_size=48), dict(block_size=256), dict(rotary_dim=8), dict(rotary_dim=144),
                    dict(rotary_dim=72), dict(batch=-1), dict(batch=65536), dict(num_kv_heads=0), dict(num_q_heads=-1), dict(k_stride=100),
                    dict(k_stride=264 - 4), dict(amplitude=float("nan"))):
            assert call(block(**bad), store()) == -2, bad
        assert fn(by(block(max_tree=65, num_tokens=-1)), fake, fake, fake, fake, by(store()), fake, fake, None) == -2
        assert call(block(), store(kv_capacity=250)) == -2                         # slots that are no multiple of the block
        assert call(block(), store(block_table=fake, num_pages=4, page_size=16, max_pages_per_seq=4)) == -2
        assert call(block(), store(block_table=fake, num_pages=0, page_size=64, max_pages_per_seq=4)) == -2
        assert call(block(), store(k_scale=None)) == -1 and call(block(), store(k_scale=None, v_scale=None)) == -1
        assert call(block(), store(k_scale=fake + 2)) == -2 and call(block(), store(k=fake + 8)) == -2
        assert call(block(), store(k=None)) == -1 and call(block(), store(), k=None) == -1 and call(block(), store(), lens=None) == -1
        assert call(block(), store(), q=fake + 8) == -2
        assert call(block(freqs=None), store()) == -1
        assert call(block(batch=0), store()) == 0
    # ---- attention
    def window(**kw):
        return ref(E.WindowDesc(2, 10, 8, 4, 2, 128, 32, 0, 0, 0.0, None, 0, fake, 1 << 30, None), **kw)

    for fn, tree in ((lib.eagle_window_attn, False), (lib.eagle_tree_window_attn, True)):
        call = lambda d, s, q=fake, out=fake: fn(by(d), q, by(s), fake, fake, out, None)  # noqa: E731, B023
        assert fn(None, fake, by(store()), fake, fake, fake, None) == -1 and fn(by(window()), fake, None, fake, fake, fake, None) == -1
        for bad in (dict(head_dim=96), dict(head_dim=64), dict(num_q_heads=5), dict(num_q_heads=34), dict(num_kv_heads=0), dict(batch=65536), dict(block_size=24),
                    dict(block_size=-16), dict(block_size=0), dict(window=-1), dict(sinks=-1), dict(sm_scale=-1.0), dict(sm_scale=float("nan"))):
            assert call(window(**bad), store()) == -2, bad
        if tree:
            assert call(window(max_tree=65), store()) == -2 and call(window(window=63), store()) == -2 and call(window(max_tree=-1), store()) == -2
            assert call(window(max_tree=0), store()) == 0
        else:
            assert call(window(num_tokens=-1), store()) == -2 and call(window(num_tokens=0), store()) == 0
        assert call(window(), store(k_scale=None, v_scale=None)) == -1
        assert call(window(block_size=0), store(k_scale=None, v_scale=None), q=fake + 8) == -2
        assert call(window(), store(), out=fake + 16) == -2
        assert call(window(workspace=None), store()) == -3 and call(window(workspace=fake + 16), store()) == -3
        assert call(window(workspace_bytes=1000), store()) == -3
        assert call(window(), store(), q=None) == -1 and call(window(), store(v=None)) == -1
    assert lib.eagle_window_attn_workspace(None) == 0 and lib.eagle_window_attn_workspace(by(window(num_q_heads=5, max_tree=0))) == 0
    assert lib.eagle_window_attn_workspace(by(window(max_tree=65))) == 0
    # the size covers single tokens over either kind of cache, and fewer tokens
    for hq, hkv, d in ((32, 8, 128), (16, 1, 128), (8, 8, 64)):
        most = E.eagle_window_attn_workspace(40, 1000, hq, hkv, d)
        assert all(E.eagle_window_attn_workspace(40, n, hq, hkv, d) <= most for n in (0, 1, 40, 41, 500))
        assert most >= E.eagle_chunk_attn_workspace(40, 1000, hq, hkv, d)
    # ---- sampling
    def sample(**kw):
        return ref(E.SampleDesc(2, 3, 100, 0, None, None, None, None, None, None), **kw)

    call = lambda d, z=fake, u=fake, t=fake, p=2 * fake: lib.eagle_sample(by(d), z, u, t, p, None)  # noqa: E731
    assert lib.eagle_sample(None, fake, fake, fake, fake, None) == -1
    for bad in (dict(batch=-1), dict(batch=65536), dict(rows=-1), dict(vocab=0), dict(vocab=(1 << 20) + 1), dict(batch=65535, rows=1 << 20)):
        assert call(sample(**bad)) == -2, bad
    assert call(sample(), z=None) == -1 and call(sample(), u=None) == -1 and call(sample(), t=None, p=None) == -1
    assert call(sample(), z=fake + 2) == -2 and call(sample(), p=fake) == -2 and call(sample(), p=2 * fake + 1) == -2
    assert call(sample(batch=0)) == 0 and call(sample(rows=0)) == 0
    assert E.launch_count() == before
    assert E.status_string(-12) not in ("unknown status", E.status_string(-11))


def test_stores_that_do_not_fit_are_refused(lib):
    from paper_2401_15077_b200 import binding as E
    codes = torch.zeros(2, 2, 64, 128, dtype=torch.uint8)
    scale = torch.ones(2, 2, 4)
    kv = E.KVStore(codes, codes, k_scale=scale, v_scale=scale, block_size=16)
    assert kv.block_size == 16 and kv.fp8 and kv.batch == 2
    for kw in (dict(block_size=16), dict(k_scale=scale, v_scale=scale, block_size=24), dict(k_scale=scale, v_scale=scale, block_size=32),
               dict(k_scale=scale[:, :, :2], v_scale=scale, block_size=16), dict(k_scale=scale, v_scale=scale), dict(k_scale=scale.double(), v_scale=scale, block_size=16),
               dict(k_scale=scale, v_scale=scale, block_size=-16)):
        with pytest.raises(E.EagleError):
            E.KVStore(codes, codes, **kw)
    with pytest.raises(E.EagleError):
        E.eagle_window_attn_workspace(1, 10, 6, 4, 128)
    with pytest.raises(E.EagleError):
        E.eagle_sample(torch.zeros(1, 1, 8))                 # not on a GPU


def test_the_status_of_a_scale_has_a_name(lib):
    from paper_2401_15077_b200 import binding
    assert len({binding.status_string(c) for c in range(-13, 1)}) == 14 and binding.status_string(-13) != "unknown status"
