"""Pins of the 64-bit definitions behind the calls around verification, and what the library answers without a GPU: rotary
frequencies, workspace sizes and refusals."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import serving as S


@pytest.fixture(scope="module")
def E():
    from paper_2401_15077_b200 import binding, build
    build.build()
    binding.load()
    return binding


# ------------------------------------------------------------------------------------------------------------ definitions
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotated_products_depend_on_the_distance_only(interleaved):
    rng = np.random.default_rng(1)
    q, k = rng.standard_normal((2, 64))
    freqs, _ = S.rope_frequencies(32)
    at = lambda x, p: S.rotate(x, p, freqs, interleaved, 1.0)  # noqa: E731
    for i, j in [(0, 0), (5, 3), (1000, 17)]:
        assert at(q, i) @ at(k, j) == pytest.approx(at(q, i + 411) @ at(k, j + 411), abs=1e-9)
    assert np.array_equal(at(q, 0), q) and np.array_equal(at(q, 7)[32:], q[32:])
    z = at(q, 7)
    a, b = (slice(0, 32, 2), slice(1, 32, 2)) if interleaved else (slice(0, 16), slice(16, 32))
    assert np.allclose(z[a] + 1j * z[b], (q[a] + 1j * q[b]) * np.exp(7j * freqs))


def test_chunk_attention_is_causal_library_attention_and_a_chain_tree(oracle):
    rng = np.random.default_rng(2)
    n, L, Hq, Hkv, D = 6, 9, 4, 2, 64
    q = torch.tensor(rng.standard_normal((n, Hq, D))).bfloat16()
    k, v = (torch.tensor(rng.standard_normal((1, Hkv, L + n, D))).bfloat16() for _ in range(2))
    out, spread = S.chunk_attn(q, k, v, [L], [0, n])
    mask = torch.ones(n, L + n, dtype=torch.bool).tril(L)
    want = torch.nn.functional.scaled_dot_product_attention(q.double().transpose(0, 1)[None], k.double().repeat_interleave(2, 1),
                                                            v.double().repeat_interleave(2, 1), attn_mask=mask)
    assert np.allclose(out, want[0].transpose(0, 1).numpy(), atol=1e-12)
    chain = torch.arange(-1, n - 1, dtype=torch.int32)[None]
    tree = oracle.tree_verify_attn(q[None], k, v, torch.tensor([L], dtype=torch.int32), chain, torch.tensor([n], dtype=torch.int32))
    assert np.allclose(out, tree[0], atol=1e-12)
    assert (spread >= np.abs(out) - 1e-12).all()
    # through a block table
    pages = torch.full((3, Hkv, 16, D), float("nan"), dtype=torch.bfloat16)
    kp, vp = pages.clone(), pages.clone()
    kp[2, :, :15], vp[2, :, :15] = k[0], v[0]
    paged, _ = S.chunk_attn(q, kp, vp, [L], [0, n], block_table=np.array([[2]]))
    assert np.array_equal(paged, out)


def test_logit_adjustment_by_hand():
    z = np.array([[[2.0, -2.0, 1.0, 0.5, 3.0]] * 3])
    # prompt: 0; generated: 1 twice; the tree: node 0 draws 2, its child draws 1
    out = S.logits_adjust(z, np.array([[2, 1]]), np.array([[-1, 0]]), history=np.array([[0, 1, 1, 9]]), history_len=[3], prompt_len=[1],
                          repetition=[2.0], presence=[0.25], frequency=[0.5], bias_tokens=np.array([[4, 4]]), bias_values=np.array([[1.0, 2.0]]),
                          allowed=np.array([[[31], [30], [31]]]))
    base = [1.0, -4.0 - 1.0 - 0.25, 1.0, 0.5, 6.0]
    assert out[0, 0].tolist() == base
    assert out[0, 1].tolist() == [-np.inf, base[1], 0.5 - 0.5 - 0.25, 0.5, 6.0]
    assert out[0, 2].tolist() == [1.0, -4.0 - 1.5 - 0.25, 0.5 - 0.5 - 0.25, 0.5, 6.0]


def test_e4m3_values(oracle):
    table = S.e4m3(np.arange(256))
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(table, want, equal_nan=True)


# ------------------------------------------------------------------------------------------------------------ frequencies
KINDS = [dict(), dict(kind="linear", factor=4.0), dict(kind="ntk", factor=8.0), dict(kind="yarn", factor=16.0, context=4096.0),
         dict(kind="yarn", factor=1.0, context=100.0), dict(kind="banded", factor=8.0, context=8192.0, low=1.0, high=4.0)]


@pytest.mark.parametrize("kw", KINDS)
@pytest.mark.parametrize("dim,base", [(16, 10000.0), (64, 10000.0), (128, 500000.0)])
def test_frequencies_match_the_definition(E, kw, dim, base):
    got, amplitude = E.eagle_rope_frequencies(dim, base, **kw)
    want, want_amplitude = S.rope_frequencies(dim, base, **kw)
    assert np.allclose(got.numpy(), want, rtol=1e-13, atol=0) and amplitude == pytest.approx(want_amplitude, rel=1e-7)


def test_stretched_frequencies_at_their_ends(E):
    plain, _ = E.eagle_rope_frequencies(128)
    yarn, amplitude = E.eagle_rope_frequencies(128, kind="yarn", factor=16.0, context=4096.0)
    assert torch.equal(yarn[:8], plain[:8]) and torch.allclose(yarn[-8:] * 16, plain[-8:], rtol=1e-14) and amplitude > 1
    banded, one = E.eagle_rope_frequencies(128, kind="banded", factor=8.0, context=8192.0, low=1.0, high=4.0)
    assert torch.equal(banded[:8], plain[:8]) and torch.allclose(banded[-8:] * 8, plain[-8:], rtol=1e-14) and one == 1.0
    assert (banded[1:] <= banded[:-1]).all() and (yarn[1:] <= yarn[:-1]).all()
    ntk, _ = E.eagle_rope_frequencies(128, kind="ntk", factor=8.0)
    assert ntk[0] == 1.0 and float(ntk[-1] * 8) == pytest.approx(float(plain[-1]), rel=1e-12)


@pytest.mark.parametrize("dim,kw", [(15, {}), (0, {}), (-2, {}), (64, dict(base=1.0)), (64, dict(base=math.nan)), (64, dict(kind="linear", factor=0.5)),
                                    (64, dict(kind="ntk", factor=math.inf)), (2, dict(kind="ntk", factor=2.0)), (64, dict(kind="yarn", factor=2.0)),
                                    (64, dict(kind="banded", factor=2.0, context=10.0, low=4.0, high=1.0)), (64, dict(kind="other"))])
def test_frequencies_refuse(E, dim, kw):
    with pytest.raises(E.EagleError):
        E.eagle_rope_frequencies(dim, **kw)


# ------------------------------------------------------------------------------------------------------------ refusals
FAKE = 1 << 20       # an aligned address that is never read: every call here is refused, or has nothing to do


def _store(E, **kw):
    f = dict(k=FAKE, v=FAKE, k_scale=None, v_scale=None, kv_capacity=100, block_table=None, num_pages=0, page_size=0, max_pages_per_seq=0)
    f.update(kw)
    return E.KVStoreDesc(**f)


ROPE = dict(batch=2, num_tokens=5, max_tree=4, num_q_heads=4, num_kv_heads=2, head_dim=64, rotary_dim=64, freqs=FAKE)
NULL, SHAPE, WORKSPACE = -1, -2, -3


@pytest.mark.parametrize("tree", [False, True])
def test_rope_append_refuses_before_any_launch(E, tree):
    lib, before = E.load(), E.launch_count()
    fn = lib.eagle_tree_rope_append if tree else lib.eagle_rope_append

    def call(desc=(), store=(), **args):
        a = dict(q=FAKE, k=FAKE, v=FAKE, q_out=2 * FAKE, lens=FAKE, order=FAKE)
        a.update(args)
        d, s = E.RopeDesc(**{**ROPE, **dict(desc)}), _store(E, **dict(store))
        return fn(ctypes.byref(d), a["q"], a["k"], a["v"], a["q_out"], ctypes.byref(s), a["lens"], a["order"], None)

    assert fn(None, FAKE, FAKE, FAKE, FAKE, None, FAKE, FAKE, None) == NULL
    assert fn(ctypes.byref(E.RopeDesc(**ROPE)), FAKE, FAKE, FAKE, FAKE, None, FAKE, FAKE, None) == NULL
    for bad in (dict(batch=-1), dict(batch=65536), dict(head_dim=96), dict(rotary_dim=8), dict(rotary_dim=24), dict(rotary_dim=80), dict(num_kv_heads=0),
                dict(num_q_heads=-1), dict(max_tree=65) if tree else dict(num_tokens=-1), dict(q_stride=255), dict(q_stride=248), dict(k_stride=120),
                dict(v_stride=132), dict(amplitude=math.nan), dict(amplitude=math.inf)):
        assert call(desc=bad) == SHAPE, bad
    for bad, want in ((dict(k=FAKE + 8), SHAPE), (dict(k_scale=FAKE), NULL), (dict(k_scale=FAKE, v_scale=FAKE), SHAPE), (dict(kv_capacity=-1), SHAPE),
                      (dict(block_table=FAKE, num_pages=0, page_size=16, max_pages_per_seq=1), SHAPE),
                      (dict(block_table=FAKE, num_pages=4, page_size=24, max_pages_per_seq=1), SHAPE),
                      (dict(block_table=FAKE, num_pages=4, page_size=8, max_pages_per_seq=1), SHAPE),
                      (dict(block_table=FAKE, num_pages=4, page_size=16, max_pages_per_seq=-1), SHAPE),
                      (dict(block_table=FAKE, num_pages=1 << 30, page_size=16, max_pages_per_seq=1), SHAPE), (dict(k=None), NULL), (dict(v=None), NULL)):
        assert call(store=bad) == want, bad
    for name in ("q", "k", "v", "q_out", "lens", "order"):
        assert call(**{name: None}) == NULL
        if name not in ("lens", "order"):
            assert call(**{name: FAKE + 8}) == SHAPE
    assert call(desc=dict(freqs=None)) == NULL
    assert call(desc=dict(q_stride=512), q_out=FAKE) == SHAPE                       # in place only over the same rows
    assert call(desc=dict(batch=0), q=None) == 0 and call(desc=dict(num_tokens=0, max_tree=0), q=None) == 0
    assert E.launch_count() == before


CHUNK = dict(batch=2, num_tokens=5, num_q_heads=8, num_kv_heads=2, head_dim=128, sm_scale=0.0, workspace=FAKE, workspace_bytes=1 << 40)


def test_chunk_attn_refuses_before_any_launch(E):
    lib, before = E.load(), E.launch_count()

    def call(desc=(), store=(), **args):
        a = dict(q=FAKE, lens=FAKE, start=FAKE, out=FAKE)
        a.update(args)
        d, s = E.ChunkDesc(**{**CHUNK, **dict(desc)}), _store(E, **dict(store))
        return lib.eagle_chunk_attn(ctypes.byref(d), a["q"], ctypes.byref(s), a["lens"], a["start"], a["out"], None)

    assert lib.eagle_chunk_attn(None, FAKE, None, FAKE, FAKE, FAKE, None) == NULL
    for bad in (dict(batch=-1), dict(batch=65536), dict(num_tokens=-1), dict(num_q_heads=9), dict(num_q_heads=34), dict(num_kv_heads=0), dict(head_dim=96),
                dict(sm_scale=-1.0), dict(sm_scale=math.nan), dict(sm_scale=math.inf)):
        assert call(desc=bad) == SHAPE, bad
    assert call(store=dict(k_scale=FAKE, v_scale=FAKE)) == SHAPE                    # fp8 caches are not taken here
    assert call(store=dict(kv_capacity=-1)) == SHAPE and call(store=dict(v=FAKE + 4)) == SHAPE
    for name in ("q", "lens", "start", "out"):
        assert call(**{name: None}) == NULL
    assert call(q=FAKE + 8) == SHAPE and call(out=FAKE + 16) == SHAPE
    assert call(desc=dict(workspace=None)) == WORKSPACE and call(desc=dict(workspace=FAKE + 128)) == WORKSPACE
    need = E.eagle_chunk_attn_workspace(2, 5, 8, 2, 128)
    assert call(desc=dict(workspace_bytes=need - 1)) == WORKSPACE
    assert call(desc=dict(batch=0), q=None) == 0 and call(desc=dict(num_tokens=0), q=None) == 0
    with pytest.raises(E.EagleError):
        E.eagle_chunk_attn_workspace(1, 1, 17, 1, 128)
    assert E.eagle_chunk_attn_workspace(0, 0, 8, 8, 64) > 0
    assert E.launch_count() == before


LOGITS = dict(batch=2, max_tree=3, vocab=100)


def test_logits_adjust_refuses_before_any_launch(E):
    lib, before = E.load(), E.launch_count()

    def call(desc=(), **args):
        a = dict(logits=FAKE, tokens=FAKE, parent=FAKE, out=FAKE)
        a.update(args)
        return lib.eagle_tree_logits_adjust(ctypes.byref(E.LogitsDesc(**{**LOGITS, **dict(desc)})), a["logits"], a["tokens"], a["parent"], a["out"], None)

    assert lib.eagle_tree_logits_adjust(None, FAKE, FAKE, FAKE, FAKE, None) == NULL
    for bad in (dict(batch=-1), dict(batch=65536), dict(max_tree=-1), dict(max_tree=65), dict(vocab=0), dict(vocab=(1 << 30) + 1), dict(history_cap=-1),
                dict(max_bias=-1), dict(max_bias=1025), dict(bf16=1)):              # (bf16: out is the logits' own memory here)
        assert call(desc=bad) == SHAPE, bad
    for name in ("logits", "tokens", "parent", "out"):
        assert call(**{name: None}) == NULL
    assert call(desc=dict(history=FAKE, history_cap=4)) == NULL and call(desc=dict(bias_tokens=FAKE, max_bias=4)) == NULL
    assert call(logits=FAKE + 2) == SHAPE and call(out=FAKE + 2) == SHAPE
    assert call(desc=dict(batch=0), logits=None) == 0
    assert E.launch_count() == before


def test_binding_refuses_host_tensors(E):
    k = torch.zeros(1, 2, 16, 64, dtype=torch.bfloat16)
    kv = E.KVStore(k, k.clone())
    q, lens, start, freqs = torch.zeros(3, 4, 64, dtype=torch.bfloat16), torch.zeros(1, dtype=torch.int32), torch.tensor([0, 3], dtype=torch.int32), torch.ones(32, dtype=torch.float64)
    with pytest.raises(E.EagleError, match="current CUDA device"):
        E.eagle_rope_append(q, q[:, :2], q[:, :2], kv, lens, start, freqs)
    with pytest.raises(E.EagleError, match="current CUDA device"):
        E.eagle_chunk_attn(q, kv, lens, start)
    with pytest.raises(E.EagleError, match="current CUDA device"):
        E.eagle_tree_logits_adjust(torch.zeros(1, 1, 10))
    for bad in (dict(k_scale=torch.ones(1, 2)), dict(block_table=torch.zeros(3, dtype=torch.int32)), dict(block_table=torch.zeros(1, 1))):
        with pytest.raises(E.EagleError):
            E.KVStore(k, k.clone(), **bad)
    with pytest.raises(E.EagleError):
        E.KVStore(k, k[:, :, :8])


def test_chunk_workspace_covers_calls_with_fewer_tokens(E):
    """A workspace sized for a call's most tokens serves every smaller one: the size never falls as tokens are added."""
    for batch in (1, 7, 300, 65535):
        for hq, hkv, d in ((32, 8, 128), (16, 1, 64), (40, 40, 64), (128, 8, 128)):
            counts = sorted({0, 1, batch // 2, batch - 1, batch, batch + 1, 2 * batch, 10 * batch, 100000})
            sizes = [E.eagle_chunk_attn_workspace(batch, n, hq, hkv, d) for n in counts]
            # (calls with no more tokens than sequences run another kernel with other needs)
            few = [s for n, s in zip(counts, sizes) if n <= batch]
            assert few == sorted(few) and all(s >= few[-1] for n, s in zip(counts, sizes) if n > batch)
            assert sizes == sorted(sizes)


def test_the_usual_ends_of_a_band_are_those_of_its_kind():
    from paper_2401_15077_b200 import binding, build
    build.build()
    for kind, low, high in (("banded", 1.0, 4.0), ("yarn", 1.0, 32.0)):
        kw = dict(base=500000.0, kind=kind, factor=8.0, context=8192.0)
        got, amplitude = binding.eagle_rope_frequencies(128, **kw)
        want, amplitude_want = S.rope_frequencies(128, low=low, high=high, **kw)
        assert np.allclose(got.numpy(), want, rtol=1e-12, atol=0) and abs(amplitude - amplitude_want) < 1e-6
        given, _ = binding.eagle_rope_frequencies(128, low=2.0, high=16.0, **kw)
        assert np.allclose(given.numpy(), S.rope_frequencies(128, low=2.0, high=16.0, **kw)[0], rtol=1e-12, atol=0)


def test_row_strides_of_lone_and_missing_rows(E):
    """What stands for the stride in the descriptor (0: dense) when there is no second row."""
    one = torch.zeros(4, 1, 64, dtype=torch.bfloat16)
    assert E._rope_rows(one.transpose(0, 1), "q", torch.Size((1,)), one.device) == (one.data_ptr(), 0)
    assert E._rope_rows(one.transpose(0, 1)[None], "q", torch.Size((1, 1)), one.device) == (one.data_ptr(), 0)
    assert E._rope_rows(one.transpose(0, 1)[:0], "q", torch.Size((0,)), one.device)[1] == 0
    wide = torch.zeros(3, 10, 64, dtype=torch.bfloat16)
    assert E._rope_rows(wide[:, 2:6], "q", torch.Size((3,)), wide.device) == (wide.data_ptr() + 2 * 64 * 2, 640)
    assert E._rope_rows(wide[:, None, 2:6], "q", torch.Size((3, 1)), wide.device)[1] == 640
