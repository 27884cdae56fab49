"""The calls around verification together with it, as a serving engine uses them for one layer: two chunks of every prompt go
into a paged cache and attend it, then verification steps run: the draft tree's keys go in, tree attention reads them, the target's
rows are adjusted, the walk accepts, the path is committed, and the bonus token of the step becomes the next chunk.

Every stage is checked against its 64-bit definition on the inputs it really had (the cache as the GPU holds it, the adjusted logits
that the walk reads), with that stage's own tolerance: the next stage's inputs are the GPU's."""
import numpy as np
import pytest
import torch

import oracle as O
from oracle import serving as S
from oracle.compare import compare_with_oracle

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
B, HQ, HKV, D, T, V, PAGE, PAGES = 3, 8, 2, 128, 11, 1200, 16, 48


@pytest.fixture(scope="module")
def E():
    from paper_2401_15077_b200 import binding, build
    build.build()
    binding.load()
    O.build()
    assert torch.cuda.is_available()
    return binding


class Engine:
    """One layer of three sequences over a pool of pages; `lens` is the committed length of each."""

    def __init__(self, E, seed):
        self.E, self.g, self.r = E, torch.Generator().manual_seed(seed), np.random.default_rng(seed)
        self.k, self.v = (torch.full((PAGES, HKV, PAGE, D), float("nan"), dtype=torch.bfloat16, device=DEV) for _ in range(2))
        order = torch.randperm(PAGES, generator=self.g).to(torch.int32)
        self.table = order.view(B, -1).contiguous().to(DEV)
        self.kv = E.KVStore(self.k, self.v, block_table=self.table)
        self.lens = torch.zeros(B, dtype=torch.int32, device=DEV)
        self.freqs, self.amplitude = E.eagle_rope_frequencies(D, kind="yarn", factor=4.0, context=256.0, device=DEV)
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)

    def ok(self):
        torch.cuda.synchronize()
        assert int(self.status.item()) == 0, self.E.status_string(int(self.status.item()))

    def rows(self, *lead):
        return torch.randn(*lead, HQ + 2 * HKV, D, generator=self.g).bfloat16()

    def cache(self):
        return self.k.cpu(), self.v.cpu(), self.table.cpu()

    def check_rotary(self, qkv, q_out, before, **where):
        q, k, v = qkv.split((HQ, HKV, HKV), dim=-2)
        want, stored = S.rope_append(q, k, v, self.lens.cpu(), self.freqs.cpu().numpy(), amplitude=self.amplitude, **where)
        live = ~np.isnan(want)
        loose = 8e-7 * 2 * float(qkv.double().abs().max()) * self.amplitude
        assert (np.abs(q_out.cpu().double().numpy() - want)[live] <= 2.0 ** -8 * np.abs(want[live]) + loose).all()
        ck, cv, table = self.cache()
        for b, slot, key, value in stored:
            page, row = S.place_of(b, slot, table.numpy(), PAGE)
            assert (np.abs(ck[page, :, row].double().numpy() - key) <= 2.0 ** -8 * np.abs(key) + loose).all()
            assert np.array_equal(cv[page, :, row].double().numpy(), value)
            before[0][page, :, row], before[1][page, :, row] = ck[page, :, row], cv[page, :, row]
        assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(before, (ck, cv)))

    def chunk(self, n):
        """New tokens of every sequence: into the cache, attended, committed."""
        E, starts = self.E, np.concatenate([[0], np.cumsum(n)])
        start = torch.tensor(starts, dtype=torch.int32, device=DEV)
        qkv, before = self.rows(int(starts[-1])), self.cache()[:2]
        q, k, v = qkv.to(DEV).split((HQ, HKV, HKV), dim=-2)
        q = E.eagle_rope_append(q, k, v, self.kv, self.lens, start, self.freqs, amplitude=self.amplitude, status=self.status)
        out = E.eagle_chunk_attn(q, self.kv, self.lens, start, status=self.status)
        self.ok()
        self.check_rotary(qkv, q, before, token_start=starts)
        ck, cv, table = self.cache()
        want, spread = S.chunk_attn(q.cpu(), ck, cv, self.lens.cpu(), starts, block_table=table)
        err = np.abs(out.cpu().double().numpy() - want)
        assert (err <= 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 5e-4) * spread).all()
        self.lens += torch.tensor(n, dtype=torch.int32, device=DEV)

    def verify(self, history, prompt_len):
        E, sizes = self.E, [int(x) for x in self.r.integers(1, T + 1, B)]
        parent = np.full((B, T), 2 ** 30, dtype=np.int32)
        for b, m in enumerate(sizes):
            for i in range(m):
                parent[b, i] = self.r.integers(-1, i)
        tree, size = torch.tensor(parent, device=DEV), torch.tensor(sizes, dtype=torch.int32, device=DEV)
        # ---- keys of the tree, tree attention
        qkv, before = self.rows(B, T), self.cache()[:2]
        q, k, v = qkv.to(DEV).split((HQ, HKV, HKV), dim=-2)
        q_out = torch.zeros(B, T, HQ, D, dtype=torch.bfloat16, device=DEV)
        E.eagle_tree_rope_append(q, k, v, self.kv, self.lens, tree, self.freqs, q_out, tree_sizes=size, amplitude=self.amplitude, status=self.status)
        out = E.eagle_tree_verify_attn_paged(q_out, self.k, self.v, self.table, self.lens, tree, tree_sizes=size, status=self.status)
        self.ok()
        self.check_rotary(qkv, q_out, before, tree_parent=parent, tree_sizes=sizes)
        ck, cv, table = self.cache()
        ref = O.tree_verify_attn_paged(q_out.cpu(), ck, cv, table, self.lens.cpu(), tree.cpu(), size.cpu())
        err = np.abs(out.cpu().double().numpy() - ref)
        assert err.max() <= 2e-2 and err.mean() <= 2e-3
        # ---- logits: draft rows are near the target's, so that nodes are accepted
        z = torch.randn(B, T + 1, V, generator=self.g) * 2
        draft = torch.stack([torch.stack([z[b, (parent[b, i] if i < sizes[b] else -1) + 1] for i in range(T)]) for b in range(B)])
        draft = draft + 0.3 * torch.randn(draft.shape, generator=self.g)
        tokens = torch.distributions.Categorical(logits=draft).sample().to(torch.int32)
        h = torch.zeros(B, max(len(x) for x in history), dtype=torch.int32)
        for b, x in enumerate(history):
            h[b, :len(x)] = torch.tensor(x, dtype=torch.int32)
        allowed = torch.tensor(self.r.integers(-2 ** 31, 2 ** 31, (B, T + 1, (V + 31) // 32)) | 0x55555555, dtype=torch.int64).to(torch.int32)
        kw = dict(tree_sizes=size.cpu(), history=h, history_len=torch.tensor([len(x) for x in history], dtype=torch.int32),
                  prompt_len=torch.tensor(prompt_len, dtype=torch.int32), repetition=torch.tensor([1.2, 1.0, 0.8]),
                  presence=torch.tensor([0.1, 0.0, -0.2]), frequency=torch.tensor([0.05, 0.2, 0.0]),
                  bias_tokens=torch.tensor([[1, 1], [5, 6], [7, 8]], dtype=torch.int32), bias_values=torch.tensor([[0.5, 0.25], [9.0, -9.0], [0.0, 1.0]]),
                  allowed=allowed)
        adjusted = torch.full(z.shape, -1e30, device=DEV)
        E.eagle_tree_logits_adjust(z.to(DEV), tokens.to(DEV), tree, adjusted, status=self.status, **{n: t.to(DEV) for n, t in kw.items()})
        self.ok()
        want = S.logits_adjust(z, tokens, parent, **{**kw, "tree_sizes": sizes})
        live, got = np.isfinite(want), adjusted.cpu().double().numpy()
        assert (np.abs(got - want)[live] <= 1e-6 * (np.abs(z.double().numpy()) * 2 + 20)[live]).all() and np.isneginf(got[np.isneginf(want)]).all()
        # ---- walk and commit
        uniforms, greedy = torch.rand(B, T + 1, generator=self.g), torch.tensor([0, 1, 0], dtype=torch.uint8)
        alen = torch.zeros(B, dtype=torch.int32, device=DEV)
        path, bonus = E.eagle_tree_accept_logits(adjusted, draft.to(DEV), tokens.to(DEV), tree, uniforms.to(DEV), 0.9, tree_sizes=size, greedy=greedy.to(DEV),
                                                 accept_len=alen, status=self.status)
        new_len, _ = E.eagle_tree_commit_paged(self.k, self.v, self.table, self.lens, path, T, status=self.status)
        self.ok()
        r = O.tree_accept_logits(adjusted.cpu(), draft, tokens, tree.cpu(), uniforms, 0.9, tree_sizes=size.cpu(), greedy=greedy)
        compare_with_oracle(r, path.cpu().numpy(), bonus.cpu().numpy(), alen.cpu().numpy(), greedy.numpy())
        c = O.tree_commit_paged(ck, cv, table, self.lens.cpu(), path.cpu(), T)
        assert np.array_equal(new_len.cpu().numpy(), c["new_seq_lens"])
        for mine, ref in ((self.k, c["k_pages"]), (self.v, c["v_pages"])):
            assert np.array_equal(mine.cpu().view(torch.int16).numpy().view(np.uint16), ref)
        self.lens = new_len
        for b in range(B):
            for node in path[b].tolist():
                if node >= 0:
                    history[b].append(int(tokens[b, node]))
            token = int(bonus[b])
            assert (int(allowed[b, (int(path[b, int(alen[b]) - 1]) if int(alen[b]) else -1) + 1, token // 32]) >> (token % 32)) & 1, "a masked token was drawn"
            history[b].append(token)
        return alen.cpu().tolist()


def test_prompts_then_verification_steps(E):
    engine = Engine(E, 21)
    prompt = [70, 3, 41]
    engine.chunk([64, 3, 0])
    engine.chunk([6, 0, 41])
    assert engine.lens.tolist() == prompt
    history, accepted = [[int(x) for x in engine.r.integers(0, V, n)] for n in prompt], []
    for _ in range(4):
        accepted += engine.verify(history, prompt)
        engine.chunk([1, 1, 1])              # the step's extra token has no keys yet
        assert engine.lens.tolist() == [len(h) for h in history]
    assert max(accepted) > 0


def test_a_short_chunk_is_a_chain_tree(E):
    """Chunks of up to 64 tokens are what tree attention computes on a chain: the two kernels agree within their roundings."""
    engine = Engine(E, 22)
    engine.chunk([90, 17, 33])
    n = 23
    qkv = engine.rows(B, n)
    q, k, v = (x.contiguous() for x in qkv.to(DEV).split((HQ, HKV, HKV), dim=-2))
    chain = torch.arange(-1, n - 1, dtype=torch.int32, device=DEV)
    start = torch.arange(0, (B + 1) * n, n, dtype=torch.int32, device=DEV)
    q_tree = E.eagle_tree_rope_append(q, k, v, engine.kv, engine.lens, chain, engine.freqs, shared_tree=True)
    ck, cv, _ = engine.cache()
    q_chunk = E.eagle_rope_append(q.flatten(0, 1), k.flatten(0, 1), v.flatten(0, 1), engine.kv, engine.lens, start, engine.freqs)
    assert torch.equal(q_tree.flatten(0, 1), q_chunk)
    assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip((ck, cv), engine.cache()))
    a = E.eagle_tree_verify_attn_paged(q_tree, engine.k, engine.v, engine.table, engine.lens, chain, shared_tree=True).flatten(0, 1)
    b = E.eagle_chunk_attn(q_chunk, engine.kv, engine.lens, start)
    _, spread = S.chunk_attn(q_chunk.cpu(), ck, cv, engine.lens.cpu(), start.cpu().numpy(), block_table=engine.table.cpu())
    # each side is off by the rounding of its output and of its probabilities
    far = np.abs(a.cpu().double().numpy() - b.cpu().double().numpy())
    assert (far <= 2 * (2.0 ** -8 * np.abs(b.cpu().double().numpy()) + (2.0 ** -8 + 5e-4) * spread) + 1e-6).all()


def test_calls_on_two_streams_with_workspaces_of_their_own(E):
    """Independent calls may overlap: each has its own workspace (torch's allocator hands it out per stream)."""
    torch.cuda.synchronize()
    cases = []
    for seed in (1, 2):
        g = torch.Generator().manual_seed(seed)
        k, v = (torch.randn(4, HKV, 700, D, generator=g).bfloat16().to(DEV) for _ in range(2))
        q = torch.randn(4 * 50, HQ, D, generator=g).bfloat16().to(DEV)
        lens = torch.tensor([600, 10, 333, 0], dtype=torch.int32, device=DEV)
        start = torch.arange(0, 201, 50, dtype=torch.int32, device=DEV)
        cases.append((q, E.KVStore(k, v), lens, start, E.eagle_chunk_attn(q, E.KVStore(k, v), lens, start)))
    torch.cuda.synchronize()
    streams, outs = [torch.cuda.Stream() for _ in cases], [[], []]
    for _ in range(5):
        for i, (q, kv, lens, start, _) in enumerate(cases):
            with torch.cuda.stream(streams[i]):
                outs[i].append(E.eagle_chunk_attn(q, kv, lens, start))
    torch.cuda.synchronize()
    for i, c in enumerate(cases):
        assert all(torch.equal(o.view(torch.int16), c[4].view(torch.int16)) for o in outs[i])
