"""The calls over a block-scaled cache together, as a serving engine with a sliding window uses them for one layer: prompts in chunks, then
verification steps with top-k, top-p and min-p: the draft tree's keys go into the cache's blocks, windowed tree attention reads them, the target's
and the draft's rows become distributions under the same filters, the walk accepts on them, the path is committed as bytes, the bonus
token becomes the next chunk, and at last plain decoding draws tokens.

Every stage is checked against its 64-bit definition on the inputs it really had (the cache as the GPU holds it), with that stage's own
tolerance; the other test files derive them."""
import numpy as np
import pytest
import torch

import oracle as O
from oracle import serving as S
from oracle.compare import compare_with_oracle

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
B, HQ, HKV, D, T, V, PAGE, PAGES, BLOCK, WINDOW, SINKS = 3, 8, 2, 128, 11, 1200, 32, 30, 16, 70, 3


@pytest.fixture(scope="module")
def E():
    from paper_2401_15077_b200 import binding, build
    build.build()
    binding.load()
    O.build()
    assert torch.cuda.is_available()
    return binding


class Engine:
    def __init__(self, E, seed):
        self.E, self.g, self.r = E, torch.Generator().manual_seed(seed), np.random.default_rng(seed)
        self.k, self.v = (torch.full((PAGES, HKV, PAGE, D), 0x7f, dtype=torch.uint8, device=DEV) for _ in range(2))
        self.ks, self.vs = (torch.full((PAGES, HKV, PAGE // BLOCK), float("nan"), device=DEV) for _ in range(2))
        self.table = torch.randperm(PAGES, generator=self.g).to(torch.int32).view(B, -1).contiguous().to(DEV)
        self.kv = E.KVStore(self.k, self.v, block_table=self.table, k_scale=self.ks, v_scale=self.vs, block_size=BLOCK)
        self.lens = torch.zeros(B, dtype=torch.int32, device=DEV)
        self.freqs, _ = E.eagle_rope_frequencies(D, device=DEV)
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)

    def ok(self):
        torch.cuda.synchronize()
        assert int(self.status.item()) == 0, self.E.status_string(int(self.status.item()))

    def rows(self, *lead):
        return torch.randn(*lead, HQ + 2 * HKV, D, generator=self.g).bfloat16()

    def cache(self):
        return [t.cpu() for t in (self.k, self.v, self.ks, self.vs)]

    def check_append(self, qkv, q_out, before, **order):
        q, k, v = qkv.split((HQ, HKV, HKV), dim=-2)
        rows, res = S.block_append(q, k, v, [t.numpy() for t in before], self.lens.cpu(), self.freqs.cpu().numpy(), BLOCK, block_table=self.table.cpu(), **order)
        live = ~np.isnan(rows)
        assert (np.abs(q_out.cpu().double().numpy() - rows)[live] <= 2.0 ** -8 * np.abs(rows[live]) + 1e-5).all()
        now = self.cache()
        for (values, codes, scales), c, s in zip(res, now[:2], now[2:]):
            c, s = c.numpy(), s.double().numpy()
            assert np.array_equal(s, scales, equal_nan=True)
            new = ~np.isnan(values)
            assert np.array_equal(c[~new], codes[~new])
            best = np.abs(S.e4m3(S.nearest_code(values[new])) - values[new])
            assert (np.abs(S.e4m3(c[new]) - values[new]) <= best + 2e-6 * 448).all()

    def check_attention(self, out, q, **order):
        k, v, ks, vs = self.cache()
        want, spread = S.window_attn(q.cpu(), k, v, self.lens.cpu(), block_table=self.table.cpu(), k_scale=ks, v_scale=vs, block=BLOCK, window=WINDOW,
                                     sinks=SINKS, **order)
        live = ~np.isnan(want)
        err = np.abs(out.cpu().double().numpy() - want)[live]
        assert (err <= 2.0 ** -8 * np.abs(want[live]) + (2.0 ** -11 + 5e-4) * spread[live]).all()

    def chunk(self, n):
        E, starts = self.E, np.concatenate([[0], np.cumsum(n)])
        start = torch.tensor(starts, dtype=torch.int32, device=DEV)
        qkv, before = self.rows(int(starts[-1])), self.cache()
        q, k, v = qkv.to(DEV).split((HQ, HKV, HKV), dim=-2)
        q = E.eagle_block_append(q, k, v, self.kv, self.lens, start, self.freqs, status=self.status)
        out = E.eagle_window_attn(q, self.kv, self.lens, start, window=WINDOW, sinks=SINKS, status=self.status)
        self.ok()
        self.check_append(qkv, q, before, token_start=starts)
        self.check_attention(out, q, token_start=starts)
        self.lens += torch.tensor(n, dtype=torch.int32, device=DEV)

    def verify(self):
        E, sizes = self.E, [int(x) for x in self.r.integers(1, T + 1, B)]
        parent = np.full((B, T), 2 ** 30, dtype=np.int32)
        for b, m in enumerate(sizes):
            for i in range(m):
                parent[b, i] = self.r.integers(-1, i)
        tree, size = torch.tensor(parent, device=DEV), torch.tensor(sizes, dtype=torch.int32, device=DEV)
        qkv, before = self.rows(B, T), self.cache()
        q, k, v = qkv.to(DEV).split((HQ, HKV, HKV), dim=-2)
        q_out = torch.zeros(B, T, HQ, D, dtype=torch.bfloat16, device=DEV)
        E.eagle_tree_block_append(q, k, v, self.kv, self.lens, tree, self.freqs, q_out, tree_sizes=size, status=self.status)
        out = E.eagle_tree_window_attn(q_out, self.kv, self.lens, tree, tree_sizes=size, window=WINDOW, sinks=SINKS, status=self.status)
        self.ok()
        order = {"tree_parent": torch.tensor(parent), "tree_sizes": sizes}
        self.check_append(qkv, q_out, before, **order)
        self.check_attention(out, q_out, **order)
        # ---- distributions under one set of filters, draft rows near the target's
        z = torch.randn(B, T + 1, V, generator=self.g) * 2
        zd = torch.stack([torch.stack([z[b, (parent[b, i] if i < sizes[b] else -1) + 1] for i in range(T)]) for b in range(B)])
        zd = zd + 0.3 * torch.randn(zd.shape, generator=self.g)
        kw = {"temperature": torch.tensor([0.9, 0.0, 0.7]), "top_k": torch.tensor([0, 0, 300]).int(), "top_p": torch.tensor([0.95, 1.0, 0.9]),
              "min_p": torch.tensor([0.0, 0.0, 0.01])}
        on = {n: t.to(DEV) for n, t in kw.items()}
        tokens, small = E.eagle_sample(zd.to(DEV), torch.rand(B, T, generator=self.g).to(DEV), num_rows=size, with_probs=True, status=self.status, **on)
        target = torch.zeros(B, T + 1, V, device=DEV)
        E.eagle_sample(z.to(DEV), probs=target, num_rows=size + 1, status=self.status, **on)
        self.ok()
        for b in range(B):
            each = {n: t[b].item() for n, t in kw.items()}
            for r in range(sizes[b] + 1):
                want = S.sample(z[b, r].numpy(), None, **each)[1]
                assert (np.abs(target[b, r].cpu().double().numpy() - want) <= (2.0 ** -24 + 1e-9) * want).all()
            for r in range(sizes[b]):
                want = S.sample(zd[b, r].numpy(), None, **each)[1]
                assert want[int(tokens[b, r])] > 0
        # ---- walk and commit
        uniforms, greedy = torch.rand(B, T + 1, generator=self.g), torch.tensor([0, 1, 0], dtype=torch.uint8)
        live = torch.arange(T)[None, :, None] < torch.tensor(sizes)[:, None, None]
        small, tokens = torch.where(live.to(DEV), small, 0.0), torch.where(live[:, :, 0].to(DEV), tokens, 0)
        alen = torch.zeros(B, dtype=torch.int32, device=DEV)
        path, bonus = E.eagle_tree_accept(target, small, tokens, tree, uniforms.to(DEV), tree_sizes=size, greedy=greedy.to(DEV), accept_len=alen, status=self.status)
        values = [S.e4m3(c.cpu().numpy()) * s.cpu().double().numpy().repeat(BLOCK, -1)[..., None] for c, s in ((self.k, self.ks), (self.v, self.vs))]
        new_len, _ = E.eagle_tree_commit_paged(self.k.view(torch.bfloat16), self.v.view(torch.bfloat16), self.table, self.lens, path, T, status=self.status)
        self.ok()
        r = O.tree_accept(target.cpu(), small.cpu(), tokens.cpu(), tree.cpu(), uniforms, tree_sizes=size.cpu(), greedy=greedy)
        compare_with_oracle(r, path.cpu().numpy(), bonus.cpu().numpy(), alen.cpu().numpy(), greedy.numpy())
        now = [S.e4m3(c.cpu().numpy()) * s.cpu().double().numpy().repeat(BLOCK, -1)[..., None] for c, s in ((self.k, self.ks), (self.v, self.vs))]
        table = self.table.cpu().numpy()
        for b in range(B):                                   # the accepted nodes' keys and values, wherever they lay
            L = int(self.lens[b])
            for j, node in enumerate(path[b, :int(alen[b])].tolist()):
                at, to = S.place_of(b, L + node, table, PAGE), S.place_of(b, L + j, table, PAGE)
                for was, x in zip(values, now):
                    assert np.array_equal(was[at[0], :, at[1]], x[to[0], :, to[1]])
        self.lens = new_len
        return alen.cpu().tolist()


def test_prompts_then_verification_steps_then_decoding(E):
    engine = Engine(E, 31)
    engine.chunk([64, 3, 0])
    engine.chunk([6, 0, 141])
    accepted = []
    for _ in range(4):
        accepted += engine.verify()
        engine.chunk([1, 1, 1])              # the step's extra token has no keys yet
    assert max(accepted) > 0
    z, u = torch.randn(B, 1, V, generator=engine.g).bfloat16(), torch.rand(B, 1, generator=engine.g)
    tokens, _ = E.eagle_sample(z.to(DEV), u.to(DEV), top_p=torch.full((B,), 0.8, device=DEV), status=engine.status)
    engine.ok()
    for b in range(B):
        t, _, margin = S.sample(z[b, 0].float().numpy(), float(u[b, 0]), top_p=float(np.float32(0.8)))
        assert margin < 1e-9 or int(tokens[b, 0]) == t
