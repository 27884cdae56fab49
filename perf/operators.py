"""What is measured of the operators around tree verification: rotary positions with the write into the cache, attention of a chunk of
new tokens over that cache, and penalties, biases and grammar masks on the logits that acceptance reads.

A case is a dict of plain values; `prepare` makes its inputs from a seed, `run` is one pass through the operator (the plain form in
elementary torch operations, or with `own` the library's call), `exact` the same from the definitions in 64 bits, and `work` what a
pass cannot do without.  Ragged lengths follow from the case alone (its number "mix"), everything else from the seed."""
import math
import random

import torch

own = False
DEV = "cuda"


# ------------------------------------------------------------------------------------------------------------------ cases
def _rope(name, form, heads, head_dim, batch, n_lo, n_hi, l_lo, l_hi, page, fp8=False, rotary=None, interleaved=False, amplitude=1.0, mix=1):
    return {"name": name, "op": "rope", "form": form, "hq": heads[0], "hkv": heads[1], "d": head_dim, "batch": batch, "n_lo": n_lo, "n_hi": n_hi,
            "l_lo": l_lo, "l_hi": l_hi, "page": page, "fp8": fp8, "rotary": rotary or head_dim, "interleaved": interleaved,
            "amplitude": amplitude, "mix": mix}


def _attn(name, heads, head_dim, batch, chunks, n_lo, n_hi, l_lo, l_hi, page, mix=1):
    return {"name": name, "op": "attn", "hq": heads[0], "hkv": heads[1], "d": head_dim, "batch": batch, "chunks": chunks, "n_lo": n_lo,
            "n_hi": n_hi, "l_lo": l_lo, "l_hi": l_hi, "page": page, "mix": mix}


def _logits(name, batch, t_lo, t_hi, vocab, history, bf16=False, penalties=True, bias=0, grammar=False, mix=1):
    return {"name": name, "op": "logits", "batch": batch, "t_lo": t_lo, "t_hi": t_hi, "vocab": vocab, "history": history, "bf16": bf16,
            "penalties": penalties, "bias": bias, "grammar": grammar, "mix": mix}


def listed():
    return [
        # one sequence's next token, 32 heads without groups: a call's latency
        _rope("rope_one_token", "chunk", (32, 32), 128, 1, 1, 1, 2048, 2048, 0),
        # the draft trees of a serving batch (16 to 64 nodes over prefixes of 512 to 8192) on their way into a paged cache
        _rope("rope_trees_paged", "tree", (32, 8), 128, 64, 16, 64, 512, 8192, 64),
        # a long prompt's chunk far into the context (scaled frequencies change the amplitude too)
        _rope("rope_prompt_far", "chunk", (64, 8), 128, 1, 8192, 8192, 98304, 98304, 64, amplitude=1.2079),
        # ragged chunks into an fp8 cache, half of each head rotated, pairs next to one another
        _rope("rope_ragged_fp8", "chunk", (32, 8), 128, 23, 0, 611, 0, 5000, 32, fp8=True, rotary=64, interleaved=True),
        # every sequence's next token over a paged cache: the keys and values are read once for a few rows
        _attn("attn_decode", (32, 8), 128, 64, 64, 1, 1, 512, 8192, 64),
        # one token over one long context: only a split of the context fills the machine
        _attn("attn_one_long", (64, 8), 128, 1, 1, 1, 1, 65536, 65536, 64),
        # two chunks of prompts beside single tokens, in odd sizes
        _attn("attn_mixed", (32, 8), 128, 25, 2, 500, 1003, 100, 4001, 32),
        # a whole prompt at once, heads without groups, contiguous cache
        _attn("attn_prompt", (32, 32), 128, 1, 1, 4096, 4096, 0, 0, 0),
        # chunks of two prompts over long prefixes: the tensor cores' case
        _attn("attn_prompt_long", (32, 8), 128, 2, 2, 2048, 2048, 16384, 16384, 64),
        # short ragged prompts with small heads
        _attn("attn_ragged_d64", (16, 4), 64, 9, 9, 0, 701, 0, 300, 16),
        # the target's rows of a serving batch of draft trees, everything switched on
        _logits("logits_trees", 64, 16, 64, 32000, 4096, bias=100, grammar=True),
        # plain decoding: one row a sequence, as the output layer leaves it, a large odd vocabulary
        _logits("logits_rows_bf16", 16, 0, 0, 129537, 2000, bf16=True),
    ]


HEADS = ((8, 8), (16, 4), (32, 8), (32, 32), (64, 8), (12, 3), (10, 2), (7, 1), (16, 1))


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op, mix = rng.choice(("rope", "rope", "attn", "attn", "logits")), rng.randrange(1 << 20)
    heads, d = rng.choice(HEADS), rng.choice((64, 128, 128))
    if op == "rope":
        fp8 = d == 128 and rng.random() < 0.4
        rotary = rng.choice((d, d, 16 * rng.randint(1, d // 16)))
        more = dict(fp8=fp8, rotary=rotary, interleaved=rng.random() < 0.5, amplitude=rng.choice((1.0, 1.0, 1.1386)), mix=mix)
        page = rng.choice((0, 16, 32, 64, 128, 256))
        if rng.random() < 0.4:
            n, b, far = rng.randint(1, 64), _log(rng, 1, 64), _log(rng, 1, 8192)
            c = _rope("", "tree", heads, d, b, rng.randint(1, n), n, rng.randint(0, far), far, page, **more)
        else:
            n, b = _log(rng, 1, 4096), _log(rng, 1, 32)
            n = min(n, max(1, 8192 // b))
            far = _log(rng, 1, max(2, 65536 // b))
            c = _rope("", "chunk", heads, d, b, rng.randint(0, n), n, rng.randint(0, far), far, page, **more)
    elif op == "attn":
        b, n, far = _log(rng, 1, 64), _log(rng, 1, 4096), _log(rng, 1, 65536)
        chunks = rng.choice((b, 1 + rng.randrange(b)))
        # what the plain form holds at once, and the operations, stay below those of the largest listed case
        while b * heads[0] * n * (n + far) > 2.0e9 or b * heads[1] * (n + far) * d > 5.0e8:
            n, far = max(1, n * 2 // 3), max(1, far * 4 // 5)
        c = _attn("", heads, d, b, chunks, rng.randint(0, n), n, rng.randint(0, far), far, rng.choice((0, 16, 32, 64, 128, 256)), mix=mix)
    else:
        t = rng.choice((0, rng.randint(1, 64)))
        vocab = _log(rng, 1000, 150000)
        b = max(1, min(_log(rng, 1, 64), int(1.2e8 / (vocab * (t + 1)))))
        c = _logits("", b, rng.randint(0, t), t, vocab, _log(rng, 1, 8192), bf16=rng.random() < 0.5, penalties=rng.random() < 0.8,
                    bias=rng.choice((0, rng.randint(1, 300))), grammar=rng.random() < 0.5, mix=mix)
    del c["name"]
    return c


def _lengths(c):
    """(new tokens, prefix) of every sequence; a tree has n_hi nodes at the most."""
    r = random.Random(c["mix"])
    n = [c["n_hi"]] + [r.randint(c["n_lo"], c["n_hi"]) for _ in range(c["batch"] - 1)]
    if c["op"] == "attn":
        n = [v if i < c["chunks"] else 1 for i, v in enumerate(n)]
    return n, [r.randint(c["l_lo"], c["l_hi"]) for _ in range(c["batch"])]


def _tree_sizes(c):
    r = random.Random(c["mix"])
    return [c["t_hi"]] + [r.randint(c["t_lo"], c["t_hi"]) for _ in range(c["batch"] - 1)]


# ------------------------------------------------------------------------------------------------------------------ inputs
def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _parents(r, n, max_depth=6):
    """A random tree: every node hangs below an earlier one that is not too deep, or below the context (-1)."""
    parent, depth = [], []
    for i in range(n):
        p = r.randint(-1, i - 1)
        while p >= 0 and depth[p] >= max_depth:
            p = parent[p]
        parent.append(p)
        depth.append(1 if p < 0 else depth[p] + 1)
    return parent


def _cache(c, lengths, g, r):
    """The cache (random throughout: what earlier sequences left behind is there too), its block table and scales."""
    kv, d, batch, page = c["hkv"], c["d"], c["batch"], c["page"]
    need = [a + b for a, b in zip(*lengths)]
    if page:
        used = [-(-v // page) for v in need]
        pages, per = sum(used) + 3, max(max(used), 1)
        free, table = list(range(pages)), []
        r.shuffle(free)
        for u in used:
            table.append([free.pop() for _ in range(u)] + [-1] * (per - u))
        shape, table = (pages, kv, page, d), _ints(table)
    else:
        shape, table = (batch, kv, max(max(need), 1) + 5, d), None
    if c.get("fp8"):
        k, v = (torch.randint(0, 120, shape, dtype=torch.uint8, device=DEV, generator=g) for _ in range(2))
        scales = [torch.rand(batch, kv, device=DEV, generator=g) * 0.01 + 0.005 for _ in range(2)]
    else:
        k, v = (torch.randn(shape, dtype=torch.bfloat16, device=DEV, generator=g) for _ in range(2))
        scales = [None, None]
    return {"k": k, "v": v, "table": table, "k_scale": scales[0], "v_scale": scales[1]}


def prepare(case, seed):
    c, g, r = case, torch.Generator(device=DEV).manual_seed(seed), random.Random(seed)
    if c["op"] == "logits":
        return _prepare_logits(c, g, r)
    n, prefix = lengths = _lengths(c)
    s = {"c": c, "cache": _cache(c, lengths, g, r), "seq_lens": _ints(prefix), "n": n, "prefix": prefix}
    tree = c.get("form") == "tree"
    rows = c["batch"] * c["n_hi"] if tree else sum(n)
    lead = (c["batch"], c["n_hi"]) if tree else (rows,)
    starts = [0]
    for v in n:
        starts.append(starts[-1] + v)
    s["token_start"] = _ints(starts)
    if tree:
        s["tree_sizes"] = _ints(n)
        s["tree_parent"] = _ints([_parents(r, v) + [0] * (c["n_hi"] - v) for v in n])
    if c["op"] == "rope":
        # queries, keys and values as one projection leaves them: side by side in a row
        heads = c["hq"] + 2 * c["hkv"]
        s["qkv"] = torch.randn(*lead, heads, c["d"], dtype=torch.bfloat16, device=DEV, generator=g)
        i = torch.arange(c["rotary"] // 2, dtype=torch.float64, device=DEV)
        s["freqs"] = torch.pow(torch.tensor(10000.0, dtype=torch.float64, device=DEV), -2.0 * i / c["rotary"])
        s["q_out"] = torch.zeros(*lead, c["hq"], c["d"], dtype=torch.bfloat16, device=DEV)
    else:
        s["q"] = torch.randn(rows, c["hq"], c["d"], dtype=torch.bfloat16, device=DEV, generator=g)
    return s


def _prepare_logits(c, g, r):
    b, t, v = c["batch"], c["t_hi"], c["vocab"]
    sizes = _tree_sizes(c)
    s = {"c": c, "sizes": sizes, "tree_sizes": _ints(sizes)}
    z = torch.randn(b, t + 1, v, device=DEV, generator=g) * 2.0
    s["logits"] = z.to(torch.bfloat16) if c["bf16"] else z
    s["out"] = torch.zeros(b, t + 1, v, device=DEV)
    s["tree_parent"] = _ints([_parents(r, n) + [0] * (t - n) for n in sizes]).reshape(b, t)
    # tokens as text has them: a few often, most seldom
    often = lambda *shape: (torch.rand(*shape, device=DEV, generator=g).pow(4.0) * v).to(torch.int32).clamp_(0, v - 1)  # noqa: E731
    s["draft_tokens"] = often(b, t)
    if c["penalties"]:
        s["history"] = often(b, c["history"])
        s["history_len"] = _ints([c["history"]] + [r.randint(0, c["history"]) for _ in range(b - 1)])
        s["prompt_len"] = (s["history_len"].double() * torch.rand(b, device=DEV, generator=g)).to(torch.int32)
        s["repetition"] = 1.0 + 0.5 * torch.rand(b, device=DEV, generator=g)
        s["presence"] = torch.rand(b, device=DEV, generator=g)
        s["frequency"] = 0.5 * torch.rand(b, device=DEV, generator=g)
    if c["bias"]:
        s["bias_tokens"] = torch.stack([torch.randperm(v, device=DEV, generator=g)[: c["bias"]] for _ in range(b)]).to(torch.int32)
        s["bias_values"] = torch.randn(b, s["bias_tokens"].shape[1], device=DEV, generator=g) * 3.0
        s["bias_len"] = _ints([r.randint(0, s["bias_tokens"].shape[1]) for _ in range(b)])
    if c["grammar"]:
        words = -(-v // 32)
        s["allowed"] = torch.randint(-(1 << 31), 1 << 31, (b, t + 1, words), dtype=torch.int32, device=DEV, generator=g)
    return s


# ------------------------------------------------------------------------------------------------------------------ one pass
def run(state):
    s, c = state, state["c"]
    if c["op"] == "rope":
        return _own_rope(s, c) if own else _plain_rope(s, c)
    if c["op"] == "attn":
        return _own_attn(s) if own else _plain_attn(s, c)
    return _own_logits(s) if own else _plain_logits(s, c)


def _own_store(s):
    from paper_2401_15077_b200 import binding as E
    a = s["cache"]
    return E, E.KVStore(a["k"], a["v"], block_table=a["table"], k_scale=a["k_scale"], v_scale=a["v_scale"])


def _own_rope(s, c):
    E, store = _own_store(s)
    q, k, v = s["qkv"].split((c["hq"], c["hkv"], c["hkv"]), dim=-2)
    more = {"interleaved": c["interleaved"], "amplitude": c["amplitude"]}
    if c["form"] == "tree":
        q = E.eagle_tree_rope_append(q, k, v, store, s["seq_lens"], s["tree_parent"], s["freqs"], s["q_out"], tree_sizes=s["tree_sizes"], **more)
    else:
        q = E.eagle_rope_append(q, k, v, store, s["seq_lens"], s["token_start"], s["freqs"], s["q_out"], **more)
    return _cache_out(s, q)


def _own_attn(s):
    E, store = _own_store(s)
    return E.eagle_chunk_attn(s["q"], store, s["seq_lens"], s["token_start"])


def _own_logits(s):
    from paper_2401_15077_b200 import binding as E
    names = ("history", "history_len", "prompt_len", "repetition", "presence", "frequency", "bias_tokens", "bias_values", "bias_len", "allowed")
    return E.eagle_tree_logits_adjust(s["logits"], s["draft_tokens"], s["tree_parent"], s["out"], tree_sizes=s["tree_sizes"],
                                      **{n: s[n] for n in names if n in s})


def _cache_out(s, q):
    a = s["cache"]
    if a["k_scale"] is None:
        return {"q": q, "k": a["k"], "v": a["v"]}
    return {"q": q, "k": a["k"].view(torch.float8_e4m3fn), "v": a["v"].view(torch.float8_e4m3fn)}


def _owners(s, rows):
    """The sequence of every packed token and its place in the chunk."""
    at = torch.arange(rows, device=DEV)
    seq = torch.searchsorted(s["token_start"].long(), at, right=True) - 1
    return seq, at - s["token_start"].long()[seq]


def _ancestors(parent, sizes):
    """[b, i, m]: 1 where m is node i or one of its ancestors; nothing for nodes past the tree's size."""
    b, t = parent.shape
    at = torch.arange(t, device=DEV)
    live = (at[None] < sizes[:, None]).float()
    up = (parent.long()[:, :, None] == at[None, None]).float() * live[:, :, None]
    reach = torch.eye(t, device=DEV)[None] * live[:, :, None] + up
    for _ in range(6):  # paths of up to 64 nodes
        reach = (reach @ reach).clamp_(max=1.0)
    return reach


def _plain_rope(s, c):
    q, k, v = s["qkv"].split((c["hq"], c["hkv"], c["hkv"]), dim=-2)
    a, half = s["cache"], c["rotary"] // 2
    if c["form"] == "tree":
        b, t = s["tree_parent"].shape
        depth = _ancestors(s["tree_parent"], s["tree_sizes"]).sum(2).long()
        seq, node = torch.arange(b, device=DEV).repeat_interleave(t), torch.arange(t, device=DEV).repeat(b)
        live = node < s["tree_sizes"].long()[seq]
        place, slot = s["seq_lens"].long()[seq] + depth.flatten() - 1, s["seq_lens"].long()[seq] + node
        q, k, v = (x.flatten(0, 1) for x in (q, k, v))
    else:
        seq, node = _owners(s, q.shape[0])
        live, place = None, s["seq_lens"].long()[seq] + node
        slot = place
    angle = place.double()[:, None] * s["freqs"][None]
    cos, sin = (f(angle).float()[:, None] * c["amplitude"] for f in (torch.cos, torch.sin))

    def turned(x):
        x = x.float()
        y = x.clone()
        i, j = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if c["interleaved"] else (slice(0, half), slice(half, 2 * half))
        y[..., i], y[..., j] = x[..., i] * cos - x[..., j] * sin, x[..., j] * cos + x[..., i] * sin
        return y

    q, k, v = turned(q).to(torch.bfloat16), turned(k), v.float()
    if live is not None:
        keep = live.nonzero().flatten()
        s["q_out"].view(-1, c["hq"], c["d"])[keep] = q[keep]
        k, v, seq, slot = k[keep], v[keep], seq[keep], slot[keep]
    else:
        s["q_out"].copy_(q)
    if a["k_scale"] is not None:
        k, v = (torch.clamp(x / z[seq][..., None], -448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8) for x, z in ((k, a["k_scale"]), (v, a["v_scale"])))
    else:
        k, v = k.to(torch.bfloat16), v.to(torch.bfloat16)
    if a["table"] is not None:
        page, row = a["table"].long()[seq, slot // c["page"]], slot % c["page"]
    else:
        page, row = seq, slot
    a["k"][page, :, row], a["v"][page, :, row] = k, v
    return _cache_out(s, s["q_out"])


def _plain_attn(s, c):
    """Every sequence padded to the longest: scores, causal mask, softmax, weighted sum."""
    a, rows, group = s["cache"], s["q"].shape[0], c["hq"] // c["hkv"]
    b, n, most = c["batch"], max(s["n"]), max(x + y for x, y in zip(s["n"], s["prefix"]))
    seq, node = _owners(s, rows)
    q = torch.zeros(b, n, c["hq"], c["d"], device=DEV)
    q[seq, node] = s["q"].float()
    at = torch.arange(most, device=DEV)
    used = at[None] < (s["seq_lens"] + s["token_start"][1:] - s["token_start"][:-1]).long()[:, None]
    if a["table"] is not None:
        page = torch.where(used, a["table"].long()[:, at // c["page"]], 0)
        k, v = (x[page, :, (at % c["page"])[None].expand(b, -1)].float() for x in (a["k"], a["v"]))  # [b, slot, head, d]
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    else:
        k, v = a["k"][:, :, :most].float(), a["v"][:, :, :most].float()
    v = torch.where(used[:, None, :, None], v, 0.0)
    q = q.view(b, n, c["hkv"], group, c["d"]).permute(0, 2, 3, 1, 4).reshape(b, c["hkv"], group * n, c["d"])
    z = (q @ k.transpose(2, 3)).view(b, c["hkv"], group, n, most).mul_(1.0 / math.sqrt(c["d"]))
    sees = at[None, None] <= s["seq_lens"].long()[:, None, None] + torch.arange(n, device=DEV)[None, :, None]
    z.masked_fill_(~sees[:, None, None], float("-inf"))
    z.sub_(z.amax(-1, keepdim=True)).exp_()
    z.div_(z.sum(-1, keepdim=True))
    o = (z.view(b, c["hkv"], group * n, most) @ v).view(b, c["hkv"], group, n, c["d"]).permute(0, 3, 1, 2, 4).reshape(b, n, c["hq"], c["d"])
    return o[seq, node].to(torch.bfloat16)


def _plain_logits(s, c):
    b, t, v = c["batch"], c["t_hi"], c["vocab"]
    z = s["logits"].float()
    if c["penalties"]:
        at = torch.arange(c["history"], device=DEV)[None]
        prompt = at < s["prompt_len"][:, None]
        written = (at < s["history_len"][:, None]) & ~prompt
        tokens = s["history"].long()
        in_prompt = torch.zeros(b, v, device=DEV).scatter_add_(1, tokens, prompt.float()) > 0
        count = torch.zeros(b, 1, v, device=DEV)
        count[:, 0].scatter_add_(1, tokens, written.float())
        if t:
            reach = _ancestors(s["tree_parent"], s["tree_sizes"])
            path = torch.zeros(b, t + 1, v, device=DEV)
            path[:, 1:].scatter_add_(2, s["draft_tokens"].long()[:, None].expand(-1, t, -1), reach)
            count = count + path
        rho, phi, pi = (s[k][:, None, None] for k in ("repetition", "frequency", "presence"))
        z = torch.where((count > 0) | in_prompt[:, None], torch.where(z > 0, z / rho, z * rho), z)
        z = z - phi * count - pi * (count > 0)
    if c["bias"]:
        on = torch.arange(s["bias_tokens"].shape[1], device=DEV)[None] < s["bias_len"][:, None]
        z = z + torch.zeros(b, v, device=DEV).scatter_add_(1, s["bias_tokens"].long(), torch.where(on, s["bias_values"], 0.0))[:, None]
    if c["grammar"]:
        at = torch.arange(v, device=DEV)
        z = torch.where((s["allowed"][:, :, at // 32] >> (at % 32)) & 1 != 0, z, float("-inf"))
    live = torch.arange(t + 1, device=DEV)[None] <= s["tree_sizes"][:, None]
    return torch.where(live[:, :, None], z, s["out"])


# ------------------------------------------------------------------------------------------------------------------ work
def work(case):
    c = case
    if c["op"] == "logits":
        rows, v = sum(_tree_sizes(c)) + c["batch"], c["vocab"]
        n = rows * v * ((2 if c["bf16"] else 4) + 4) + (rows * -(-v // 32) * 4 if c["grammar"] else 0)
        return {"bytes": n + (c["batch"] * c["history"] * 2 if c["penalties"] else 0), "flops": rows * v}
    n, prefix = _lengths(c)
    row = c["d"] * 2
    if c["op"] == "rope":
        store = row // 2 if c["fp8"] else row
        return {"bytes": sum(n) * ((c["hq"] + 2 * c["hkv"]) * row + c["hq"] * row + 2 * c["hkv"] * store), "flops": sum(n) * (c["hq"] + c["hkv"]) * c["rotary"] * 3}
    keys = sum(x + y for x, y in zip(n, prefix) if x)
    pairs = sum(x * y + x * (x + 1) // 2 for x, y in zip(n, prefix))
    return {"bytes": keys * c["hkv"] * row * 2 + sum(n) * c["hq"] * row * 2, "flops": 4 * pairs * c["hq"] * c["d"]}


# ------------------------------------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"rope": _exact_rope, "attn": _exact_attn, "logits": _exact_logits}[case["op"]](s, case)


def _depths(parent):
    depth = []
    for p in parent:
        depth.append(1 if p < 0 else depth[p] + 1)
    return depth


def _exact_rope(s, c):
    """Sequence by sequence, as complex numbers: a pair times e^(i angle)."""
    a, paged, fp8 = s["cache"], s["cache"]["table"] is not None, s["cache"]["k_scale"] is not None
    out = _cache_out(s, s["q_out"])
    q_out, k_out, v_out = out["q"].double(), out["k"].double(), out["v"].double()
    for b, (n, first) in enumerate(zip(s["n"], s["prefix"])):
        if not n:
            continue
        if c["form"] == "tree":
            x, depth = s["qkv"][b, :n].double(), torch.tensor(_depths(s["tree_parent"][b, :n].tolist()), device=DEV)
        else:
            start = int(s["token_start"][b])
            x, depth = s["qkv"][start:start + n].double(), torch.arange(1, n + 1, device=DEV)
        turn = torch.polar(torch.full((n, c["rotary"] // 2), float(c["amplitude"]), dtype=torch.float64, device=DEV), (first + depth - 1).double()[:, None] * s["freqs"])
        r, qk = c["rotary"], x[:, : c["hq"] + c["hkv"]].clone()
        if c["interleaved"]:
            w = torch.view_as_complex(qk[..., :r].reshape(n, -1, r // 2, 2).contiguous()) * turn[:, None]
            qk[..., :r] = torch.view_as_real(w).flatten(-2)
        else:
            w = torch.complex(qk[..., : r // 2], qk[..., r // 2:r]) * turn[:, None]
            qk[..., :r] = torch.cat((w.real, w.imag), -1)
        k, v = qk[:, c["hq"]:], x[:, c["hq"] + c["hkv"]:]
        if fp8:
            k, v = k / a["k_scale"][b].double()[:, None], v / a["v_scale"][b].double()[:, None]
            k, v = k.clamp(-448, 448), v.clamp(-448, 448)
        if c["form"] == "tree":
            q_out[b, :n] = qk[:, : c["hq"]]
        else:
            q_out[start:start + n] = qk[:, : c["hq"]]
        slot = torch.arange(first, first + n, device=DEV)
        page, row = (a["table"][b].long()[slot // c["page"]], slot % c["page"]) if paged else (torch.full_like(slot, b), slot)
        k_out[page, :, row], v_out[page, :, row] = k, v
    return {"q": q_out, "k": k_out, "v": v_out}


def _exact_attn(s, c):
    """Head by head, some queries at a time."""
    a, group, out = s["cache"], c["hq"] // c["hkv"], torch.zeros(*s["q"].shape, dtype=torch.float64, device=DEV)
    for b, (n, first) in enumerate(zip(s["n"], s["prefix"])):
        if not n:
            continue
        start, slot = int(s["token_start"][b]), torch.arange(first + n, device=DEV)
        if a["table"] is not None:
            page, row = a["table"][b].long()[slot // c["page"]], slot % c["page"]
        else:
            page, row = torch.full_like(slot, b), slot
        for h in range(c["hkv"]):
            k, v = a["k"][page, h, row].double(), a["v"][page, h, row].double()
            q = s["q"][start:start + n, h * group:(h + 1) * group].double()
            for lo in range(0, n, 1024):
                z = torch.einsum("igd,jd->gij", q[lo:lo + 1024], k) / math.sqrt(c["d"])
                z = z + torch.where(slot[None] > first + torch.arange(lo, min(n, lo + 1024), device=DEV)[:, None], float("-inf"), 0.0)
                out[start + lo:start + min(n, lo + 1024), h * group:(h + 1) * group] = torch.einsum("gij,jd->igd", torch.softmax(z, -1), v)
    return out


def _exact_logits(s, c):
    """Row by row of the trees, token counts by bincount."""
    v, out = c["vocab"], s["out"].double()
    for b, n in enumerate(s["sizes"]):
        z = s["logits"][b, : n + 1].double()
        if c["penalties"]:
            h, p = s["history"][b, : int(s["history_len"][b])].long(), int(s["prompt_len"][b])
            prompt, count = torch.bincount(h[:p], minlength=v) > 0, torch.bincount(h[p:], minlength=v)
            count = count[None].repeat(n + 1, 1)
            parent, tokens = s["tree_parent"][b, :n].tolist(), s["draft_tokens"][b, :n].tolist()
            rows, cols = [], []
            for i in range(n):
                m = i
                while m >= 0:
                    rows.append(i + 1)
                    cols.append(tokens[m])
                    m = parent[m]
            if rows:
                count.index_put_((torch.tensor(rows, device=DEV), torch.tensor(cols, device=DEV)), torch.ones(len(rows), dtype=count.dtype, device=DEV), accumulate=True)
            rho, phi, pi = (s[k][b].double() for k in ("repetition", "frequency", "presence"))
            seen = (count > 0) | prompt
            z = torch.where(seen & (z > 0), z / rho, torch.where(seen, z * rho, z)) - phi * count - pi * (count > 0)
        if c["bias"]:
            m = int(s["bias_len"][b])
            z.index_add_(1, s["bias_tokens"][b, :m].long(), s["bias_values"][b, :m].double()[None].repeat(n + 1, 1))
        if c["grammar"]:
            bits = (s["allowed"][b, : n + 1, :, None] >> torch.arange(32, device=DEV)) & 1
            z[bits.flatten(1)[:, :v] == 0] = float("-inf")
        out[b, : n + 1] = z
    return out
