"""What is measured of a cache held in 8 bits with a scale for each block of slots and head, of attention with a sliding window and a few
first slots that stay visible, and of the draws at the end of a step: new keys and values into the blocks (rotated on the way), attention
of chunks, single tokens and draft trees over such a cache or a bf16 one, and sampling with temperature, top-k, top-p and min-p.

A case is a dict of plain values; `prepare` makes its inputs from a seed, `run` is one pass through the operator (the plain form in
elementary torch operations, or with `own` the library's call), `exact` the same from the definitions in 64 bits, and `work` what a
pass cannot do without.  Ragged lengths follow from the case alone (its number "mix"), everything else from the seed."""
import math
import random

import torch

own = False
DEV = "cuda"


# ------------------------------------------------------------------------------------------------------------------ cases
def _append(name, form, heads, batch, n_lo, n_hi, l_lo, l_hi, page, block, rotary=128, interleaved=False, amplitude=1.0, mix=1):
    return {"name": name, "op": "append", "form": form, "hq": heads[0], "hkv": heads[1], "d": 128, "batch": batch, "n_lo": n_lo, "n_hi": n_hi,
            "l_lo": l_lo, "l_hi": l_hi, "page": page, "block": block, "chunks": batch, "rotary": rotary, "interleaved": interleaved,
            "amplitude": amplitude, "mix": mix}


def _attn(name, form, heads, d, batch, chunks, n_lo, n_hi, l_lo, l_hi, page, block=0, window=0, sinks=0, mix=1):
    return {"name": name, "op": "attn", "form": form, "hq": heads[0], "hkv": heads[1], "d": d, "batch": batch, "chunks": chunks, "n_lo": n_lo,
            "n_hi": n_hi, "l_lo": l_lo, "l_hi": l_hi, "page": page, "block": block, "window": window, "sinks": sinks, "mix": mix}


def _sample(name, batch, r_lo, r_hi, vocab, bf16, tokens, probs, top_k, top_p, min_p, mix=1):
    return {"name": name, "op": "sample", "batch": batch, "r_lo": r_lo, "r_hi": r_hi, "vocab": vocab, "bf16": bf16, "tokens": tokens,
            "probs": probs, "top_k": top_k, "top_p": top_p, "min_p": min_p, "mix": mix}


def listed():
    return [
        # one sequence's next token in the middle of a block, 32 heads without groups: a call's latency
        _append("append_one_token", "chunk", (32, 32), 1, 1, 1, 2083, 2083, 64, 64),
        # the draft trees of a serving batch (16 to 64 nodes behind prefixes of 512 to 8192)
        _append("append_trees", "tree", (32, 8), 64, 16, 64, 512, 8192, 64, 32),
        # a long prompt's chunk far into the context (scaled frequencies change the amplitude too), half of each head rotated
        _append("append_prompt_far", "chunk", (64, 8), 1, 8192, 8192, 98304, 98304, 64, 64, rotary=64, interleaved=True, amplitude=1.2079),
        # every sequence's next token, each with its last 4096 slots and four first ones
        _attn("window_decode", "chunk", (32, 8), 128, 64, 64, 1, 1, 512, 16384, 64, window=4096, sinks=4),
        # chunks of two prompts far behind the window's length: the tensor cores' case
        _attn("window_prompt", "chunk", (32, 8), 128, 2, 2, 2048, 2048, 16384, 16384, 64, window=4096, sinks=4),
        # short ragged prompts with small heads, an odd window
        _attn("window_ragged_d64", "chunk", (16, 4), 64, 9, 9, 0, 701, 0, 900, 16, window=250, sinks=1),
        # every sequence's next token over 8-bit keys and values: what serving does most
        _attn("block_decode", "chunk", (32, 8), 128, 64, 64, 1, 1, 512, 8192, 64, block=64),
        # one token over one long context: only a split of the context fills the machine
        _attn("block_one_long", "chunk", (64, 8), 128, 1, 1, 1, 1, 65536, 65536, 64, block=32),
        # verification of a serving batch's draft trees over 8-bit keys and values
        _attn("block_trees", "tree", (32, 8), 128, 64, 64, 16, 64, 512, 8192, 64, block=32),
        # chunks of two prompts over long prefixes in 8 bits
        _attn("block_prompt", "chunk", (32, 8), 128, 2, 2, 2048, 2048, 16384, 16384, 64, block=64),
        # plain decoding: one row a sequence, as the output layer leaves it, a large odd vocabulary, all filters
        _sample("sample_rows_bf16", 64, 1, 1, 129537, True, True, False, True, True, True),
        # the target's rows of draft trees as the distributions that acceptance reads
        _sample("sample_trees", 16, 17, 65, 32000, False, False, True, False, True, False),
    ]


HEADS = ((8, 8), (16, 4), (32, 8), (32, 32), (64, 8), (12, 3), (10, 2), (7, 1), (16, 1))


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op, mix, heads = rng.choice(("append", "window", "block", "block", "sample")), rng.randrange(1 << 20), rng.choice(HEADS)
    block = rng.choice((16, 32, 64, 128))
    page = rng.choice((0, 0, block, block, 2 * block, 256))
    if op == "append":
        rotary = rng.choice((128, 128, 16 * rng.randint(1, 8)))
        more = dict(rotary=rotary, interleaved=rng.random() < 0.5, amplitude=rng.choice((1.0, 1.0, 1.1386)), mix=mix)
        if rng.random() < 0.4:
            n, b, far = rng.randint(1, 64), _log(rng, 1, 64), _log(rng, 1, 8192)
            c = _append("", "tree", heads, b, rng.randint(1, n), n, rng.randint(0, far), far, page, block, **more)
        else:
            n, b = _log(rng, 1, 4096), _log(rng, 1, 32)
            n = min(n, max(1, 8192 // b))
            far = _log(rng, 1, max(2, 65536 // b))
            c = _append("", "chunk", heads, b, rng.randint(0, n), n, rng.randint(0, far), far, page, block, **more)
    elif op == "sample":
        vocab, probs = _log(rng, 1000, 150000), rng.random() < 0.5
        rows = rng.choice((1, rng.randint(1, 65)))
        b = max(1, min(_log(rng, 1, 64), int(3.0e7 / (vocab * rows))))
        c = _sample("", b, rng.randint(1, rows), rows, vocab, rng.random() < 0.5, not probs or rng.random() < 0.5, probs, rng.random() < 0.5,
                    rng.random() < 0.7, rng.random() < 0.4, mix=mix)
    else:
        d = 128 if op == "block" else rng.choice((64, 128, 128))
        window = _log(rng, 64, 8192) if op == "window" or rng.random() < 0.3 else 0
        more = dict(block=block if op == "block" else 0, window=window, sinks=rng.choice((0, 1, 4, rng.randint(0, 300))) if window else 0, mix=mix)
        tree = rng.random() < 0.3
        b, n, far = _log(rng, 1, 64), rng.randint(1, 64) if tree else _log(rng, 1, 4096), _log(rng, 1, 65536)
        chunks = b if tree else rng.choice((b, 1 + rng.randrange(b)))
        # what the plain form holds at once, and the operations, stay below those of the largest listed case
        while b * heads[0] * n * (n + far) > 2.0e9 or b * heads[1] * (n + far) * d > 5.0e8:
            n, far = max(1, n * 2 // 3), max(1, far * 4 // 5)
        c = _attn("", "tree" if tree else "chunk", heads, d, b, chunks, rng.randint(0, n), n, rng.randint(0, far), far, page, **more)
    del c["name"]
    return c


def _lengths(c):
    """(new tokens, prefix) of every sequence; a tree has n_hi nodes at the most."""
    r = random.Random(c["mix"])
    n = [c["n_hi"]] + [r.randint(c["n_lo"], c["n_hi"]) for _ in range(c["batch"] - 1)]
    n = [v if i < c["chunks"] else 1 for i, v in enumerate(n)]
    return n, [r.randint(c["l_lo"], c["l_hi"]) for _ in range(c["batch"])]


def _row_counts(c):
    r = random.Random(c["mix"])
    return [c["r_hi"]] + [r.randint(c["r_lo"], c["r_hi"]) for _ in range(c["batch"] - 1)]


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
    """The cache (random throughout: what earlier sequences left behind is there too), its block table and its blocks' scales."""
    kv, d, batch, page, block = c["hkv"], c["d"], c["batch"], c["page"], c["block"]
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
        most = max(max(need), 1) + 5
        shape, table = (batch, kv, -(-most // block) * block if block else most, d), None
    if block:
        k, v = (torch.randint(0, 120, shape, dtype=torch.uint8, device=DEV, generator=g) +
                128 * torch.randint(0, 2, shape, dtype=torch.uint8, device=DEV, generator=g) for _ in range(2))
        blocks = (*shape[:2], shape[2] // block)
        if c["op"] == "append":   # as an append leaves them: powers of two
            scales = [torch.exp2(torch.randint(-9, -6, blocks, device=DEV, generator=g).float()) for _ in range(2)]
        else:
            scales = [torch.rand(blocks, device=DEV, generator=g) * 0.01 + 0.005 for _ in range(2)]
    else:
        k, v = (torch.randn(shape, dtype=torch.bfloat16, device=DEV, generator=g) for _ in range(2))
        scales = [None, None]
    return {"k": k, "v": v, "table": table, "k_scale": scales[0], "v_scale": scales[1], "block": block}


def prepare(case, seed):
    c, g, r = case, torch.Generator(device=DEV).manual_seed(seed), random.Random(seed)
    if c["op"] == "sample":
        return _prepare_sample(c, g)
    n, prefix = lengths = _lengths(c)
    s = {"c": c, "cache": _cache(c, lengths, g, r), "seq_lens": _ints(prefix), "n": n, "prefix": prefix}
    tree = c["form"] == "tree"
    lead = (c["batch"], c["n_hi"]) if tree else (sum(n),)
    if tree:
        s["parents"] = [_parents(r, v) for v in n]
        s["tree_sizes"] = _ints(n)
        s["tree_parent"] = _ints([p + [0] * (c["n_hi"] - v) for p, v in zip(s["parents"], n)])
    else:
        starts = [0]
        for v in n:
            starts.append(starts[-1] + v)
        s["token_start"] = _ints(starts)
    if c["op"] == "append":
        # queries, keys and values as one projection leaves them: side by side in a row
        heads = c["hq"] + 2 * c["hkv"]
        s["qkv"] = torch.randn(*lead, heads, c["d"], dtype=torch.bfloat16, device=DEV, generator=g)
        i = torch.arange(c["rotary"] // 2, dtype=torch.float64, device=DEV)
        s["freqs"] = torch.pow(torch.tensor(10000.0, dtype=torch.float64, device=DEV), -2.0 * i / c["rotary"])
        s["q_out"] = torch.zeros(*lead, c["hq"], c["d"], dtype=torch.bfloat16, device=DEV)
    else:
        s["q"] = torch.randn(*lead, c["hq"], c["d"], dtype=torch.bfloat16, device=DEV, generator=g)
    return s


def _prepare_sample(c, g):
    b, rows, v = c["batch"], c["r_hi"], c["vocab"]
    counts = _row_counts(c)
    s = {"c": c, "counts": counts, "num_rows": _ints(counts)}
    z = torch.randn(b, rows, v, device=DEV, generator=g) * 3.0
    s["logits"] = z.to(torch.bfloat16) if c["bf16"] else z
    rand = lambda: torch.rand(b, device=DEV, generator=g)  # noqa: E731
    # one sequence in eight is greedy
    s["temperature"] = torch.where(rand() < 0.125, 0.0, 0.5 + rand())
    if c["top_k"]:
        s["top_k"] = torch.exp(rand() * math.log(v) * 0.8).to(torch.int32)
    if c["top_p"]:
        s["top_p"] = 0.8 + 0.199 * rand()
    if c["min_p"]:
        s["min_p"] = 0.1 * rand()
    if c["tokens"]:
        s["uniforms"] = torch.rand(b, rows, device=DEV, generator=g)
        s["token_out"] = torch.full((b, rows), -7, dtype=torch.int32, device=DEV)
    if c["probs"]:
        s["prob_out"] = torch.zeros(b, rows, v, device=DEV)
    return s


# ------------------------------------------------------------------------------------------------------------------ one pass
def run(state):
    s, c = state, state["c"]
    if c["op"] == "append":
        return _own_append(s, c) if own else _plain_append(s, c)
    if c["op"] == "attn":
        return _own_attn(s, c) if own else _plain_attn(s, c)
    return _own_sample(s) if own else _plain_sample(s, c)


def _own_store(s):
    from paper_2401_15077_b200 import binding as E
    a = s["cache"]
    return E, E.KVStore(a["k"], a["v"], block_table=a["table"], k_scale=a["k_scale"], v_scale=a["v_scale"], block_size=a["block"])


def _own_append(s, c):
    E, store = _own_store(s)
    q, k, v = s["qkv"].split((c["hq"], c["hkv"], c["hkv"]), dim=-2)
    more = {"interleaved": c["interleaved"], "amplitude": c["amplitude"]}
    if c["form"] == "tree":
        E.eagle_tree_block_append(q, k, v, store, s["seq_lens"], s["tree_parent"], s["freqs"], s["q_out"], tree_sizes=s["tree_sizes"], **more)
    else:
        E.eagle_block_append(q, k, v, store, s["seq_lens"], s["token_start"], s["freqs"], s["q_out"], **more)
    return _append_out(s)


def _own_attn(s, c):
    E, store = _own_store(s)
    more = {"window": c["window"], "sinks": c["sinks"]}
    if c["form"] == "tree":
        return E.eagle_tree_window_attn(s["q"], store, s["seq_lens"], s["tree_parent"], tree_sizes=s["tree_sizes"], **more)
    return E.eagle_window_attn(s["q"], store, s["seq_lens"], s["token_start"], **more)


def _own_sample(s):
    from paper_2401_15077_b200 import binding as E
    E.eagle_sample(s["logits"], s.get("uniforms"), s.get("token_out"), s.get("prob_out"), num_rows=s["num_rows"],
                   **{n: s[n] for n in ("temperature", "top_k", "top_p", "min_p") if n in s})
    return _sample_out(s)


def _append_out(s):
    a = s["cache"]
    return {"q": s["q_out"], "k": a["k"].view(torch.float8_e4m3fn), "v": a["v"].view(torch.float8_e4m3fn), "k_scale": a["k_scale"],
            "v_scale": a["v_scale"]}


def _sample_out(s):
    return {n: s[n] for n in ("token_out", "prob_out") if n in s}


# ------------------------------------------------------------------------------------------------------------ plain forms
def _places(s, c):
    """Of every live row: its sequence, its place among the sequence's new tokens and its depth below the prefix (a chunk's tokens: the
    place), and for trees which of its sequence's nodes each row sees."""
    if c["form"] != "tree":
        at = torch.arange(sum(s["n"]), device=DEV)
        seq = torch.searchsorted(s["token_start"].long(), at, right=True) - 1
        place = at - s["token_start"].long()[seq]
        return seq, place, place, at, None
    b, t = s["tree_parent"].shape
    node = torch.arange(t, device=DEV)
    live = (node[None] < s["tree_sizes"][:, None]).float()
    up = (s["tree_parent"].long()[:, :, None] == node[None, None]).float() * live[:, :, None]
    reach = torch.eye(t, device=DEV)[None] * live[:, :, None] + up
    for _ in range(6):  # paths of up to 64 nodes
        reach = (reach @ reach).clamp_(max=1.0)
    keep = live.flatten().nonzero().flatten()
    seq, place = keep // t, keep % t
    return seq, place, reach.sum(2).long().flatten()[keep] - 1, keep, reach > 0


def _addresses(s, c, seq, slot):
    a = s["cache"]
    if a["table"] is None:
        return seq, slot
    return a["table"].long()[seq, slot // c["page"]], slot % c["page"]


def _codes(x):
    return torch.clamp(x, -448.0, 448.0).to(torch.float8_e4m3fn)


def _plain_append(s, c):
    a, half, block = s["cache"], c["rotary"] // 2, c["block"]
    seq, place, depth, row, _ = _places(s, c)
    first = s["seq_lens"].long()[seq]
    angle = (first + depth).double()[:, None] * s["freqs"][None]
    cos, sin = (f(angle).float()[:, None] * c["amplitude"] for f in (torch.cos, torch.sin))
    q, k, v = s["qkv"].flatten(0, -3)[row].float().split((c["hq"], c["hkv"], c["hkv"]), dim=-2)
    i, j = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if c["interleaved"] else (slice(0, half), slice(half, 2 * half))

    def turned(x):
        y = x.clone()
        y[..., i], y[..., j] = x[..., i] * cos - x[..., j] * sin, x[..., j] * cos + x[..., i] * sin
        return y

    s["q_out"].flatten(0, -3)[row] = turned(q).to(torch.bfloat16)
    page, at = _addresses(s, c, seq, first + place)
    per = a["k_scale"].shape[2]
    number = page * per + at // block                       # the block of every new token
    # blocks that hold older tokens, too: the first of each sequence that does not begin with it
    lens = s["seq_lens"].long()
    part = ((lens % block != 0) & (_ints(s["n"]) > 0)).nonzero().flatten()
    part_page, part_at = _addresses(s, c, part, lens[part])
    part_number = part_page * per + part_at // block
    for codes, scales, x in ((a["k"], a["k_scale"], turned(k)), (a["v"], a["v_scale"], v)):
        flat = scales.transpose(1, 2).reshape(-1, c["hkv"])  # [page and block, head]
        group = seq if c["form"] == "tree" else number       # what shares a scale: a tree's tokens, or a block's
        top = torch.zeros(max(flat.shape[0], c["batch"]), c["hkv"], device=DEV)
        top.scatter_reduce_(0, group[:, None].expand(-1, c["hkv"]), x.abs().amax(-1), "amax")
        mantissa, exponent = torch.frexp(top)
        need = torch.exp2((exponent - 9 + (mantissa > 0.875)).clamp(-40, 120).float())
        need = torch.where(top > 0, need, 2.0 ** -40)
        old = flat[part_number]
        wanted = need[part if c["form"] == "tree" else part_number]
        grown = torch.maximum(old, wanted)
        need[part if c["form"] == "tree" else part_number] = grown
        new = flat.clone()
        new[number] = need[group]
        # older codes of a block whose scale has grown
        slot = (part_at // block * block)[:, None] + torch.arange(block, device=DEV)
        view = codes.view(torch.float8_e4m3fn).float()[part_page[:, None], :, slot]         # [part, slot, head, d]
        again = _codes(view * (old / grown)[:, None, :, None]).view(torch.uint8)
        older = (slot < part_at[:, None])[:, :, None, None] & (grown > old)[:, None, :, None]
        codes[part_page[:, None], :, slot] = torch.where(older, again, codes[part_page[:, None], :, slot])
        codes[page, :, at] = _codes(x / new[number][:, :, None]).view(torch.uint8)
        scales.copy_(new.view(scales.shape[0], per, c["hkv"]).transpose(1, 2))
    return _append_out(s)


def _plain_attn(s, c):
    """Every sequence padded to the longest: scores, mask, softmax, weighted sum."""
    a, group, b, block = s["cache"], c["hq"] // c["hkv"], c["batch"], c["block"]
    n, most = max(max(s["n"]), 1), max(x + y for x, y in zip(s["n"], s["prefix"]))
    seq, place, depth, row, reach = _places(s, c)
    out = torch.zeros_like(s["q"])
    q = torch.zeros(b, n, c["hq"], c["d"], device=DEV)
    q[seq, place] = s["q"].flatten(0, -3)[row].float()
    at, lens = torch.arange(most, device=DEV), s["seq_lens"].long()
    used = at[None] < (lens + _ints(s["n"]))[:, None]
    if a["table"] is not None:
        page = torch.where(used, a["table"].long()[:, at // c["page"]], 0)
        slot = (at % c["page"])[None].expand(b, -1)
    else:
        page, slot = torch.arange(b, device=DEV)[:, None].expand(-1, most), at[None].expand(b, -1)

    def load(codes, scales):
        if not block:
            return codes[page, :, slot].float().transpose(1, 2)              # [b, head, slot, d]
        x = codes.view(torch.float8_e4m3fn)[page, :, slot].float() * scales[page, :, slot // block][..., None]
        return x.transpose(1, 2)

    k, v = load(a["k"], a["k_scale"]), load(a["v"], a["v_scale"])
    v = torch.where(used[:, None, :, None], v, 0.0)
    q = q.view(b, n, c["hkv"], group, c["d"]).permute(0, 2, 3, 1, 4).reshape(b, c["hkv"], group * n, c["d"])
    z = (q @ k.transpose(2, 3)).view(b, c["hkv"], group, n, most).mul_(1.0 / math.sqrt(c["d"]))
    # position of every row, and what it sees: the prefix and its path (or the tokens before it), within the window or among the first
    where = lens[:, None] + torch.arange(n, device=DEV)[None]
    if reach is None:
        sees = at[None, None] <= where[:, :, None]
    else:
        where[seq, place] = lens[seq] + depth
        own_part = (at[None] - lens[:, None]).clamp(0, n - 1)
        sees = torch.where((at[None] < lens[:, None])[:, None], True, reach.gather(2, own_part[:, None].expand(-1, n, -1)) & used[:, None])
    if c["window"]:
        near = at[None, None] > (where - c["window"])[:, :, None]
        if reach is not None:
            near = near | (at[None] >= lens[:, None])[:, None]               # (no path is as long as a window)
        sees = sees & (near | (at < c["sinks"]))
    z.masked_fill_(~sees[:, None, None], float("-inf"))
    z.sub_(z.amax(-1, keepdim=True)).exp_()
    z.div_(z.sum(-1, keepdim=True))
    o = (z.view(b, c["hkv"], group * n, most) @ v).view(b, c["hkv"], group, n, c["d"]).permute(0, 3, 1, 2, 4).reshape(b, n, c["hq"], c["d"])
    out.flatten(0, -3)[row] = o[seq, place].to(torch.bfloat16)
    return out


def _plain_sample(s, c):
    """Rows sorted in descending order (equal ones by their index), prefix sums over it, a prefix sum in ascending order for the draw."""
    b, rows, v = c["batch"], c["r_hi"], c["vocab"]
    live = (torch.arange(rows, device=DEV)[None] < s["num_rows"][:, None]).flatten()
    per = lambda name, off: (s[name][:, None].expand(b, rows).flatten()[live][:, None] if name in s else off)  # noqa: E731
    z, order = torch.sort(s["logits"].view(b * rows, v)[live].float(), dim=1, descending=True, stable=True)
    t = per("temperature", None).double()
    greedy = t == 0
    w = ((z.double() - z[:, :1].double()) / torch.where(greedy, 1.0, t)).exp_()
    rank = torch.arange(v, device=DEV)[None]
    keep = (rank == 0) | ~greedy
    if "top_k" in s:
        top_k = per("top_k", None)
        keep &= (rank < top_k) | (top_k <= 0)
    if "top_p" in s:
        kept = torch.where(keep, w, 0.0)
        before = kept.cumsum(1) - kept
        keep &= (before < per("top_p", None).double() * kept.sum(1, keepdim=True)) | (rank == 0)
    if "min_p" in s:
        keep &= w >= per("min_p", None).double()
    w = torch.where(keep, w, 0.0)
    w = torch.zeros_like(w).scatter_(1, order, w)
    if "prob_out" in s:
        s["prob_out"].view(b * rows, v)[live] = (w / w.sum(1, keepdim=True)).float()
    if "token_out" in s:
        mass = w.cumsum(1)
        u = s["uniforms"].flatten()[live].double()[:, None]
        s["token_out"].view(-1)[live] = torch.searchsorted(mass, u * mass[:, -1:], right=True).flatten().clamp_(max=v - 1).to(torch.int32)
    return _sample_out(s)


# ---------------------------------------------------------------------------------------------------------------- floors
def work(case):
    c = case
    if c["op"] == "sample":
        rows, v = sum(_row_counts(c)), c["vocab"]
        return {"bytes": rows * (v * ((2 if c["bf16"] else 4) + (4 if c["probs"] else 0)) + 8), "flops": rows * v * 4}
    n, prefix = _lengths(c)
    d, hq, hkv = c["d"], c["hq"], c["hkv"]
    if c["op"] == "append":
        return {"bytes": sum(n) * d * (hq * 4 + hkv * 2 * 3) + sum(-(-v // c["block"]) for v in n) * hkv * 8,
                "flops": sum(n) * (hq + hkv) * c["rotary"] * 3}
    slots = pairs = 0
    for i, (m, first) in enumerate(zip(n, prefix)):
        if not m:
            continue
        w = c["window"] or first + m
        lo = max(0, first + 1 - w)
        slots += first + m - lo + min(c["sinks"], lo)
        if c["form"] == "tree":
            pairs += m * (first - lo + min(c["sinks"], lo)) + m * 3
        else:
            for p in range(first, first + m):
                near = max(0, p + 1 - w)
                pairs += p + 1 - near + min(c["sinks"], near)
    size = 1 + 4 / c["block"] / d if c["block"] else 2
    return {"bytes": int(sum(n) * hq * d * 4 + slots * hkv * d * 2 * size), "flops": 4 * pairs * hq * d}


# ------------------------------------------------------------------------------------------------- definitions in 64 bits
def exact(case, seed):
    c = case
    if c["op"] == "attn":
        n, prefix = _lengths(c)
        if 4 * c["hq"] * c["d"] * sum(a * (a + b) for a, b in zip(n, prefix)) > 1.2e13:
            return None
    s = prepare(case, seed)
    return {"append": _exact_append, "attn": _exact_attn, "sample": _exact_sample}[c["op"]](s, c)


def _depths(s, c, b):
    if c["form"] != "tree":
        return list(range(s["n"][b]))
    depth = []
    for p in s["parents"][b]:
        depth.append(0 if p < 0 else depth[p] + 1)
    return depth


def _e4m3(codes):
    x = codes.long()
    e, m = (x >> 3) & 15, (x & 7).double()
    y = torch.where(e == 0, m * 2.0 ** -9, (1.0 + m / 8.0) * torch.exp2((e - 7).double()))
    return torch.where(x >= 128, -y, y)


def _exact_append(s, c):
    """Sequence by sequence, block by block.  Codes are e4m3, so the nearest one is looked up among all of them."""
    a, block, half = s["cache"], c["block"], c["rotary"] // 2
    values = _e4m3(torch.arange(127, device=DEV))
    middles, even = (values[1:] + values[:-1]) / 2, torch.arange(126, device=DEV) % 2 == 0
    q_out = s["q_out"].double()

    def nearest(x):
        i = torch.searchsorted(middles, x.abs().contiguous())             # (a middle counts as below: the lower code)
        tie = middles[i.clamp(max=125)] == x.abs()
        i = torch.where(tie & ~even[i.clamp(max=125)], i + 1, i)
        return i.to(torch.uint8) + 128 * torch.signbit(x).to(torch.uint8)

    def power(top):
        e = -40
        while top > 448.0 * 2.0 ** e and e < 120:
            e += 1
        return 2.0 ** e

    for b, (n, first) in enumerate(zip(s["n"], s["prefix"])):
        if not n:
            continue
        rows = s["qkv"][b, :n] if c["form"] == "tree" else s["qkv"][int(s["token_start"][b]):int(s["token_start"][b + 1])]
        x = rows.double()
        angle = (torch.tensor(_depths(s, c, b), device=DEV, dtype=torch.float64) + first)[:, None, None] * s["freqs"]
        cos, sin = c["amplitude"] * torch.cos(angle), c["amplitude"] * torch.sin(angle)
        turning = x[:, :c["hq"] + c["hkv"], :2 * half]
        if c["interleaved"]:
            even_part, odd_part = turning.unflatten(-1, (half, 2)).unbind(-1)
            turned = torch.stack((even_part * cos - odd_part * sin, odd_part * cos + even_part * sin), -1).flatten(-2)
        else:
            lo, hi = turning[..., :half], turning[..., half:]
            turned = torch.cat((lo * cos - hi * sin, hi * cos + lo * sin), -1)
        x[:, :c["hq"] + c["hkv"], :2 * half] = turned
        target = q_out[b, :n] if c["form"] == "tree" else q_out[int(s["token_start"][b]):int(s["token_start"][b + 1])]
        target.copy_(x[:, :c["hq"]])
        for codes, scales, new in ((a["k"], a["k_scale"], x[:, c["hq"]:c["hq"] + c["hkv"]]), (a["v"], a["v_scale"], x[:, c["hq"] + c["hkv"]:])):
            tree_top = new.abs().amax((0, 2)).tolist()
            for lo in range(first // block * block, first + n, block):
                page, at = (int(a["table"][b, lo // c["page"]]), lo % c["page"]) if a["table"] is not None else (b, lo)
                i, j = max(lo, first) - first, min(lo + block, first + n) - first
                tops = tree_top if c["form"] == "tree" else new[i:j].abs().amax((0, 2)).tolist()
                part = first - first // block * block
                start_page, start_at = (int(a["table"][b, first // c["page"]]), first % c["page"]) if a["table"] is not None and part else (b, first)
                if lo == first // block * block:
                    before = scales[start_page, :, start_at // block].tolist() if part else [0.0] * c["hkv"]
                held = before if (lo < first or c["form"] == "tree") else [0.0] * c["hkv"]
                grown = [max(o, power(t)) for o, t in zip(held, tops)]
                if lo < first:
                    for h in range(c["hkv"]):
                        if grown[h] > before[h]:
                            codes[page, h, at:at + part] = nearest(_e4m3(codes[page, h, at:at + part]) * (before[h] / grown[h]))
                scale = torch.tensor(grown, dtype=torch.float64, device=DEV)
                scales[page, :, at // block] = scale.float()
                codes[page, :, at + i + first - lo:at + j + first - lo] = nearest(new[i:j] / scale[None, :, None]).transpose(0, 1)
    return {"q": q_out, "k": _e4m3(a["k"]), "v": _e4m3(a["v"]), "k_scale": a["k_scale"].double(), "v_scale": a["v_scale"].double()}


def _exact_attn(s, c):
    """Head by head, some queries at a time."""
    a, group, block = s["cache"], c["hq"] // c["hkv"], c["block"]
    out = torch.zeros(*s["q"].shape, dtype=torch.float64, device=DEV)
    for b, (n, first) in enumerate(zip(s["n"], s["prefix"])):
        if not n:
            continue
        slot = torch.arange(first + n, device=DEV)
        if a["table"] is not None:
            page, row = a["table"][b].long()[slot // c["page"]], slot % c["page"]
        else:
            page, row = torch.full_like(slot, b), slot
        depth = torch.tensor(_depths(s, c, b), device=DEV)
        hidden = torch.zeros(n, first + n, dtype=torch.bool, device=DEV)
        if c["form"] == "tree":
            path = torch.zeros(n, n, dtype=torch.bool)
            for i, p in enumerate(s["parents"][b]):
                if p >= 0:
                    path[i] = path[p]
                path[i, i] = True
            hidden[:, first:] = ~path.to(DEV)
            place = torch.cat((torch.arange(first, device=DEV), first + depth))
        else:
            hidden[:] = slot[None] > (first + depth)[:, None]
            place = slot
        if c["window"]:
            hidden |= (place[None] <= (first + depth - c["window"])[:, None]) & (place >= c["sinks"])[None]
        start = 0 if c["form"] == "tree" else int(s["token_start"][b])
        q_rows, o_rows = (s["q"][b], out[b]) if c["form"] == "tree" else (s["q"][start:start + n], out[start:start + n])
        for h in range(c["hkv"]):
            if block:
                k, v = (_e4m3(x[page, h, row]) * y[page, h, row // block].double()[:, None] for x, y in ((a["k"], a["k_scale"]), (a["v"], a["v_scale"])))
            else:
                k, v = a["k"][page, h, row].double(), a["v"][page, h, row].double()
            q = q_rows[:n, h * group:(h + 1) * group].double()
            for lo in range(0, n, 1024):
                z = torch.einsum("igd,jd->gij", q[lo:lo + 1024], k) / math.sqrt(c["d"])
                z = z.masked_fill(hidden[lo:lo + 1024], float("-inf"))
                o_rows[lo:min(n, lo + 1024), h * group:(h + 1) * group] = torch.einsum("gij,jd->igd", torch.softmax(z, -1), v)
    return out


def _exact_sample(s, c):
    """Row by row: what is kept is found from the values in ascending order of -z, then drawn in ascending order of the index."""
    v, res = c["vocab"], _sample_out(s)
    for name in res:
        if name == "prob_out":
            res[name] = res[name].double()
    for b, rows in enumerate(s["counts"]):
        t = float(s["temperature"][b])
        k = int(s["top_k"][b]) if "top_k" in s and int(s["top_k"][b]) > 0 else v
        top_p = float(s["top_p"][b]) if "top_p" in s else 1.0
        min_p = float(s["min_p"][b]) if "min_p" in s else 0.0
        for r in range(rows):
            z = s["logits"][b, r].double()
            if t == 0.0:
                p = torch.zeros(v, dtype=torch.float64, device=DEV)
                p[(z == z.max()).nonzero()[0]] = 1.0
            else:
                p = torch.softmax(z / t, 0)
                order = torch.argsort(-z, stable=True)[:k]
                ahead = p[order].cumsum(0) / p[order].sum()
                if "top_p" in s:
                    order = order[:1 + int((ahead[:-1] < top_p).sum())]
                order = order[p[order] >= min_p * p[order[0]]]
                kept = torch.zeros_like(p)
                kept[order] = p[order] / p[order].sum()
                p = kept
            if "prob_out" in res:
                res["prob_out"][b, r] = p
            if "token_out" in res:
                res["token_out"][b, r] = int(torch.searchsorted(p.cumsum(0), float(s["uniforms"][b, r]) * p.sum(), right=True).clamp(max=v - 1))
    return res
