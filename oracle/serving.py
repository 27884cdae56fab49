"""64-bit definitions of the calls around verification (rotary append, chunk attention, logit adjustment), in plain numpy.

Test infrastructure like the rest of this package: written from the formulas in the header's comments, token by token and
row by row, sharing nothing with the CUDA library.  Tensors come in as torch CPU tensors or numpy arrays."""
from __future__ import annotations

import math

import numpy as np


def _f64(t):
    if t is None:
        return None
    return t.detach().double().numpy() if hasattr(t, "detach") else np.asarray(t, dtype=np.float64)


def _ints(t):
    if t is None:
        return None
    return (t.detach().numpy() if hasattr(t, "detach") else np.asarray(t)).astype(np.int64)


def e4m3(codes):
    """Values of fp8 codes: 1 sign, 4 exponent (bias 7), 3 mantissa bits; 0x7f and 0xff are NaN."""
    c = np.asarray(codes).astype(np.int64)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e == 0, m / 8.0 * 2.0 ** -6, (1 + m / 8.0) * 2.0 ** (e.astype(np.float64) - 7))
    v = np.where((c & 127) == 127, np.nan, v)
    return np.where(c & 128, -v, v)


def rope_frequencies(rotary_dim, base=10000.0, kind="plain", factor=1.0, context=0.0, low=1.0, high=32.0):
    R, out, amplitude = rotary_dim, [], 1.0
    if kind == "ntk":
        base = base * factor ** (R / (R - 2))
    if kind == "yarn":
        place = lambda turns: R * math.log(context / (2 * math.pi * turns)) / (2 * math.log(base))  # noqa: E731
        lo, hi = max(math.floor(place(high)), 0), min(math.ceil(place(low)), R - 1)
        hi = lo + 0.001 if hi <= lo else hi
        amplitude = 0.1 * math.log(factor) + 1.0
    for m in range(R // 2):
        f = base ** (-2.0 * m / R)
        if kind == "linear":
            f = f / factor
        elif kind == "yarn":
            ramp = min(max((m - lo) / (hi - lo), 0.0), 1.0)
            f = f * (1 - ramp) + f / factor * ramp
        elif kind == "banded":
            wave = 2 * math.pi / f
            if wave > context / low:
                f = f / factor
            elif wave >= context / high:
                s = (context / wave - low) / (high - low)
                f = (1 - s) * f / factor + s * f
        out.append(f)
    return np.array(out), amplitude


def depths(parent):
    d = []
    for p in parent:
        d.append(1 if p < 0 else d[p] + 1)
    return d


def rotate(x, position, freqs, interleaved, amplitude):
    """One head-shaped array [..., D] turned by one position."""
    x, half = x.copy(), len(freqs)
    for m, f in enumerate(freqs):
        i, j = (2 * m, 2 * m + 1) if interleaved else (m, m + half)
        c, s = amplitude * math.cos(position * f), amplitude * math.sin(position * f)
        a, b = x[..., i].copy(), x[..., j].copy()
        x[..., i], x[..., j] = a * c - b * s, b * c + a * s
    return x


def place_of(b, slot, block_table, page_size):
    """(first index, row) of a slot in the cache tensor; None when its page entry is unusable."""
    if block_table is None:
        return b, slot
    return int(block_table[b, slot // page_size]), slot % page_size


def rope_append(q, k, v, seq_lens, freqs, *, token_start=None, tree_parent=None, tree_sizes=None, positions=None, interleaved=False,
                amplitude=1.0):
    """(rows of q, [(sequence, slot, key rows [Hkv, D], value rows)]) in fp64, before any rounding.  q rows of tokens that are not
    placed are NaN."""
    q, k, v, lens = _f64(q), _f64(k), _f64(v), _ints(seq_lens)
    out, stored = np.full(q.shape, np.nan), []
    for b, L in enumerate(lens):
        if tree_parent is not None:
            n = q.shape[1] if tree_sizes is None else int(tree_sizes[b])
            place = [((b, i), L + i, L + d - 1) for i, d in enumerate(depths(_ints(tree_parent)[b, :n]))]
        else:
            s, e = int(token_start[b]), int(token_start[b + 1])
            place = [((t,), L + t - s, L + t - s if positions is None else int(positions[t])) for t in range(s, e)]
        for at, slot, pos in place:
            out[at] = rotate(q[at], pos, freqs, interleaved, amplitude)
            stored.append((b, int(slot), rotate(k[at], pos, freqs, interleaved, amplitude), v[at]))
    return out, stored


def chunk_attn(q, k_cache, v_cache, seq_lens, token_start, *, block_table=None, sm_scale=None):
    """(out, spread) fp64 [N, Hq, D]: the attention, and sum_j p_j |v_j|, which roundings of the probabilities scale with.  Rows outside
    every sequence are NaN."""
    q, k, v, lens, starts, table = _f64(q), _f64(k_cache), _f64(v_cache), _ints(seq_lens), _ints(token_start), _ints(block_table)
    N, Hq, D = q.shape
    Hkv, page = k.shape[1], k.shape[2]
    G, scale = Hq // Hkv, 1 / math.sqrt(D) if sm_scale is None else sm_scale
    out, spread = np.full(q.shape, np.nan), np.full(q.shape, np.nan)
    for b, L in enumerate(lens):
        s, e = starts[b], starts[b + 1]
        if e == s:
            continue
        where = [place_of(b, j, table, page) for j in range(L + e - s)]
        first, row = np.array([w[0] for w in where]), np.array([w[1] for w in where])
        for h in range(Hq):
            kk, vv = k[first, h // G, row], v[first, h // G, row]
            for i in range(e - s):
                z = scale * (kk[:L + i + 1] @ q[s + i, h])
                p = np.exp(z - z.max())
                p /= p.sum()
                out[s + i, h] = p @ vv[:L + i + 1]
                spread[s + i, h] = p @ np.abs(vv[:L + i + 1])
    return out, spread


def logits_adjust(logits, draft_tokens=None, tree_parent=None, *, tree_sizes=None, history=None, history_len=None, prompt_len=None,
                  repetition=None, presence=None, frequency=None, bias_tokens=None, bias_values=None, bias_len=None, allowed=None):
    """fp64 [B, T + 1, V]; rows past a tree's size are NaN."""
    z = _f64(logits)
    B, rows, V = z.shape
    out = np.full(z.shape, np.nan)
    of = lambda t, b, default: default if t is None else float(t[b])  # noqa: E731
    for b in range(B):
        n = rows - 1 if tree_sizes is None else int(tree_sizes[b])
        parent = [] if n == 0 else [int(x) for x in tree_parent[b, :n]]
        for r in range(n + 1):
            prompt, count = np.zeros(V, bool), np.zeros(V)
            if history is not None:
                for i in range(int(history_len[b])):
                    t = int(history[b, i])
                    if prompt_len is not None and i < int(prompt_len[b]):
                        prompt[t] = True
                    else:
                        count[t] += 1
            node = r - 1
            while node >= 0:
                count[int(draft_tokens[b, node])] += 1
                node = parent[node]
            row = z[b, r].copy()
            for t in np.nonzero(prompt | (count > 0))[0]:
                rho = of(repetition, b, 1.0)
                row[t] = row[t] / rho if row[t] > 0 else row[t] * rho
                if count[t] > 0:
                    row[t] -= of(frequency, b, 0.0) * count[t] + of(presence, b, 0.0)
            if bias_tokens is not None:
                for i in range(bias_tokens.shape[1] if bias_len is None else int(bias_len[b])):
                    row[int(bias_tokens[b, i])] += float(bias_values[b, i])
            if allowed is not None:
                words = _ints(allowed)[b, r]
                bits = (words[np.arange(V) // 32] >> (np.arange(V) % 32)) & 1
                row[bits == 0] = -np.inf
            out[b, r] = row
    return out


# ---------------------------------------------------------------------------------------- block-scaled caches, windows, sampling
def block_scale(magnitude):
    """The least 2^e, -40 <= e <= 120, with magnitude <= 448 * 2^e."""
    e = -40
    while e < 120 and magnitude > 448.0 * 2.0 ** e:
        e += 1
    return 2.0 ** e


_E4M3 = e4m3(np.arange(127))


def nearest_code(x):
    """Code of the e4m3 number nearest to x (ties to the even code, magnitudes above 448 become 448, NaN becomes 0x7f)."""
    x = np.asarray(x, dtype=np.float64)
    a = np.minimum(np.abs(np.where(np.isnan(x), 0.0, x)), 448.0)
    hi = np.clip(np.searchsorted(_E4M3, a), 1, 126)
    below, above = a - _E4M3[hi - 1], _E4M3[hi] - a
    code = np.where((below < above) | ((below == above) & (hi % 2 == 1)), hi - 1, hi)
    return np.where(np.isnan(x), 127, code + 128 * np.signbit(x)).astype(np.uint8)


def block_append(q, k, v, cache, seq_lens, freqs, block, *, block_table=None, token_start=None, tree_parent=None, tree_sizes=None, positions=None,
                 interleaved=False, amplitude=1.0):
    """(rows of q, expected cache): ``cache`` is (k codes, v codes, k_scale, v_scale) as numpy arrays, copied.  In place of the codes the
    expected cache has fp64 arrays of code values before rounding (x / scale), NaN where nothing is stored, and the codes as they should be
    everywhere else."""
    out, stored = rope_append(q, k, v, seq_lens, freqs, token_start=token_start, tree_parent=tree_parent, tree_sizes=tree_sizes, positions=positions,
                              interleaved=interleaved, amplitude=amplitude)
    table, page = _ints(block_table), cache[0].shape[2]
    res = []
    for which in (0, 1):
        codes, scales = cache[which].copy(), cache[2 + which].astype(np.float64)
        values = np.full(codes.shape, np.nan)
        groups = {}
        for b, slot, key, value in stored:                   # what shares a scale: a tree's tokens, or a block's
            groups.setdefault((b, -1 if tree_parent is not None else slot // block), []).append((slot, (key, value)[which]))
        for (b, _), rows in groups.items():
            L = int(seq_lens[b])
            for h in range(codes.shape[1]):
                mags = np.abs(np.stack([x[h] for _, x in rows]))
                mags = mags[np.isfinite(mags)]
                s = block_scale(mags.max() if mags.size else 0.0)
                first = min(slot for slot, _ in rows) // block
                if L % block and first == L // block:
                    at, row = place_of(b, L, table, page)
                    old = scales[at, h, row // block]
                    if s > old:
                        sl = (at, h, slice(row - L % block, row))
                        codes[sl] = nearest_code(e4m3(codes[sl]) * (old / s))
                    s = max(s, old)
                for slot, x in rows:
                    at, row = place_of(b, slot, table, page)
                    values[at, h, row] = x[h] / s
                    scales[at, h, row // block] = s
        res.append((values, codes, scales))
    return out, res


def window_attn(q, k_cache, v_cache, seq_lens, *, token_start=None, tree_parent=None, tree_sizes=None, block_table=None, k_scale=None, v_scale=None,
                block=0, window=0, sinks=0, sm_scale=None):
    """(out, spread) as ``chunk_attn``, with a window, over bf16 or block-scaled codes; trees: q [B, T, Hq, D], rows past a tree's size NaN."""
    q, lens, table = _f64(q), _ints(seq_lens), _ints(block_table)
    k, v = (e4m3(x.numpy()) if block else _f64(x) for x in (k_cache, v_cache))
    ks, vs = _f64(k_scale), _f64(v_scale)
    Hkv, page, D = k.shape[1], k.shape[2], q.shape[-1]
    Hq = q.shape[-2]
    G, scale = Hq // Hkv, 1 / math.sqrt(D) if sm_scale is None else sm_scale
    out, spread = np.full(q.shape, np.nan), np.full(q.shape, np.nan)
    for b, L in enumerate(lens):
        if tree_parent is not None:
            n = q.shape[1] if tree_sizes is None else int(tree_sizes[b])
            parent = [int(x) for x in tree_parent[b, :n]]
            depth, rows = depths(parent), [(b, i) for i in range(n)]
        else:
            n = int(token_start[b + 1]) - int(token_start[b])
            parent, depth = list(range(-1, n - 1)), list(range(1, n + 1))
            rows = [(int(token_start[b]) + i,) for i in range(n)]
        for i in range(n):
            p = int(L) + depth[i] - 1
            path, m = [], i
            while m >= 0:
                path.append(int(L) + m)
                m = parent[m]
            if tree_parent is None and window:               # a chunk's own tokens can be outside of the window, too
                path = [j for j in path if j > p - window or j < sinks]
            seen = [j for j in range(int(L)) if not window or j > p - window or j < sinks] + path[::-1]
            where = [place_of(b, j, table, page) for j in seen]
            at, row = np.array([w[0] for w in where]), np.array([w[1] for w in where])
            for h in range(Hkv):
                kk, vv = k[at, h, row], v[at, h, row]
                if block:
                    kk, vv = kk * ks[at, h, row // block][:, None], vv * vs[at, h, row // block][:, None]
                for g in range(h * G, (h + 1) * G):
                    z = scale * (kk @ q[rows[i]][g])
                    w = np.exp(z - z.max())
                    w /= w.sum()
                    out[rows[i]][g], spread[rows[i]][g] = w @ vv, w @ np.abs(vv)
    return out, spread


def sample(row, u=None, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, distribution, distance of the draw from the nearest border of its token) of one row of logits in fp64."""
    z = np.array(row, dtype=np.float64)
    z[np.isnan(z)] = -np.inf
    V, top = len(z), z.max()
    if top == -np.inf:
        return -1, np.zeros(V), 1.0
    with np.errstate(invalid="ignore", over="ignore"):
        w = np.exp((z - top) / temperature) if temperature > 0 else np.zeros(V)
    w[z == top] = 1.0
    w[z == -np.inf] = 0.0
    w[np.isnan(w)] = 0.0                                     # a finite value beside infinite ones
    order = sorted(range(V), key=lambda i: (-z[i], i))
    if not temperature > 0:
        order = order[:1]
    if 0 < top_k < V:
        order = order[:top_k]
    if top_p < 1:
        total, run, kept = math.fsum(w[i] for i in order), 0.0, []
        for i in order:
            if kept and not run < top_p * total:
                break
            kept.append(i)
            run += w[i]
        order = kept
    if min_p > 0:
        order = [i for i in order if w[i] >= min(min_p, 1.0)]
    p = np.zeros(V)
    p[order] = w[order]
    p /= math.fsum(p)
    if u is None:
        return None, p, 1.0
    c = np.cumsum(p)
    t = min(int(np.searchsorted(c, u * c[-1], side="right")), int(np.nonzero(p)[0][-1]))
    return t, p, float(min(abs(c - u * c[-1])))
