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
