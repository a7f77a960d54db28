"""Plain references of the serving calls around the paged dINT4 cache: what a row sees, attention over it in binary64,
a step's plan, the rotation."""
import numpy as np
import torch

from kv_util import decode_pages


def seen_with_sinks(n, c, i, causal, window, sinks):
    """Positions that row i of c rows of a sequence of n tokens sees."""
    p = n - c + i
    if p < 0:
        return []
    return [j for j in range(p + 1 if causal else n) if not window or j > p - window or j < sinks]


def seen_in_tree(n, c, i, mask, window, sinks):
    """The same for a drafted row with `mask`, an integer of bits."""
    base = n - c
    if base + i < 0:
        return []
    mask &= (1 << c) - 1
    p = base + bin(mask).count("1") - 1
    first = max(0, base + max(1, bin(mask).count("1")) - window) if window else 0
    front = [j for j in range(max(base, 0)) if not window or j >= first or j < sinks]
    assert not window or mask == 0 or first == max(0, p + 1 - window)
    return front + [base + j for j in range(c) if mask >> j & 1 and base + j >= 0]


def mask_words(masks, words):
    """Integers of bits -> int32 [rows, words]."""
    raw = np.array([[(m >> (32 * w)) & 0xFFFFFFFF for w in range(words)] for m in masks], np.uint32).reshape(len(masks), words)
    return torch.from_numpy(raw.view(np.int32).copy())


def tree_masks(parents):
    got = []
    for j, p in enumerate(parents):
        got.append((got[p] if p >= 0 else 0) | 1 << j)
    return got


def attention_where(Q, cache, bt, H, scale, seen):
    """Binary64 attention over the cached values at the positions seen[row].  Returns (o, lse, allowance) as
    kv_util.attention_reference, whose docstring derives the allowance; the number of additions of the value product is
    counted over all tokens of the sequence, whether seen or not."""
    rows, Hq, D = Q.shape
    G, P = Hq // H, bt.P
    K, V, ks, vs = decode_pages(cache, H, D, P)
    Qd = Q.cpu().double()
    o = torch.zeros(rows, Hq, D, dtype=torch.float64)
    lse = torch.full((rows, Hq), -np.inf, dtype=torch.float64)
    allow = torch.zeros_like(o)
    row = 0
    for b, (n, c) in enumerate(zip(bt.lens, bt.counts)):
        pages = torch.from_numpy(bt.table_host[b, :-(-n // P)]).long().clamp(min=0)      # (-1: a page that is gone, unseen)
        Kb, Vb = (x[pages].transpose(0, 1).reshape(H, -1, D).repeat_interleave(G, 0) for x in (K, V))
        ksb, vsb = (x[pages].transpose(0, 1).reshape(H, -1).repeat_interleave(G, 0) for x in (ks, vs))
        for i in range(c):
            at = torch.tensor(seen[row], dtype=torch.long)
            if len(at):
                k, v, q = Kb[:, at], Vb[:, at], Qd[row]
                s = torch.einsum("hnd,hd->hn", k, q) * scale
                lse[row] = torch.logsumexp(s, -1)
                p = torch.exp(s - lse[row][:, None])
                o[row] = torch.einsum("hn,hnd->hd", p, v)
                ds = (D / 16 + 4) * 2.0 ** -23 * 30 * q.abs().sum(-1, keepdim=True) * ksb[:, at] * scale + 2.0 ** -20 * (1 + s.abs())
                allow[row] = (torch.einsum("hn,hnd->hd", p * ds, (v - o[row][:, None]).abs())
                              + (2.0 ** -11 + 2.0 ** -20) * torch.einsum("hn,hnd->hd", p, v.abs())
                              + 2.0 ** -23 * (n / 16 + 40) * (p * 30 * vsb[:, at]).sum(-1, keepdim=True))
            row += 1
    return o, lse, allow


def plan_reference(held, kept, add, table, free, count, P, rows):
    """A step's plan, one page at a time.  Returns None where it is refused, else a dict."""
    B, most = table.shape
    table, free = table.copy(), free.copy()
    stack = list(free[:count])
    had = [-(-h // P) for h in held]
    has = [-(-(k + a) // P) for k, a in zip(kept, add)]
    for b in range(B):
        for i in range(has[b], had[b]):
            stack.append(table[b, i])
    grown = list(stack)
    if sum(max(0, n - h) for n, h in zip(has, had)) > len(stack) or sum(add) > rows or len(stack) > len(free):
        return None
    for b in range(B):
        for i in range(had[b], has[b]):
            table[b, i] = stack.pop()
    free[count:len(stack)] = grown[count:len(stack)]
    cu = np.concatenate([[0], np.cumsum(add)])
    positions, slots = np.zeros(rows, np.int32), np.full(rows, -1, np.int64)
    r = 0
    for b in range(B):
        for p in range(kept[b], kept[b] + add[b]):
            positions[r], slots[r] = p, int(table[b, p // P]) * P + p % P
            r += 1
    return dict(table=table, free=free, count=np.array([len(stack)], np.int32), cu=cu.astype(np.int32), lens=np.array([k + a for k, a in zip(kept, add)], np.int32),
                positions=positions, slots=slots)


def rotate_reference(x, positions, axis, inv_freq, interleaved):
    """numpy: x [rows, heads, D] float32, positions [axes, rows], axis [pairs], inv_freq float32 [pairs] -> float32, the header's operations
    one by one."""
    pairs = len(inv_freq)
    angle = positions[axis].T.astype(np.float64) * inv_freq.astype(np.float64)        # [rows, pairs]
    c, s = np.cos(angle).astype(np.float32)[:, None], np.sin(angle).astype(np.float32)[:, None]
    i = np.arange(pairs)
    ia, ib = (2 * i, 2 * i + 1) if interleaved else (i, i + pairs)
    a, b = x[..., ia], x[..., ib]
    y = x.copy()
    y[..., ia], y[..., ib] = a * c - b * s, b * c + a * s
    return y
