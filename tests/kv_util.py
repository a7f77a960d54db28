"""Plain references of the paged dINT4 cache and the attention over it, from the definitions in
include/w4a8.h, and a seeded batch on the device."""
import numpy as np
import torch

import paper_2311_05161_b200 as w4a8

LARGEST = {torch.float16: 65504.0, torch.bfloat16: 3.3895313892515355e38}


def quantize_vectors(x):
    """numpy float32 [..., D] -> (levels float64 in steps, step float32 [..., 1], z int [..., 1]): binary32
    operations one by one, as the header writes them."""
    x = np.asarray(x, np.float32)
    one = np.float32(1)
    lo = np.minimum(np.float32(0), x.min(-1, keepdims=True))
    hi = np.maximum(np.float32(0), x.max(-1, keepdims=True))
    raw = (hi * np.float32(0.5) - lo * np.float32(0.5)) / np.float32(6.5)
    step = ((raw.view(np.uint32) + np.uint32(8)) & ~np.uint32(15)).view(np.float32)
    step = np.where(raw < np.float32(2.0 ** -100), one, step).astype(np.float32)
    r = one / step
    z = np.clip(np.rint(-lo * r), 0, 13)
    u = x * r
    plain = np.clip(np.rint(u) + z, 0, 13) - z
    special = (np.abs(u) > np.float32(0.25)) & (np.abs(u) <= np.float32(0.75))
    return np.where(special, 0.5 * np.sign(u), plain).astype(np.float64), step, z.astype(np.int64)


def levels_of(z):
    return sorted([k - z for k in range(14)] + [0.5, -0.5])


def encode_block(K, V):
    """K, V numpy float32 [16, D] of one head -> the block's bytes."""
    D = K.shape[1]
    out = np.zeros(16 * (D + 8), np.uint8)
    words = out[16 * D:].view(np.uint32)
    for which, x in enumerate((K, V)):
        lev, step, z = quantize_vectors(x)
        for s in range(16):
            zz = int(z[s, 0])
            table = levels_of(zz)
            rank = [table.index(v) for v in lev[s]]
            code = np.zeros(D // 2, np.uint8)
            for i in range(D // 4):
                h = sum(rank[4 * i + k] << (4 * k) for k in range(4))
                h = ((h << 2) | (h >> 14)) & 0xFFFF
                code[2 * i], code[2 * i + 1] = h & 255, h >> 8
            if which == 0:
                out[s * (D // 2):(s + 1) * (D // 2)] = code
            else:
                c = D // 16
                for g in range(8):
                    at = 8 * D + ((s // 8 * 8 + g) * 8 + s % 8) * c
                    out[at:at + c] = code[g * c:(g + 1) * c]
            words[16 * which + s] = int(step[s].view(np.uint32)[0]) | zz
    return out


def decode_pages(cache, H, D, P):
    """uint8 cache [pages, bytes] -> K, V values, step: [pages, H, P, D] float64 x 2, [pages, H, P] x 2."""
    raw = cache.cpu().view(-1, H, P // 16, 16 * (D + 8))
    word = raw[..., 16 * D:].contiguous().view(torch.int32).view(raw.shape[0], H, P // 16, 2, 16)
    table = torch.tensor([levels_of(min(z, 13)) for z in range(16)], dtype=torch.float64)
    vals, steps = [], []
    for which in (0, 1):
        c = raw[..., 8 * D * which:8 * D * (which + 1)]
        c = c.reshape(*c.shape[:3], 2, 8, 8, D // 16).transpose(-3, -2) if which else c
        c = c.reshape(raw.shape[0], H, P, D // 4, 2).long()
        h = c[..., 0] + 256 * c[..., 1]
        h = (h >> 2) | ((h & 3) << 14)
        rank = torch.stack([(h >> (4 * k)) & 15 for k in range(4)], -1).reshape(raw.shape[0], H, P, D)
        w = word[..., which, :].reshape(raw.shape[0], H, P)
        step = (w & ~15).view(torch.float32).double()
        vals.append(torch.gather(table[(w & 15).long()], -1, rank) * step[..., None])
        steps.append(step)
    return vals[0], vals[1], steps[0], steps[1]


class Batch:
    """A seeded batch: sequence lengths, rows per sequence, a page table of shuffled pages."""

    def __init__(self, lens, rows=None, P=16, pad_rows=0, extra_pages=2, seed=0):
        rng = np.random.default_rng(seed)
        self.lens, self.P = list(lens), P
        self.counts = [1] * len(lens) if rows is None else list(rows)
        need = [-(-n // P) for n in lens]
        self.max_pages = max(1, max(need))
        self.num_pages = sum(need) + extra_pages
        perm = rng.permutation(self.num_pages)
        # entries that no token needs name no page: reading one is reported
        table = np.full((len(lens), self.max_pages), -7, np.int32)
        at = 0
        for b, n in enumerate(need):
            table[b, :n] = perm[at:at + n]
            at += n
        self.table_host = table
        self.table = torch.from_numpy(table).cuda()
        self.kv_lens = torch.tensor(self.lens, dtype=torch.int32).cuda()
        self.start = np.concatenate([[0], np.cumsum(self.counts)])
        self.used = int(self.start[-1])
        self.rows = self.used + pad_rows
        self.cu = None if rows is None else torch.tensor(self.start, dtype=torch.int32).cuda()

    def positions(self):
        """(sequence, position) of every used row."""
        return [(b, n - c + i) for b, (n, c) in enumerate(zip(self.lens, self.counts)) for i in range(c)]


def vectors(shape, seed, dtype, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g) * torch.exp(0.7 * torch.randn(shape[-2:], generator=g))
    return ((x + 0.4 * torch.randn(shape[-2:], generator=g)) * scale).to(dtype)


def filled_cache(bt, H, D, seed=1, dtype=torch.float16, scale=1.0):
    """A cache whose every page holds quantized vectors, written by kv_append."""
    P = bt.P
    cache = w4a8.new_kv_cache(bt.num_pages, P, H, D)
    ws = w4a8.new_kv_workspace(1, 1, H, H, D)
    table = torch.arange(bt.num_pages, dtype=torch.int32, device="cuda").view(1, -1)
    n = bt.num_pages * P
    K, V = vectors((n, H, D), seed, dtype, scale).cuda(), vectors((n, H, D), seed + 1, dtype, scale).cuda()
    w4a8.kv_append(K, V, cache, table, torch.tensor([n], dtype=torch.int32, device="cuda"), ws,
                   cu_rows=torch.tensor([0, n], dtype=torch.int32, device="cuda"))
    w4a8.check_status(ws)
    return cache


def attention_reference(Q, cache, bt, H, scale, causal=True, window=0):
    """Binary64 attention over the cached values.  Returns (o, lse, allowance): the allowance covers
    what the kernel rounds besides its output.

    A score is s = (step * scale) * sum_d q_d level_d.  The kernel contracts exact products in binary32
    with the levels offset by up to 30 and takes the offset out again: at most D / 16 + 4 additions, each
    off by 2^-23 of at most 30 sum |q|, so |ds| <= (D / 16 + 4) 2^-23 30 sum|q| step scale, plus a few
    binary32 roundings of s itself.  A weight p enters the value product as binary16 (2^-11), and its exponential
    is good to 2^-21; so o is off by sum_j p_j |v_j - o| (ds_j) + 2^-11 sum_j p_j |v_j| to first order.  The value
    product carries an offset of up to 30 steps in binary32: 2^-23 of it per addition, n / 16 + 40
    additions."""
    rows, Hq, D = Q.shape
    G, P = Hq // H, bt.P
    K, V, ks, vs = decode_pages(cache, H, D, P)
    Qd = Q.cpu().double()
    o = torch.zeros(rows, Hq, D, dtype=torch.float64)
    lse = torch.full((rows, Hq), -np.inf, dtype=torch.float64)
    allow = torch.zeros_like(o)
    row = 0
    for b, (n, c) in enumerate(zip(bt.lens, bt.counts)):
        pages = torch.from_numpy(bt.table_host[b, :-(-n // P)]).long()
        Kb, Vb = (x[pages].transpose(0, 1).reshape(H, -1, D)[:, :n] for x in (K, V))
        ksb, vsb = (x[pages].transpose(0, 1).reshape(H, -1)[:, :n] for x in (ks, vs))
        for i in range(c):
            pos = n - c + i
            hi = pos + 1 if causal else n
            lo = max(0, pos + 1 - window) if window else 0
            if pos >= 0 and hi > lo:
                for h in range(Hq):
                    k, v = Kb[h // G, lo:hi], Vb[h // G, lo:hi]
                    q = Qd[row, h]
                    s = (k @ q) * scale
                    lse[row, h] = torch.logsumexp(s, 0)
                    p = torch.exp(s - lse[row, h])
                    o[row, h] = p @ v
                    ds = (D / 16 + 4) * 2.0 ** -23 * 30 * q.abs().sum() * ksb[h // G, lo:hi] * scale
                    ds = ds + 2.0 ** -20 * (1 + s.abs())
                    offset = 30 * vsb[h // G, lo:hi]
                    allow[row, h] = ((p * ds) @ (v - o[row, h]).abs() + (2.0 ** -11 + 2.0 ** -20) * (p @ v.abs())
                                     + 2.0 ** -23 * ((hi - lo) / 16 + 40) * (p @ offset))
            row += 1
    return o, lse, allow


def check_attention(O, o, allow, dtype):
    """O against o: half a step of the output type besides the allowance."""
    got = O.double().cpu()
    tol = allow * 1.05 + torch.finfo(dtype).eps / 2 * o.abs() + torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
    bad = ~((got - o).abs() <= tol)
    assert not bad.any(), f"{int(bad.sum())} outputs beyond tolerance, first at {tuple(int(i) for i in bad.nonzero()[0])}: " \
        f"worst {float(((got - o).abs() / tol).max()):.3g} of it"
