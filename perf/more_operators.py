"""Operators of serving with a 4-bit paged cache, with their plain forms: the batch's plan on the device, rotary positions with
the cache write, attention with a window and sinks, attention of drafted trees and the acceptance of a path.

Five operators, in the order in which a serving step meets them:

  plan    page table, row offsets, positions and slots of a step from the requests' lengths, pages taken from and
          given back to a free list (kv_plan)
  rope    rotary positions with one or several axes on queries and keys; the keys and values enter the cache
          (rope_kv_append)
  sinks   attention with a sliding window and a few first tokens that stay visible (kv_attention_sinks)
  tree    attention of the rows of a tree of drafted tokens: the cached tokens before them, and their own
          ancestors by a mask (kv_attention_tree)
  accept  the accepted path's tokens move to the front of the drafted ones (kv_accept), here between the write
          of the drafts (kv_append) and a read of their slots (kv_read)

The cache: pages of P tokens; a page holds, for each key/value head, P / 16 blocks of 16 tokens; a
block is [16][D/2] bytes of key codes, D/2 * 16 bytes of value codes, sixteen 32-bit words for
the keys and sixteen for the values.  Such a word is the binary32 step with its last four
mantissa bits replaced by the zero-point z.  A token's vector is quantized by Eq. 5 of the dINT4
format over its D elements (step = range / 13, levels -z..13-z and the two specials +-1/2); what is
stored is a level's rank 0..15 in ascending order.  Four ranks r0..r3 of consecutive elements make
the 16-bit number r0 + 16 r1 + 256 r2 + 4096 r3, stored rotated left by two bits.  Keys are stored
token by token; values as [2][8][8][D/16] bytes: half of the block, slice of D/8 elements, token
of the half, bytes of the slice.

`own` False: plain torch operations.  `own` True: the framework's entry points.
"""
import math
import random

import torch

own = False

F16, BF16, F32, F64 = torch.float16, torch.bfloat16, torch.float32, torch.float64
TYPES = {"f16": F16, "bf16": BF16}
LARGEST = {F16: 65504.0, BF16: 3.3895313892515355e38}


# ---------------------------------------------------------------------------- the cases
def listed():
    return [
        # a decode step of eight requests, one token each: latency
        dict(name="plan, 8 x 1 token", op="plan", B=8, mix="decode", hi=3000, P=64, spare=0),
        # a large engine's step: requests that go on, prompts that begin, drafts taken back, requests that ended
        dict(name="plan, 1500 requests, prompts", op="plan", B=1500, mix="all", hi=1200, P=32, spare=77),
        # eight requests' next tokens, queries, keys and values slices of one projection output
        dict(name="rope, 8 x 1 token, 32/8 heads", op="rope", B=8, lo=1, hi=1900, rows_lo=1, rows_hi=1, Hq=32, Hkv=8, D=128, rot=128, P=64,
             x="bf16", axes=1, base=10000.0, interleaved=False, fused=True),
        # four prompts with an image each: three axes
        dict(name="rope, 4 prompts with images", op="rope", B=4, lo=611, hi=4097, rows_lo=611, rows_hi=4097, Hq=32, Hkv=8, D=128, rot=128, P=64,
             x="bf16", axes=3, base=1000000.0, interleaved=False, fused=False),
        # one request far beyond its window
        dict(name="sinks, 1 x 100001, window 4096", op="sinks", B=1, lo=100001, hi=100001, rows_lo=1, rows_hi=1, Hq=32, Hkv=8, D=128, P=64,
             x="bf16", o="f16", window=4096, sinks=4),
        # a full batch of long chats with eight query heads to a key head
        dict(name="sinks, 64 ragged, window 2047", op="sinks", B=64, lo=900, hi=20000, rows_lo=1, rows_hi=1, Hq=64, Hkv=8, D=128, P=64,
             x="f16", o="f16", window=2047, sinks=5),
        # a chunk of a long prompt
        dict(name="sinks, chunk of 1024 at 9000", op="sinks", B=1, lo=9000, hi=9000, rows_lo=1024, rows_hi=1024, Hq=32, Hkv=8, D=128, P=64,
             x="bf16", o="f16", window=4096, sinks=4),
        # one request, a small tree
        dict(name="tree, 1 x 7 nodes at 2049", op="tree", B=1, lo=2049, hi=2049, rows_lo=7, rows_hi=7, Hq=32, Hkv=8, D=128, P=64,
             x="bf16", o="f16", window=0, sinks=0),
        # a batch of requests, small trees of different sizes, every head with keys of its own
        dict(name="tree, 12 ragged, 32 heads", op="tree", B=12, lo=0, hi=3500, rows_lo=3, rows_hi=13, Hq=32, Hkv=32, D=128, P=64,
             x="bf16", o="bf16", window=0, sinks=0),
        # a batch with wide trees
        dict(name="tree, 16 x up to 64 nodes", op="tree", B=16, lo=1000, hi=6000, rows_lo=40, rows_hi=64, Hq=32, Hkv=8, D=128, P=64,
             x="f16", o="f16", window=0, sinks=0),
        # eight requests, a path of a few tokens each
        dict(name="accept, 8 x 16 nodes, 8 heads", op="accept", B=8, lo=10, hi=400, rows_lo=16, rows_hi=16, most_accepted=5, Hkv=8, D=128, P=64, x="bf16"),
        # a large batch with wide trees, every head with keys of its own
        dict(name="accept, 64 x 48 nodes, 32 heads", op="accept", B=64, lo=10, hi=200, rows_lo=48, rows_hi=48, most_accepted=9, Hkv=32, D=128, P=64, x="f16"),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["plan", "rope", "rope", "sinks", "sinks", "tree", "tree", "accept"])
    if op == "plan":
        B = log(1, 1500)
        return dict(op=op, B=B, mix=rng.choice(["decode", "all", "all"]), hi=log(1, max(2, min(20000, 1_500_000 // B))), P=rng.choice([16, 32, 64, 128, 256]),
                    spare=rng.choice([0, 1, 77]))
    D, P, x = rng.choice([64, 128, 128]), rng.choice([16, 32, 64, 128]), rng.choice(["f16", "bf16"])
    Hkv = rng.choice([1, 2, 4, 8, 12, 32])
    if op == "accept":
        B, n = log(1, 64), log(1, 64)
        while B * n * Hkv > 98304:
            B = max(1, B // 2)
        return dict(op=op, B=B, lo=rng.choice([0, 1, 17]), hi=log(20, 250), rows_lo=rng.choice([1, n]), rows_hi=n, most_accepted=rng.randint(1, n), Hkv=Hkv, D=D,
                    P=P, x=x)
    G, B = rng.choice([1, 2, 4, 5, 7, 8, 16]), log(1, 64)
    if op == "rope":
        G = min(G, 64 // Hkv)
        lo = rng.choice([0, 1, 17])
        hi = lo + log(1, max(2, min(4096, 300_000 // (B * Hkv * (G + 2)))))
        rows_hi = rng.choice([1, hi, max(1, hi // 3)])
        return dict(op=op, B=B, lo=max(lo, rows_hi), hi=max(hi, rows_hi), rows_lo=rng.choice([1, rows_hi]), rows_hi=rows_hi, Hq=Hkv * G, Hkv=Hkv, D=D,
                    rot=rng.choice([D, D, D // 2, 16, 48]), P=P, x=x, axes=rng.choice([1, 1, 3, 4]), base=rng.choice([10000.0, 500000.0, 1000000.0]),
                    interleaved=rng.random() < 0.4, fused=rng.random() < 0.5)
    window = log(1, 8192)
    if op == "sinks":
        rows_hi = rng.choice([1, 1, 1, 2, 4, max(1, min(1024, 600 // B))])
        hi = log(1, max(2, min(100_000, 1_600_000 // (B * Hkv))))
        while rows_hi > 1 and B * rows_hi * Hkv * G * min(hi, window + rows_hi) > 100_000_000:
            rows_hi //= 2
        return dict(op=op, B=B, lo=rng.choice([0, 1, hi // 2, hi]), hi=hi, rows_lo=rng.choice([1, rows_hi]) if rows_hi > 1 else 1, rows_hi=rows_hi,
                    Hq=Hkv * G, Hkv=Hkv, D=D, P=P, x=x, o=rng.choice(["f16", "bf16"]), window=window, sinks=rng.choice([1, 4, 4, 16, 17, 64, 100]))
    n = log(1, 160)
    hi = log(1, max(2, min(60_000, 1_200_000 // (B * Hkv))))
    while n > 1 and B * n * Hkv * G * (hi + n) > 60_000_000:
        n //= 2
    return dict(op=op, B=B, lo=rng.choice([0, 1, hi // 2, hi]), hi=hi, rows_lo=rng.choice([1, n]), rows_hi=n, Hq=Hkv * G, Hkv=Hkv, D=D, P=P, x=x,
                o=rng.choice(["f16", "bf16"]), window=rng.choice([0, 0, 0, window]), sinks=rng.choice([0, 4]))


def _spread(n, lo, hi, salt):
    """n whole numbers from lo to hi, both among them: the case alone gives them."""
    got = [lo + (b * 2654435761 + salt * 40503 + 12345) % 1000003 % (hi - lo + 1) for b in range(n)]
    got[0] = hi
    if n > 1:
        got[n // 2] = lo
    return got


def _lengths(c):
    """Tokens of each sequence with the call's rows, and its rows.  Drafted rows come on top of lo .. hi tokens."""
    lens = _spread(c["B"], c["lo"], c["hi"], 1)
    if (c["rows_lo"], c["rows_hi"]) == (c["lo"], c["hi"]) and c["op"] not in ("tree", "accept"):
        return lens, list(lens)
    rows = _spread(c["B"], c["rows_lo"], c["rows_hi"], 2)
    if c["op"] in ("tree", "accept"):
        lens = [n + r for n, r in zip(lens, rows)]
    return lens, rows


def _requests(c):
    """plan: (held, kept, added) tokens of each request."""
    rng = random.Random(c["B"] * 1000003 + c["hi"])
    got = []
    for b in range(c["B"]):
        n = rng.randint(1, c["hi"])
        kind = "decode" if c["mix"] == "decode" else rng.choice(["decode", "decode", "prompt", "prompt", "draft", "ended", "idle"])
        if kind == "decode":
            got.append((n, n, 1))
        elif kind == "prompt":                 # from nothing, or a further chunk
            at = rng.choice([0, 0, n // 2])
            got.append((at, at, n))
        elif kind == "draft":                  # some of the drafted rows were not accepted, new ones follow
            got.append((n, max(0, n - rng.randint(0, 60)), rng.randint(1, 60)))
        else:
            got.append((n, 0, 0) if kind == "ended" else (n, n, 0))
    return got


def _tree(n, rng):
    """Parents of n drafted rows, -1 for the root's children: chains and branches."""
    return [-1 if j == 0 else rng.choice([j - 1, rng.randint(max(-1, j - 9), j - 1), rng.randint(-1, j - 1)]) for j in range(n)]


def _first(p, window):
    return max(0, p + 1 - window) if window else 0


def work(c):
    if c["op"] == "plan":
        B, P = c["B"], c["P"]
        req = _requests(c)
        rows = sum(a for _, _, a in req)
        pages = sum(abs(-(-(k + a) // P) - -(-h // P)) for h, k, a in req)
        return {"bytes": B * 12 + (B + 1) * 4 + B * 4 + rows * 12 + pages * 8, "flops": 4 * rows}
    lens, rows = _lengths(c)
    vec, T = c["D"] // 2 + 4, sum(rows)        # bytes of a cached vector: codes and one word
    if c["op"] == "rope":
        n = T * c["Hkv"] * 2
        return {"bytes": T * c["Hq"] * c["D"] * 4 + n * (2 * c["D"] + vec) + n * (2 * c["D"] + vec) + T * (8 + 4 * c["axes"]),
                "flops": 6 * T * (c["Hq"] + c["Hkv"]) * c["rot"] + 8 * n * c["D"]}
    if c["op"] == "accept":
        n = T * c["Hkv"] * 2
        moved = sum(min(c["most_accepted"], r) for r in rows) * c["Hkv"] * 2
        return {"bytes": n * (4 * c["D"] + 2 * vec) + moved * 2 * vec, "flops": 8 * n * c["D"]}
    w, sinks = c["window"], c["sinks"]
    keys = pairs = 0
    for n, r in zip(lens, rows):
        if c["op"] == "tree":
            low = _first(n - r, w)
            keys += n - low + min(sinks, low)
            pairs += r * (n - r - low + min(sinks, low)) + r * min(r, 8)
        elif n:
            first = _first(max(0, n - r), w)
            keys += n - first + min(sinks, first)
            for p in range(max(0, n - r), n):
                pairs += p + 1 - _first(p, w) + min(sinks, _first(p, w))
    return {"bytes": keys * c["Hkv"] * 2 * vec + T * c["Hq"] * c["D"] * 4, "flops": 4 * pairs * c["Hq"] * c["D"]}


# ---------------------------------------------------------------------------- inputs
def _vectors(shape, g, spread):
    """Key- or value-like vectors: some channels are larger and off centre, tokens differ in size."""
    heads, D = shape[-2:]
    gain = torch.exp(0.6 * torch.randn(heads, D, generator=g, device="cuda"))
    shift = 0.4 * torch.randn(heads, D, generator=g, device="cuda")
    size = torch.exp(0.3 * torch.randn(shape[:-1] + (1,), generator=g, device="cuda"))
    x = torch.randn(shape, generator=g, device="cuda").mul_(gain).add_(shift)
    return x.mul_(size).mul_(spread)


def _prepare_plan(c, s, g):
    req, P = _requests(c), c["P"]
    held, kept, add = (torch.tensor(x, dtype=torch.int32) for x in zip(*req))
    most = max(1, max(-(-max(h, k + a) // P) for h, k, a in req)) + 2
    have = [-(-h // P) for h, _, _ in req]
    need = sum(max(0, -(-(k + a) // P) - h) for (_, k, a), h in zip(req, have))
    pages = sum(have) + need + 5 + c["spare"]
    perm = torch.randperm(pages, generator=g, device="cuda").to(torch.int32).cpu()
    table, at = torch.full((c["B"], most), -1, dtype=torch.int32), 0
    for b, k in enumerate(have):
        table[b, :k] = perm[at:at + k]
        at += k
    free = torch.full((pages,), -1, dtype=torch.int32)
    free[:pages - at] = perm[at:]
    s.update(held=held.cuda(), kept=kept.cuda(), add=add.cuda(), table=table.cuda(), free=free.cuda(), most=most, pages=pages,
             count=torch.tensor([pages - at], dtype=torch.int32, device="cuda"), max_rows=int(add.sum()) + c["spare"])
    s["max_rows"] = max(1, s["max_rows"])
    i32 = dict(dtype=torch.int32, device="cuda")
    # the buffers that a captured step writes and its later calls read
    s["out"] = (torch.zeros(c["B"], **i32), torch.zeros(c["B"] + 1, **i32), torch.zeros(s["max_rows"], **i32),
                torch.zeros(s["max_rows"], dtype=torch.int64, device="cuda"), torch.zeros(1, **i32))
    return s


def prepare(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(c)
    if c["op"] == "plan":
        return _prepare_plan(c, s, g)
    rng = random.Random(seed)
    lens, rows = _lengths(c)
    B, P, H, D = c["B"], c["P"], c["Hkv"], c["D"]
    most = max(1, -(-max(lens) // P))
    pages = sum(-(-n // P) for n in lens) + 3
    s["lens"], s["rows"], s["most"], s["T"] = lens, rows, most, sum(rows)
    perm = torch.randperm(pages, generator=g, device="cuda").to(torch.int32).cpu()
    table, at = torch.zeros(B, most, dtype=torch.int32), 0
    for b, n in enumerate(lens):
        k = -(-n // P)
        table[b, :k] = perm[at:at + k]
        at += k
    s["table"] = table.cuda()
    s["kv_lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    cu = [0]
    for r in rows:
        cu.append(cu[-1] + r)
    s["cu"] = None if all(r == 1 for r in rows) else torch.tensor(cu, dtype=torch.int32, device="cuda")
    # for the plain forms: sequence, place and position of every row
    seq = torch.repeat_interleave(torch.arange(B), torch.tensor(rows)).cuda()
    s["seq"] = seq
    s["row_of"] = torch.arange(s["T"], device="cuda") - torch.tensor(cu, device="cuda")[seq]
    s["pos"] = s["kv_lens"][seq].long() - torch.tensor(rows, device="cuda")[seq] + s["row_of"]
    if c["op"] in ("rope", "accept"):
        s["cache"] = torch.zeros(pages, H * (P // 16) * (16 * D + 128), dtype=torch.uint8, device="cuda")
        K, V = _vectors((s["T"], H, D), g, 1.5).to(TYPES[c["x"]]), _vectors((s["T"], H, D), g, 0.7).to(TYPES[c["x"]])
        if c["op"] == "accept":
            s["K"], s["V"] = K, V
            s["counts"] = [rng.randint(1, min(c["most_accepted"], r)) for r in rows]
            s["paths"] = [sorted(rng.sample(range(r), k)) for r, k in zip(rows, s["counts"])]
            paths = torch.full((B, c["most_accepted"]), -1, dtype=torch.int32)
            for b, path in enumerate(s["paths"]):
                paths[b, :len(path)] = torch.tensor(path, dtype=torch.int32)
            s["accepted"], s["accept_lens"] = paths.cuda(), torch.tensor(s["counts"], dtype=torch.int32, device="cuda")
            return s
        Q = (1.3 * torch.randn(s["T"], c["Hq"], D, generator=g, device="cuda")).to(TYPES[c["x"]])
        if c["fused"]:                         # slices of one wider projection output
            wide = torch.cat([Q, K, V], 1)
            Q, K, V = wide[:, :c["Hq"]], wide[:, c["Hq"]:c["Hq"] + H], wide[:, c["Hq"] + H:]
        s["Q"], s["K"], s["V"] = Q, K, V
        pos = s["pos"].to(torch.int32)
        if c["axes"] > 1:                      # the middle third of a request's rows is a grid of patches
            n = torch.tensor(rows, device="cuda")[seq]
            k = s["row_of"] - n // 3
            inside, wide = (k >= 0) & (s["row_of"] < n - n // 3), (1 + (n // 3).float().sqrt()).long()
            start = s["pos"] - k
            grid = [start, start + k // wide, start + k % wide, start + k % 2]
            pos = torch.stack([torch.where(inside, grid[a], s["pos"]) for a in range(c["axes"])]).to(torch.int32)
        s["positions"] = pos.contiguous()
        half = c["rot"] // 2
        s["inv_freq"] = (c["base"] ** (-torch.arange(half, dtype=F64) * 2 / c["rot"])).to(F32).cuda()
        s["pair_axis"] = (torch.arange(half) * c["axes"] // half).to(torch.int32).cuda() if c["axes"] > 1 else None
        s["slots"] = s["table"][seq, s["pos"] // P].long() * P + s["pos"] % P
        return s
    # a filled cache, page by page
    K = _vectors((pages, H, P // 16, 16, D), g, 1.5)
    kc, km = _encode(K.to(TYPES[c["x"]]).float())
    K = _vectors((pages, H, P // 16, 16, D), g, 0.7)
    vc, vm = _encode(K.to(TYPES[c["x"]]).float())
    del K
    s["cache"] = torch.cat([kc.flatten(3), _v_order(vc).flatten(3), km.view(torch.uint8).flatten(3), vm.view(torch.uint8).flatten(3)], 3).reshape(pages, -1).contiguous()
    s["Q"] = (1.3 * torch.randn(s["T"], c["Hq"], D, generator=g, device="cuda")).to(TYPES[c["x"]])
    s["scale"] = 1.0 / math.sqrt(D)
    if c["op"] == "tree":
        words = -(-max(rows) // 32)
        s["parents"] = [_tree(r, rng) for r in rows]
        bits = []
        for parents in s["parents"]:
            mine = []
            for j, p in enumerate(parents):
                mine.append((mine[p] if p >= 0 else 0) | 1 << j)
            bits += mine
        full = 1 << 32
        mask = [[(m >> 32 * w) % full - (full if m >> (32 * w + 31) & 1 else 0) for w in range(words)] for m in bits]
        s["mask"] = torch.tensor(mask, dtype=torch.int32).view(-1, words).cuda()
    return s


# ---------------------------------------------------------------------------- the cache format
def _encode(x):
    """x [..., D] binary32 -> codes [..., D/2] uint8 (keys' order) and words [...] int32."""
    one = torch.ones((), device=x.device)
    lo, hi = x.amin(-1, keepdim=True).clamp(max=0.0), x.amax(-1, keepdim=True).clamp(min=0.0)
    raw = (hi * 0.5 - lo * 0.5) / (one * 6.5)
    step = ((raw.view(torch.int32) + 8) & ~15).view(F32)
    step = torch.where(raw < 2.0 ** -100, one * 2.0 ** -64, step)
    r = one / step
    z = torch.round(-lo * r).clamp(0, 13)
    u = x * r
    special = (u.abs() > 0.25) & (u.abs() <= 0.75)
    level = (torch.round(u) + z).clamp(0, 13) - z
    rank = torch.where(special, torch.sign(u), level + torch.sign(level)) + z + 1
    q = rank.to(torch.int32).unflatten(-1, (-1, 4))
    h = q[..., 0] | (q[..., 1] << 4) | (q[..., 2] << 8) | (q[..., 3] << 12)
    h = (((h << 2) | (h >> 14)) & 0xFFFF)
    codes = torch.where(h >= 32768, h - 65536, h).to(torch.int16).view(torch.uint8)
    return codes, (step.view(torch.int32) | z.to(torch.int32)).squeeze(-1)


def _v_order(codes):
    """Value codes of blocks [..., 16, D/2] in their stored order."""
    return codes.unflatten(-1, (8, -1)).unflatten(-3, (2, 8)).transpose(-3, -2).contiguous()


def _decode(codes, word):
    """Codes [..., D/2] uint8 and words [...] -> values [..., D] binary32."""
    h = codes.contiguous().view(torch.int16).to(torch.int32) & 0xFFFF
    h = ((h >> 2) | (h << 14)) & 0xFFFF
    rank = torch.stack([h & 15, (h >> 4) & 15, (h >> 8) & 15, h >> 12], -1).flatten(-2)
    x = (rank - (word & 15).unsqueeze(-1) - 1).to(F32)
    return (x - (x * 0.5).clamp(-1.0, 1.0)) * (word & ~15).view(F32).unsqueeze(-1)


def _stored(s, page, place):
    """Codes and words of the keys and of the values of tokens at places of pages: [..., H, D/2] and [..., H] each."""
    H, D, P = s["Hkv"], s["D"], s["P"]
    block, slot = place // 16, place % 16
    blocks = s["cache"].view(-1, H, P // 16, 16 * D + 128)
    word = s["cache"].view(torch.int32).view(-1, H, P // 16, 4 * D + 32)[..., 4 * D:].unflatten(-1, (2, 16))
    kc = blocks[..., :8 * D].unflatten(-1, (16, D // 2))[page, :, block, slot]
    vc = blocks[..., 8 * D:16 * D].unflatten(-1, (2, 8, 8, D // 16)).transpose(-3, -2)[page, :, block, slot // 8, slot % 8].flatten(-2)
    return kc, word[page, :, block, 0, slot], vc, word[page, :, block, 1, slot]


def _store(s, page, place, kc, kw, vc, vw):
    H, D, P = s["Hkv"], s["D"], s["P"]
    flat, block = s["cache"].view(-1), 16 * D + 128
    base = ((page[:, None] * H + torch.arange(H, device="cuda")) * (P // 16) + (place // 16)[:, None]) * block  # [T, H]
    slot = (place % 16)[:, None]
    four, byte, c = torch.arange(4, device="cuda"), torch.arange(D // 2, device="cuda"), D // 16
    for_v = ((slot // 8)[..., None] * 8 + byte // c) * 8 * c + (slot % 8)[..., None] * c + byte % c
    flat[(base[..., None] + slot[..., None] * (D // 2) + byte).flatten()] = kc.flatten()
    flat[(base[..., None] + 8 * D + for_v).flatten()] = vc.flatten()
    flat[(base[..., None] + 16 * D + 4 * slot[..., None] + four).flatten()] = kw.unsqueeze(-1).contiguous().view(torch.uint8).flatten()
    flat[(base[..., None] + 16 * D + 64 + 4 * slot[..., None] + four).flatten()] = vw.unsqueeze(-1).contiguous().view(torch.uint8).flatten()


# ---------------------------------------------------------------------------- plain forms
def _plain_plan(s):
    P, most, device = s["P"], s["most"], "cuda"
    held, kept, add = s["held"].long(), s["kept"].long(), s["add"].long()
    had, lens = (held + P - 1) // P, kept + add
    has = (lens + P - 1) // P
    page = torch.arange(most, device=device)
    back = (page >= has[:, None]) & (page < had[:, None])
    new = (page >= had[:, None]) & (page < has[:, None])
    F, A, count = back.sum(), new.sum(), s["count"].long()
    # the free list with what is given back on top of it, by request and page
    at = torch.where(back, count + back.flatten().cumsum(0).view(back.shape) - 1, s["pages"])
    stack = torch.cat([s["free"], s["free"][:1]]).scatter(0, at.flatten(), s["table"].flatten())[:s["pages"]]
    take = (count + F - new.flatten().cumsum(0).view(new.shape)).clamp(0, s["pages"] - 1)
    table = torch.where(new, stack[take], s["table"])
    place = torch.arange(s["pages"], device=device)
    free = torch.where((place >= count) & (place < count + F - A), stack, s["free"])
    cu = torch.cat([torch.zeros(1, dtype=torch.int64, device=device), add.cumsum(0)])
    row = torch.arange(s["max_rows"], device=device)
    b = torch.searchsorted(cu[1:], row, right=True).clamp(max=s["B"] - 1)
    there = row < cu[-1]
    pos = torch.where(there, kept[b] + row - cu[b], 0)
    slots = torch.where(there, table[b, pos // P].long() * P + pos % P, -1)
    return {"kv_lens": lens.to(torch.int32), "cu_rows": cu.to(torch.int32), "positions": pos.to(torch.int32), "slots": slots,
            "free_count": (count + F - A).to(torch.int32), "table": table, "free": free}


def _rotate(x, c, s, rot, interleaved):
    x = x.float()
    if interleaved:
        a, b = x[..., :rot:2], x[..., 1:rot:2]
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
    a, b = a * c - b * s, b * c + a * s
    turned = torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1)
    return torch.cat([turned, x[..., rot:]], -1)


def _plain_rope(s):
    dt = TYPES[s["x"]]
    pos = s["positions"].view(-1, s["T"])
    pos = pos[s["pair_axis"].long()].t() if s["pair_axis"] is not None else pos[0][:, None]
    angle = pos.double() * s["inv_freq"].double()          # [T, pairs]
    c, n = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    Q = _rotate(s["Q"], c, n, s["rot"], s["interleaved"]).clamp(-LARGEST[dt], LARGEST[dt]).to(dt)
    page, place = s["slots"] // s["P"], s["slots"] % s["P"]
    _store(s, page, place, *_encode(_rotate(s["K"], c, n, s["rot"], s["interleaved"])), *_encode(s["V"].float()))
    return {"Q": Q, **_plain_read(s)}


def _plain_read(s):
    dt = TYPES[s["x"]]
    kc, kw, vc, vw = _stored(s, s["table"][s["seq"], s["pos"] // s["P"]].long(), s["pos"] % s["P"])
    return {"K": _decode(kc, kw).clamp(-LARGEST[dt], LARGEST[dt]).to(dt), "V": _decode(vc, vw).clamp(-LARGEST[dt], LARGEST[dt]).to(dt)}


def _plain_accept(s):
    P, table = s["P"], s["table"]
    page, place = table[s["seq"], s["pos"] // P].long(), s["pos"] % P
    _store(s, page, place, *_encode(s["K"].float()), *_encode(s["V"].float()))
    base = s["kv_lens"].long() - torch.tensor(s["rows"], device="cuda")
    i = torch.arange(s["accepted"].shape[1], device="cuda")
    b, i = (i < s["accept_lens"][:, None]).nonzero(as_tuple=True)
    src, dst = base[b] + s["accepted"][b, i], base[b] + i
    _store(s, table[b, dst // P].long(), dst % P, *_stored(s, table[b, src // P].long(), src % P))
    return {"kv_lens": (base + s["accept_lens"]).to(torch.int32), **_plain_read(s)}


def _plain_attn(s):
    lens, H, P, w, dt = s["kv_lens"].long(), s["Hkv"], s["P"], s["window"], TYPES[s["o"]]
    B, n, G = s["B"], max(s["rows"]), s["Hq"] // s["Hkv"]
    counts = torch.tensor(s["rows"], device="cuda")
    base = lens - counts
    # the tokens that some row of a sequence sees: its sinks, then all from the first row's window on
    first = (base + 1 - w).clamp(min=0) if w else torch.zeros_like(lens)
    few = first.clamp(max=s["sinks"])
    S = max(1, max(min(s["sinks"], _first(m - r, w)) + m - _first(m - r, w) for m, r in zip(s["lens"], s["rows"])))
    at = torch.arange(S, device="cuda")
    key = torch.where(at < few[:, None], at, at - few[:, None] + first[:, None])               # [B, S]
    there = key < lens[:, None]
    key = torch.where(there, key, 0)
    kc, kw, vc, vw = _stored(s, s["table"].gather(1, key // P).long(), key % P)
    K, V = _decode(kc, kw).transpose(1, 2), _decode(vc, vw).transpose(1, 2)                    # [B, H, S, D]
    D = s["D"]
    Q = torch.zeros(B, n, H, G, D, device="cuda")
    Q[s["seq"], s["row_of"]] = s["Q"].float().unflatten(1, (H, G))
    pos = torch.full((B, n), -1, device="cuda")
    pos[s["seq"], s["row_of"]] = s["pos"]
    k = key[:, None]                                       # [B, 1, S]
    if s["op"] == "tree":
        bits = torch.zeros(B, n, 32 * s["mask"].shape[1], dtype=torch.bool, device="cuda")
        bits[s["seq"], s["row_of"]] = ((s["mask"][..., None] >> torch.arange(32, device="cuda")) & 1).flatten(1).bool()
        drafted = bits.gather(2, (k - base[:, None, None]).clamp(0, bits.shape[2] - 1).expand(B, n, S)) & (k >= base[:, None, None])
        depth = base[:, None] + bits.sum(-1) - 1
        seen = (k < base[:, None, None]) & (pos >= 0)[..., None]
        if w:
            seen = seen & ((k > depth[..., None] - w) | (k < s["sinks"]))
        seen = seen | drafted
    else:
        seen = (k <= pos[..., None]) & ((k > pos[..., None] - w) | (k < s["sinks"]))
    seen = seen & there[:, None]
    score = (Q.permute(0, 2, 1, 3, 4).flatten(2, 3) @ K.transpose(-1, -2)).mul_(s["scale"]).unflatten(2, (n, G))
    score.masked_fill_(~seen[:, None, :, None], -math.inf)
    top = score.amax(-1, keepdim=True).clamp(min=-3e38)
    p = score.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = (p.flatten(2, 3) @ V).unflatten(2, (n, G)) / torch.where(total > 0, total, torch.ones_like(total))
    o = o.permute(0, 2, 1, 3, 4).flatten(2, 3)[s["seq"], s["row_of"]]
    return o.clamp(-LARGEST[dt], LARGEST[dt]).to(dt)


# ---------------------------------------------------------------------------- the framework's calls
def _workspace(w4a8, s):
    """What a serving program allocates once for its largest batch."""
    if "ws" not in s:
        if s["op"] == "plan":
            s["ws"] = w4a8.new_kv_workspace(1, 1, 1, 1, 64)
        else:
            s["ws"] = w4a8.new_kv_workspace(s["T"], s["B"], s.get("Hq", s["Hkv"]), s["Hkv"], s["D"])
    return s["ws"]


def run(s):
    if own:
        import paper_2311_05161_b200 as w4a8
        ws = _workspace(w4a8, s)
        if s["op"] == "plan":
            lens, cu, pos, slots, count = w4a8.kv_plan(s["held"], s["kept"], s["add"], s["table"], s["free"], s["count"], s["P"], s["max_rows"], ws, out=s["out"])
            return {"kv_lens": lens, "cu_rows": cu, "positions": pos, "slots": slots, "free_count": count, "table": s["table"], "free": s["free"]}
        if s["op"] == "sinks":
            return w4a8.kv_attention_sinks(s["Q"], s["cache"], s["table"], s["kv_lens"], s["Hkv"], ws, s["window"], s["sinks"], cu_rows=s["cu"],
                                           scale=s["scale"], dtype=TYPES[s["o"]])
        if s["op"] == "tree":
            return w4a8.kv_attention_tree(s["Q"], s["cache"], s["table"], s["kv_lens"], s["Hkv"], ws, s["mask"], cu_rows=s["cu"], scale=s["scale"],
                                          window=s["window"], sinks=s["sinks"], dtype=TYPES[s["o"]])
        out = {}
        if s["op"] == "rope":
            out["Q"] = w4a8.rope_kv_append(s["Q"], s["K"], s["V"], s["positions"], s["inv_freq"], s["cache"], s["slots"], ws, pair_axis=s["pair_axis"],
                                           interleaved=s["interleaved"])
        else:
            w4a8.kv_append(s["K"], s["V"], s["cache"], s["table"], s["kv_lens"], ws, cu_rows=s["cu"])
            out["kv_lens"] = w4a8.kv_accept(s["cache"], s["table"], s["kv_lens"], s["accepted"], s["accept_lens"], s["Hkv"], s["D"], ws, cu_rows=s["cu"])
        out["K"], out["V"] = w4a8.kv_read(s["cache"], s["table"], s["kv_lens"], s["T"], s["Hkv"], s["D"], ws, cu_rows=s["cu"], dtype=TYPES[s["x"]])
        return out
    return {"plan": _plain_plan, "rope": _plain_rope, "sinks": _plain_attn, "tree": _plain_attn, "accept": _plain_accept}[s["op"]](s)


# ---------------------------------------------------------------------------- from the definitions, in 64 bits
def _levels():
    """Value of every rank for every zero-point, in steps: the sixteen levels of Eq. 6 in order."""
    return torch.tensor([sorted([k - z for k in range(14)] + [0.5, -0.5]) for z in range(14)], dtype=F64, device="cuda")


def _exact_cached(s, b, pages):
    """Keys and values [n, H, D] of the tokens on some pages of sequence b, from the bytes of their blocks."""
    H, D, P = s["Hkv"], s["D"], s["P"]
    raw = s["cache"][s["table"][b, pages].long()].view(-1, H, P // 16, 16 * D + 128).transpose(0, 1).reshape(H, -1, 16 * D + 128)
    word = raw[..., 16 * D:].contiguous().view(torch.int32).view(H, -1, 2, 16)
    found = []
    for which in (0, 1):
        code = raw[..., 8 * D * which:8 * D * (which + 1)]
        if which:
            code = code.reshape(H, -1, 2, 8, 8, D // 16).permute(0, 1, 2, 4, 3, 5)
        code = code.reshape(H, -1, D // 4, 2).long()
        h = code[..., 0] + 256 * code[..., 1]
        h = h // 4 + (h % 4) * 16384                       # undo the rotation
        rank = torch.stack([h // 16 ** k % 16 for k in range(4)], -1).flatten(-2)
        w = word[:, :, which].reshape(H, -1)
        value = _levels()[(w % 16).long().clamp(max=13)].gather(-1, rank) * (w - w % 16).view(F32).double()[..., None]
        found.append(value.transpose(0, 1))
    return found


def _exact_quantized(x):
    """Eq. 5 on the vectors of x [..., D] in 64 bits; the step is kept to 20 significant bits."""
    x = x.double()
    lo, hi = x.amin(-1, keepdim=True).clamp(max=0), x.amax(-1, keepdim=True).clamp(min=0)
    m, e = torch.frexp((hi - lo) / 13)
    step = torch.ldexp(torch.floor(m * 2.0 ** 20 + 0.5) / 2.0 ** 20, e)
    step = torch.where(hi - lo < 13 * 2.0 ** -100, torch.ones_like(step), step)
    z = torch.round(-lo / step).clamp(0, 13)
    u = x / step
    plain = (torch.round(u) + z).clamp(0, 13) - z
    return torch.where((u.abs() > 0.25) & (u.abs() <= 0.75), 0.5 * torch.sign(u), plain) * step


def _exact_turned(x, s):
    """Pairs of elements as complex numbers, turned by their angle."""
    x, rot = x.double(), s["rot"]
    i = torch.arange(rot // 2, device="cuda")
    a, b = (2 * i, 2 * i + 1) if s["interleaved"] else (i, i + rot // 2)
    axis = torch.zeros_like(i) if s["pair_axis"] is None else s["pair_axis"].long()
    pos = s["positions"].view(-1, s["T"]).double()
    angle = torch.stack([pos[axis[k]] * s["inv_freq"][k].double() for k in range(rot // 2)], 1)
    z = torch.complex(x[..., a], x[..., b]) * torch.polar(torch.ones_like(angle), angle)[:, None]
    y = x.clone()
    y[..., a], y[..., b] = z.real, z.imag
    return y


def exact(c, seed):
    if c["op"] == "plan":
        return None
    s = prepare(c, seed)
    if c["op"] == "rope":
        return {"Q": _exact_turned(s["Q"], s), "K": _exact_quantized(_exact_turned(s["K"], s)), "V": _exact_quantized(s["V"])}
    if c["op"] == "accept":
        order, at = [], 0
        for r, path in zip(s["rows"], s["paths"]):
            order += [at + j for j in path] + [at + j for j in range(len(path), r)]
            at += r
        order = torch.tensor(order, device="cuda")
        return {"kv_lens": None, "K": _exact_quantized(s["K"])[order], "V": _exact_quantized(s["V"])[order]}
    out, at, P, w, G = [], 0, s["P"], c["window"], c["Hq"] // c["Hkv"]
    for b in range(c["B"]):
        r, n = s["rows"][b], s["lens"][b]
        base = n - r
        low = _first(max(base, 0), w)
        few = min(c["sinks"], n)
        pages = sorted(set(range(-(-few // P))) | set(range(low // P, -(-n // P))))
        K, V = _exact_cached(s, b, torch.tensor(pages, dtype=torch.long, device="cuda"))
        key = torch.tensor([p * P + k for p in pages for k in range(P)], dtype=torch.long, device="cuda")
        q = s["Q"][at:at + r].double()
        at += r
        seen = torch.zeros(r, len(key), dtype=torch.bool, device="cuda")
        for i in range(r):
            if base + i < 0:
                continue
            if c["op"] == "tree":
                mine, j = [], i
                while j >= 0:
                    mine.append(j)
                    j = s["parents"][b][j]
                p = base + len(mine) - 1
                seen[i] = (key < base) & (((key > p - w) | (key < c["sinks"])) if w else True)
                seen[i] |= torch.isin(key, base + torch.tensor(mine, device="cuda"))
            else:
                seen[i] = (key <= base + i) & ((key > base + i - w) | (key < c["sinks"]))
        heads = []
        for h in range(c["Hkv"]):
            score = torch.einsum("rgd,nd->rgn", q[:, h * G:(h + 1) * G], K[:, h]) * s["scale"]
            score = score.masked_fill(~seen[:, None], -math.inf)
            p = torch.exp(score - torch.logsumexp(score, -1, keepdim=True).clamp(min=-1e300))
            heads.append(torch.einsum("rgn,nd->rgd", p, V[:, h]))
        out.append(torch.cat(heads, 1))
    return torch.cat(out)
