"""Operators of a quantized decoder step around the W4A8 linear layers, with their plain forms.

Four operators, in the order in which a serving step meets them:

  norm    residual addition, RMSNorm / LayerNorm and the token-wise INT8 quantizer in one pass
          (add_norm_quantize_act)
  write   new keys and values quantized to dINT4 as they enter a paged cache, and read back
          (kv_append, kv_read)
  read    a stretch of the cache read back as 16-bit keys and values (kv_read)
  attn    attention of new tokens over the 4-bit cache (kv_attention)

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

import torch

own = False

F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
TYPES = {"f16": F16, "bf16": BF16, "f32": F32}
LARGEST = {F16: 65504.0, BF16: 3.3895313892515355e38}


# ---------------------------------------------------------------------------- the cases
def listed():
    return [
        # one new token of a 4096-wide decoder layer, between the attention and the feed-forward block
        dict(name="norm, one token, 4096", op="norm", M=1, K=4096, kind="rms", bias=False, x="bf16", res="f16"),
        # a prompt's tokens in a 9216-wide layer with LayerNorm and a 32-bit residual stream
        dict(name="norm, 2048 tokens, 9216", op="norm", M=2048, K=9216, kind="layer", bias=True, x="bf16", res="f32"),
        # an odd number of tokens of several requests batched together
        dict(name="norm, 777 tokens, 5120", op="norm", M=777, K=5120, kind="rms", bias=False, x="f16", res="f16"),
        # a decode step of eight requests: one token each enters the cache
        dict(name="write, 8 x 1 token, 32 heads", op="write", B=8, lo=1, hi=1900, rows_lo=1, rows_hi=1, Hkv=32, D=128, P=64, x="bf16", fused=True),
        # prompts of four requests, of different lengths, enter the cache
        dict(name="write, 4 prompts, 8 heads", op="write", B=4, lo=611, hi=4097, rows_lo=611, rows_hi=4097, Hkv=8, D=128, P=64, x="f16", fused=False),
        # a short shared prefix is read back
        dict(name="read, 300 tokens, 8 heads", op="read", B=1, lo=300, hi=300, rows_lo=300, rows_hi=300, Hkv=8, D=128, P=16, x="f16"),
        # whole sequences leave the cache in 16 bits, to be moved to another engine
        dict(name="read, 16 sequences, 8 heads", op="read", B=16, lo=1500, hi=4096, rows_lo=1500, rows_hi=4096, Hkv=8, D=128, P=64, x="bf16"),
        # one request with a short history: latency
        dict(name="attn, 1 x 513", op="attn", B=1, lo=513, hi=513, rows_lo=1, rows_hi=1, Hq=32, Hkv=8, D=128, P=64, x="bf16", o="f16", window=0),
        # 32 requests without shared heads, of very different lengths, one of them still empty
        dict(name="attn, 32 ragged, 32 heads", op="attn", B=32, lo=0, hi=2047, rows_lo=1, rows_hi=1, Hq=32, Hkv=32, D=128, P=64, x="bf16", o="f16", window=0),
        # one request with a very long history
        dict(name="attn, 1 x 131001", op="attn", B=1, lo=131001, hi=131001, rows_lo=1, rows_hi=1, Hq=32, Hkv=8, D=128, P=64, x="f16", o="f16", window=0),
        # a full serving batch with eight query heads to a key head
        dict(name="attn, 64 ragged, 64/8 heads", op="attn", B=64, lo=1000, hi=6000, rows_lo=1, rows_hi=1, Hq=64, Hkv=8, D=128, P=64, x="bf16", o="bf16", window=0),
        # a chunk of a long prompt attends to what is cached before it and to itself
        dict(name="attn, chunk of 1024 at 4096", op="attn", B=1, lo=4096, hi=4096, rows_lo=1024, rows_hi=1024, Hq=32, Hkv=8, D=128, P=64, x="bf16", o="f16", window=0),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["norm", "norm", "write", "read", "attn", "attn", "attn"])
    if op == "norm":
        K = 128 * log(1, 128)
        return dict(op=op, M=min(log(1, 4096), 18_000_000 // K), K=K, kind=rng.choice(["rms", "layer"]), bias=rng.random() < 0.5,
                    x=rng.choice(["f16", "bf16"]), res=rng.choice(["f16", "bf16", "f32"]))
    D, P, x = rng.choice([64, 128, 128]), rng.choice([16, 32, 64, 128]), rng.choice(["f16", "bf16"])
    Hkv = rng.choice([1, 2, 4, 8, 12, 32])
    if op in ("write", "read"):
        B, lo = log(1, 32), rng.choice([0, 1, 17])
        hi = lo + log(1, max(2, min(4096, (400_000 if op == "read" else 90_000) // (B * Hkv))))
        rows_hi = rng.choice([1, hi, max(1, hi // 3)])
        return dict(op=op, B=B, lo=lo, hi=hi, rows_lo=min(rows_hi, rng.choice([0, 1, rows_hi])), rows_hi=rows_hi, Hkv=Hkv, D=D, P=P, x=x,
                    **({"fused": rng.random() < 0.5} if op == "write" else {}))
    G, B = rng.choice([1, 2, 4, 5, 7, 8, 16]), log(1, 64)
    hi = log(1, max(2, min(100_000, 1_600_000 // (B * Hkv))))
    rows_hi = rng.choice([1, 1, 1, 1, 2, 4, min(hi, max(1, 600 // B))])
    while rows_hi > 1 and B * rows_hi * Hkv * G * hi > 100_000_000:
        rows_hi //= 2
    return dict(op=op, B=B, lo=rng.choice([0, 1, hi // 2, hi]), hi=hi, rows_lo=rng.choice([0, rows_hi]) if rows_hi > 1 else 1, rows_hi=rows_hi,
                Hq=Hkv * G, Hkv=Hkv, D=D, P=P, x=x, o=rng.choice(["f16", "bf16"]), window=rng.choice([0, 0, 0, 1 + hi // 3]))


def _spread(n, lo, hi, salt):
    """n whole numbers from lo to hi, both among them: the case alone gives them."""
    got = [lo + (b * 2654435761 + salt * 40503 + 12345) % 1000003 % (hi - lo + 1) for b in range(n)]
    got[0] = hi
    if n > 1:
        got[n // 2] = lo
    return got


def _lengths(c):
    lens = _spread(c["B"], c["lo"], c["hi"], 1)
    rows = lens if (c["rows_lo"], c["rows_hi"]) == (c["lo"], c["hi"]) else _spread(c["B"], c["rows_lo"], c["rows_hi"], 2)
    return lens, list(rows)


def _visible(n, r, window):
    """Keys that the r last positions of n see, all together; a row in front of position 0 sees none."""
    total = 0
    for p in range(max(0, n - r), n):
        total += min(p + 1, window) if window else p + 1
    return total


def work(c):
    if c["op"] == "norm":
        e = c["M"] * c["K"]
        size = {"f16": 2, "bf16": 2, "f32": 4}
        return {"bytes": e * (size[c["x"]] + 2 * size[c["res"]] + 1) + c["K"] * (8 if c["bias"] else 4) + 4 * c["M"], "flops": 10 * e}
    lens, rows = _lengths(c)
    vec = c["D"] // 2 + 4                      # bytes of a cached vector: codes and one word
    if c["op"] in ("write", "read"):
        n = sum(rows) * c["Hkv"] * 2           # vectors
        moved = n * (2 * c["D"] + vec) if c["op"] == "read" else n * (4 * c["D"] + 2 * vec)
        return {"bytes": moved, "flops": 8 * n * c["D"]}
    w = c["window"]
    keys = sum(min(n, r + w - 1 if w else n) for n, r in zip(lens, rows) if r)
    pairs = sum(_visible(n, r, w) for n, r in zip(lens, rows))
    return {"bytes": keys * c["Hkv"] * 2 * vec + sum(rows) * c["Hq"] * c["D"] * 4 + 4 * sum(-(-n // c["P"]) for n in lens),
            "flops": 4 * pairs * c["Hq"] * c["D"]}


# ---------------------------------------------------------------------------- inputs
def _vectors(shape, g, spread):
    """Key- or value-like vectors: some channels are larger and off centre, tokens differ in size."""
    heads, D = shape[-2:]
    gain = torch.exp(0.6 * torch.randn(heads, D, generator=g, device="cuda"))
    shift = 0.4 * torch.randn(heads, D, generator=g, device="cuda")
    size = torch.exp(0.3 * torch.randn(shape[:-1] + (1,), generator=g, device="cuda"))
    x = torch.randn(shape, generator=g, device="cuda").mul_(gain).add_(shift)
    return x.mul_(size).mul_(spread)


def prepare(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(c)
    if c["op"] == "norm":
        M, K = c["M"], c["K"]
        loud = 1.0 + 19.0 * (torch.rand(K, generator=g, device="cuda") < 0.01)
        s["X"] = torch.randn(M, K, generator=g, device="cuda").to(TYPES[c["x"]])
        s["residual"] = (torch.randn(M, K, generator=g, device="cuda") * loud + 0.25).to(TYPES[c["res"]])
        s["weight"] = torch.exp(0.7 * torch.randn(K, generator=g, device="cuda")) / loud
        s["norm_bias"] = 0.1 * torch.randn(K, generator=g, device="cuda") / loud if c["bias"] else None
        s["eps"] = 1e-5
        return s
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
    # for the plain forms: sequence and position of every row
    seq = torch.repeat_interleave(torch.arange(B), torch.tensor(rows)).cuda()
    s["seq"] = seq
    s["row_of"] = torch.arange(s["T"], device="cuda") - torch.tensor(cu, device="cuda")[seq]
    s["pos"] = s["kv_lens"][seq].long() - torch.tensor(rows, device="cuda")[seq] + s["row_of"]
    block = 16 * D + 128
    if c["op"] == "write":
        s["cache"] = torch.zeros(pages, H * (P // 16) * block, dtype=torch.uint8, device="cuda")
        K, V = _vectors((s["T"], H, D), g, 1.5).to(TYPES[c["x"]]), _vectors((s["T"], H, D), g, 0.7).to(TYPES[c["x"]])
        if c["fused"]:                         # slices of one wider projection output
            wide = torch.cat([torch.zeros_like(K), K, V], 1)
            K, V = wide[:, H:2 * H], wide[:, 2 * H:]
        s["K"], s["V"] = K, V
        return s
    # a filled cache, page by page
    K, V = _vectors((pages, H, P // 16, 16, D), g, 1.5), None
    kc, km = _encode(K.to(TYPES[c["x"]]).float())
    V = _vectors((pages, H, P // 16, 16, D), g, 0.7)
    vc, vm = _encode(V.to(TYPES[c["x"]]).float())
    s["cache"] = torch.cat([kc.flatten(3), _v_order(vc).flatten(3), km.view(torch.uint8).flatten(3), vm.view(torch.uint8).flatten(3)], 3).reshape(pages, -1).contiguous()
    if c["op"] == "attn":
        s["Q"] = (1.3 * torch.randn(s["T"], c["Hq"], D, generator=g, device="cuda")).to(TYPES[c["x"]])
        s["scale"] = 1.0 / math.sqrt(D)
    return s


# ---------------------------------------------------------------------------- the cache format
def _encode(x):
    """x [..., D] binary32 -> codes [..., D/2] uint8 (keys' order) and words [...] int32."""
    one = torch.ones((), device=x.device)
    lo, hi = x.amin(-1, keepdim=True).clamp(max=0.0), x.amax(-1, keepdim=True).clamp(min=0.0)
    raw = (hi * 0.5 - lo * 0.5) / (one * 6.5)
    step = ((raw.view(torch.int32) + 8) & ~15).view(F32)
    step = torch.where(raw < 2.0 ** -100, one, step)
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


def _gather(s):
    """Keys and values of all sequences, padded: [B, Hkv, most * P, D] binary32 each."""
    D, P, H = s["D"], s["P"], s["Hkv"]
    blocks = s["cache"].view(-1, H, P // 16, 16 * D + 128)[s["table"].long()]
    kc = blocks[..., :8 * D].unflatten(-1, (16, D // 2))
    vc = blocks[..., 8 * D:16 * D].unflatten(-1, (2, 8, 8, D // 16)).transpose(-3, -2).flatten(-2).flatten(-3, -2)
    word = blocks[..., 16 * D:].contiguous().view(torch.int32).unflatten(-1, (2, 16))
    return [_decode(codes, w).permute(0, 2, 1, 3, 4, 5).flatten(2, 4) for codes, w in ((kc, word[..., 0, :]), (vc, word[..., 1, :]))]


# ---------------------------------------------------------------------------- plain forms
def _plain_norm(s):
    f64, one = torch.float64, torch.ones((), device="cuda")
    y = (s["X"].float() + s["residual"].float()).to(TYPES[s["res"]])
    x = y.float()
    if s["kind"] == "layer":
        x = x - x.to(f64).mean(-1, keepdim=True).to(F32)
    eps = torch.tensor(s["eps"], dtype=F32).to(f64).item()
    r = (1.0 / torch.sqrt(x.to(f64).square().mean(-1, keepdim=True) + eps)).to(F32)
    x = (x * r) * s["weight"]
    if s["norm_bias"] is not None:
        x = x + s["norm_bias"]
    amax = x.abs().amax(-1, keepdim=True)
    q = torch.round((x * ((one * 127.0) / amax)).clamp(-127.0, 127.0))
    q = torch.where(amax > 0, q, torch.zeros_like(q)).to(torch.int8)
    return {"Xq": q, "tok_scale": (amax / (one * 127.0)).squeeze(-1), "residual": y}


def _plain_write(s):
    H, D, P = s["Hkv"], s["D"], s["P"]
    flat, block = s["cache"].view(-1), 16 * D + 128
    t = (s["pos"] >= 0).nonzero().squeeze(-1)
    pos, seq = s["pos"][t], s["seq"][t]
    page = s["table"][seq, pos // P].long()
    base = ((page[:, None] * H + torch.arange(H, device="cuda")) * (P // 16) + (pos % P // 16)[:, None]) * block  # [T, H]
    slot = (pos % 16)[:, None]
    four, byte, c = torch.arange(4, device="cuda"), torch.arange(D // 2, device="cuda"), D // 16
    for_v = ((slot // 8)[..., None] * 8 + byte // c) * 8 * c + (slot % 8)[..., None] * c + byte % c
    for x, off, at, word_at in ((s["K"], 0, slot[..., None] * (D // 2) + byte, 0), (s["V"], 8 * D, for_v, 64)):
        codes, word = _encode(x[t].float())
        flat[(base[..., None] + off + at).flatten()] = codes.flatten()
        flat[(base[..., None] + 16 * D + word_at + 4 * slot[..., None] + four).flatten()] = word.unsqueeze(-1).view(torch.uint8).flatten()
    return _plain_read(s)


def _plain_read(s):
    H, D, P, dt = s["Hkv"], s["D"], s["P"], TYPES[s["x"]]
    pos = s["pos"].clamp(min=0)
    page, block, slot = s["table"][s["seq"], pos // P].long(), pos % P // 16, pos % 16
    blocks = s["cache"].view(-1, H, P // 16, 16 * D + 128)
    word = s["cache"].view(torch.int32).view(-1, H, P // 16, 4 * D + 32)[..., 4 * D:].unflatten(-1, (2, 16))
    kc = blocks[..., :8 * D].unflatten(-1, (16, D // 2))[page, :, block, slot]
    vc = blocks[..., 8 * D:16 * D].unflatten(-1, (2, 8, 8, D // 16)).transpose(-3, -2)[page, :, block, slot // 8, slot % 8].flatten(-2)
    got = []
    for which, codes in enumerate((kc, vc)):
        x = _decode(codes, word[page, :, block, which, slot])
        x = torch.where((s["pos"] >= 0)[:, None, None], x, torch.zeros_like(x))
        got.append(x.clamp(-LARGEST[dt], LARGEST[dt]).to(dt))
    return {"K": got[0], "V": got[1]}


def _plain_attn(s):
    K, V = _gather(s)
    B, H, S, D = K.shape
    n, G, dt = max(s["rows"]), s["Hq"] // s["Hkv"], TYPES[s["o"]]
    Q = torch.zeros(B, n, H, G, D, device="cuda")
    Q[s["seq"], s["row_of"]] = s["Q"].float().unflatten(1, (H, G))
    pos = torch.full((B, n), -1, device="cuda")
    pos[s["seq"], s["row_of"]] = s["pos"]
    score = (Q.permute(0, 2, 1, 3, 4).flatten(2, 3) @ K.transpose(-1, -2)).mul_(s["scale"]).unflatten(2, (n, G))
    key = torch.arange(S, device="cuda")
    seen = key <= pos[..., None]
    if s["window"]:
        seen &= key > pos[..., None] - s["window"]
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
        s["ws"] = w4a8.new_kv_workspace(s["T"], s["B"], s.get("Hq", s["Hkv"]), s["Hkv"], s["D"])
    return s["ws"]


def run(s):
    if own:
        import paper_2311_05161_b200 as w4a8
        if s["op"] == "norm":
            kind = w4a8.NORM_LAYER if s["kind"] == "layer" else w4a8.NORM_RMS
            Xq, tok, res = w4a8.add_norm_quantize_act(s["X"], s["residual"], s["weight"], s["norm_bias"], kind, s["eps"])
            return {"Xq": Xq, "tok_scale": tok, "residual": res}
        ws = _workspace(w4a8, s)
        if s["op"] == "attn":
            return w4a8.kv_attention(s["Q"], s["cache"], s["table"], s["kv_lens"], s["Hkv"], ws, cu_rows=s["cu"],
                                     scale=s["scale"], causal=True, window=s["window"], dtype=TYPES[s["o"]])
        if s["op"] == "write":
            w4a8.kv_append(s["K"], s["V"], s["cache"], s["table"], s["kv_lens"], ws, cu_rows=s["cu"])
        K, V = w4a8.kv_read(s["cache"], s["table"], s["kv_lens"], s["T"], s["Hkv"], s["D"], ws, cu_rows=s["cu"], dtype=TYPES[s["x"]])
        return {"K": K, "V": V}
    return {"norm": _plain_norm, "write": _plain_write, "read": _plain_read, "attn": _plain_attn}[s["op"]](s)


# ---------------------------------------------------------------------------- from the definitions, in 64 bits
def _levels():
    """Value of every rank for every zero-point, in steps: the sixteen levels of Eq. 6 in order."""
    return torch.tensor([sorted([k - z for k in range(14)] + [0.5, -0.5]) for z in range(14)], dtype=torch.float64, device="cuda")


def _exact_cached(s, b):
    """Keys and values [n, H, D] of sequence b from the bytes of its blocks."""
    H, D, P, n = s["Hkv"], s["D"], s["P"], s["lens"][b]
    pages = s["table"][b, :max(1, -(-n // P))].long()
    raw = s["cache"][pages].view(-1, H, P // 16, 16 * D + 128).transpose(0, 1).reshape(H, -1, 16 * D + 128)
    word = raw[..., 16 * D:].contiguous().view(torch.int32).view(H, -1, 2, 16)
    found = []
    for which in (0, 1):
        code = raw[..., 8 * D * which:8 * D * (which + 1)]
        if which:
            code = code.reshape(H, -1, 2, 8, 8, D // 16).permute(0, 1, 2, 4, 3, 5)
        code = code.reshape(H, -1, D // 4, 2).long()
        h = code[..., 0] + 256 * code[..., 1]
        h = h // 4 + (h % 4) * 16384                       # undo the rotation
        rank = torch.stack([h // 16 ** k % 16 for k in range(4)], -1).flatten(-2)[:, :n]
        w = word[:, :, which].reshape(H, -1)[:, :n]
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


def exact(c, seed):
    s = prepare(c, seed)
    if c["op"] == "norm":
        y = s["X"].double() + s["residual"].double()
        x = y.to(F32).to(TYPES[c["res"]]).double()         # the norm is that of the stored residual
        if c["kind"] == "layer":
            x = x - x.sum(-1, keepdim=True) / c["K"]
        x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / c["K"] + s["eps"]) * s["weight"].double()
        if s["norm_bias"] is not None:
            x = x + s["norm_bias"].double()
        return {"Xq": None, "tok_scale": x.abs().amax(-1) / 127, "residual": y}
    if c["op"] == "write":
        there = (s["pos"] >= 0)[:, None, None]
        return {k: torch.where(there, _exact_quantized(s[k]), 0.0) for k in ("K", "V")}
    keys, values, out = [], [], []
    at = 0
    for b in range(c["B"]):
        r, n = s["rows"][b], s["lens"][b]
        K, V = _exact_cached(s, b)
        if c["op"] == "read":
            lost = torch.zeros(max(0, r - n), c["Hkv"], c["D"], dtype=torch.float64, device="cuda")
            keys.append(torch.cat([lost, K[max(0, n - r):n]])[:r])
            values.append(torch.cat([lost, V[max(0, n - r):n]])[:r])
            continue
        q = s["Q"][at:at + r].double()
        at += r
        pos = torch.arange(n - r, n, device="cuda")
        key = torch.arange(n, device="cuda")
        seen = (key[None] <= pos[:, None]) & ((key[None] > pos[:, None] - c["window"]) if c["window"] else True)
        for h in range(c["Hkv"]):
            G = c["Hq"] // c["Hkv"]
            score = torch.einsum("rgd,nd->rgn", q[:, h * G:(h + 1) * G], K[:, h]) * s["scale"]
            score = score.masked_fill(~seen[:, None], -math.inf)
            p = torch.exp(score - torch.logsumexp(score, -1, keepdim=True).clamp(min=-1e300))
            keys.append(torch.einsum("rgn,nd->rgd", p, V[:, h]))
        out.append(torch.cat(keys, 1) if r else torch.zeros(0, c["Hq"], c["D"], dtype=torch.float64, device="cuda"))
        keys = []
    if c["op"] == "read":
        return {"K": torch.cat(keys), "V": torch.cat(values)}
    return torch.cat(out)
