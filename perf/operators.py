"""Cases for the operators of one serving step over many requests: a paged KV4 cache (written, read back, kept after a
drafted tree was checked), the attention of drafted token trees over it, and the low-rank adapters beside a shared
projection.

The cache is a pool of pages, uint8 [pages, Hkv, page_tokens / 32 * 4416].  32 tokens of one KV head are a block of 4416
bytes: key codes at 0, value codes at 2048 (64 bytes a token each), fp32 key scales at 4096 and value scales at 4224,
one byte a token of key zero-points at 4352 and of value zero-points at 4384.  Every byte belongs to one token.  A
value is scale * (code - zero).  Requests are ragged: row_start [R + 1] cuts the rows of a call, first [R] is the cache
position of a request's first row, page_table [R, max_pages] names its pages.
"""
import math
import random

import numpy as np
import torch

own = False

D = 128
BLOCK, TOKENS = 4416, 32
CLIP = 0.95
LLAMA2_HEADS, LLAMA3_HEADS = (32, 32), (32, 8)  # query and KV heads of the two models that this repository measures


# ---------------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # 48 requests decode one token each: the smallest cache write, bound by the calls themselves
        dict(name="pages-decode-48x1", op="pages", requests=48, rows=1, ragged=False, context=4000, Hkv=8, dtype="bf16", page=64, lens=1),
        # a few long prompts enter the cache, eight KV heads
        dict(name="pages-prompts-6x3000", op="pages", requests=6, rows=3000, ragged=True, context=0, Hkv=8, dtype="bf16", page=64, lens=2),
        # the cached history of some requests is read back in fp32, 32 KV heads, pages of 32 tokens
        dict(name="history-5x900-f32", op="history", requests=5, rows=900, ragged=True, context=77, Hkv=32, dtype="f32", page=32, lens=3),
        # drafts of a few requests are written, the accepted path is kept
        dict(name="verify-4x12", op="verify", requests=4, rows=12, ragged=True, context=513, Hkv=8, dtype="bf16", page=64, lens=4),
        # the same for a large batch with the widest trees, fp32 rows
        dict(name="verify-192x64-f32", op="verify", requests=192, rows=64, ragged=True, context=2000, Hkv=8, dtype="f32", page=128, lens=5),
        # one request decodes one token in fp32 over a short cache: latency
        dict(name="attend-1x1-f32", op="attention", requests=1, rows=1, ragged=False, context=1023, Hq=32, Hkv=32, dtype="f32", page=64, tree=False, lens=6),
        # a batch of ragged requests decodes one token each
        dict(name="attend-64x1", op="attention", requests=64, rows=1, ragged=False, context=8000, Hq=32, Hkv=8, dtype="bf16", page=64, tree=False, lens=7),
        # small trees of a batch of requests
        dict(name="attend-tree-16x13", op="attention", requests=16, rows=13, ragged=True, context=6000, Hq=32, Hkv=8, dtype="bf16", page=32, tree=True, lens=8),
        # the widest trees over long contexts
        dict(name="attend-tree-8x64", op="attention", requests=8, rows=64, ragged=False, context=32000, Hq=32, Hkv=8, dtype="bf16", page=64, tree=True, lens=9),
        # adapters of 40 requests that decode one token each beside a square projection
        dict(name="lora-decode-40x1", op="lora", requests=40, rows=1, ragged=False, adapters=40, rank=16, K=4096, N=4096, dtype="bf16", lens=10),
        # fp32 rows of a few short requests, a narrow projection, odd rank
        dict(name="lora-7x11-f32", op="lora", requests=7, rows=11, ragged=True, adapters=4, rank=24, K=4096, N=1024, dtype="f32", lens=11),
        # adapters of a few prompts beside the widest projection
        dict(name="lora-prompts-5x800", op="lora", requests=5, rows=800, ragged=True, adapters=8, rank=64, K=4096, N=14336, dtype="bf16", lens=12),
    ]


def draw(rng):
    def log(lo, hi):
        return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    op = rng.choice(["pages", "history", "verify", "attention", "attention", "attention", "lora", "lora"])
    c = dict(op=op, ragged=rng.random() < 0.7, dtype=rng.choice(["bf16", "bf16", "f32"]), lens=rng.randrange(1 << 30))
    if op == "lora":
        c |= dict(requests=log(1, 64), adapters=log(1, 48), rank=8 * rng.randint(1, 16),
                  K=rng.choice([1024, 4096, 4096, 11008]), N=8 * log(64, 1792))
        c["rows"] = log(1, max(1, min(1500, 4000 // c["requests"], 230_000_000 // (c["adapters"] * c["rank"] * (c["K"] + c["N"]) // 8))))
        return c
    c |= dict(Hkv=rng.choice([8, 8, 32]), page=rng.choice([32, 64, 128]))
    if op in ("pages", "history"):
        c["requests"] = log(1, 96)
        c["rows"] = log(1, max(1, min(3000, 144_000 // (c["Hkv"] * c["requests"]))))
        c["context"] = rng.choice([0, log(1, 4000)])
        return c
    c["requests"], c["rows"] = log(1, 192 if op == "verify" else 96), log(1, 64)
    if op == "verify":
        if c["Hkv"] == 32:
            c["requests"] = min(c["requests"], 48)
        c["context"] = log(1, 4000)
        return c
    c |= dict(Hq=rng.choice([32, 32, 2 * c["Hkv"]]), tree=rng.random() < 0.7)
    most = 8 * 32000 * 8 // (c["Hkv"] * c["requests"])  # cached tokens of a request: the largest listed cache in all
    most = min(most, 8 * 64 * 32000 // (c["requests"] * c["rows"]) * 32 // max(c["Hq"], c["Hkv"]) // 2, 32000)
    c["context"] = rng.choice([0, log(1, most), log(1, most), log(1, most)])
    return c


def _lengths(c):
    """Rows and cached tokens before them, request by request: from the case alone."""
    r = random.Random(c["lens"])
    rows = [r.randint(max(1, c["rows"] // 4), c["rows"]) if c["ragged"] else c["rows"] for _ in range(c["requests"])]
    most = c.get("context", 0)
    first = [r.randint(most // 8, most) if c["requests"] > 1 else most for _ in rows]
    if c["requests"] > 1:
        rows[-1], first[0] = c["rows"], most
    return rows, first


def work(c):
    rows, first = _lengths(c)
    total, size = sum(rows), 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "lora":
        r = random.Random(c["lens"] + 1)
        ids = [r.randrange(c["adapters"]) for _ in rows]
        w = len(set(ids)) * c["rank"] * (c["K"] + c["N"]) * 2
        return {"bytes": total * (c["K"] + 2 * c["N"]) * size + w, "flops": 2 * total * c["rank"] * (c["K"] + c["N"])}
    token = c["Hkv"] * 138
    x = total * c["Hkv"] * D * 2 * size
    if c["op"] == "pages":  # rows in, cache written and read, rows out
        return {"bytes": 2 * x + 2 * total * token, "flops": 0}
    if c["op"] == "history":
        return {"bytes": x + total * token, "flops": 0}
    if c["op"] == "verify":
        kept = sum(len(_path(c, i, n)) for i, n in enumerate(rows))
        return {"bytes": x + total * token + 2 * kept * token + kept * token + kept * c["Hkv"] * D * 2 * size, "flops": 0}
    cached = sum(n + f for n, f in zip(rows, first))
    return {"bytes": cached * token + 2 * total * c["Hq"] * D * size,
            "flops": 4 * D * c["Hq"] * sum(n * (n + f) for n, f in zip(rows, first))}


def _parents(c, i, n):
    """Request i's drafted tree: the parent of each of its n tokens, -1 for the root."""
    r = random.Random(c["lens"] * 1000 + i)
    return [-1] + [r.randrange(max(0, k - 12), k) for k in range(1, n)]


def _path(c, i, n):
    """The tokens of request i's tree that are accepted: a path from the root, in order."""
    r, up, path = random.Random(c["lens"] * 1000 + 500 + i), _parents(c, i, n), []
    k = r.randrange(n)
    while k >= 0:
        path.append(k)
        k = up[k]
    return path[::-1]


# ------------------------------------------------------------------------------------------------------ the layout
def _token_bytes():
    """[32, 138]: where a token's bytes stand in its block: 64 of key codes (two dimensions a byte, the even one in the low
    nibble), 64 of value codes, the two scales, the two zero-points."""
    t, d = np.arange(TOKENS)[:, None], 2 * np.arange(D // 2)[None, :]
    n, g, cq = t >> 3, t & 7, d >> 5
    key = (n * 32 + cq * 8 + (g ^ 2 * cq)) * 16 + ((d >> 3) & 3) * 4 + ((d & 7) >> 1)
    w, g, cq = d >> 5, (d >> 2) & 7, (t >> 1) & 3
    value = 2048 + (w * 32 + cq * 8 + (g ^ 2 * cq)) * 16 + n * 4 + 2 * (t & 1) + ((d & 3) >> 1)
    four = np.arange(4)[None, :]
    return np.concatenate([key, value, 4096 + 4 * t + four, 4224 + 4 * t + four, 4352 + t, 4384 + t], axis=1)


def _where(s, request, position):
    """[n, Hkv, 138]: the places in the flat pool of the bytes of tokens at `position` of `request`."""
    P, H = s["page"], s["H"]
    page = s["table"].long()[request, position // P]
    block = (page[:, None] * H + torch.arange(H, device="cuda")) * (P // TOKENS) + (position % P // TOKENS)[:, None]
    return block[..., None] * BLOCK + s["bytes_of"][position % TOKENS][:, None, :]


def _rows(s):
    """Request and cache position of every row of the call."""
    row = torch.arange(s["used"], device="cuda")
    request = torch.bucketize(row, s["row_start"].long()[1:], right=True)
    return request, s["first"].long()[request] + row - s["row_start"].long()[request]


# ------------------------------------------------------------------------------------------------- the plain forms
def _rotate(x):
    """The orthonormal Walsh-Hadamard transform of the last 128 values, natural order."""
    h = 1
    while h < D:
        a = x.reshape(*x.shape[:-1], D // (2 * h), 2, h)
        x = torch.stack([a[..., 0, :] + a[..., 1, :], a[..., 0, :] - a[..., 1, :]], dim=-2).reshape(x.shape)
        h *= 2
    return x * float(np.float32(1.0 / math.sqrt(D)))


def _quantize(x):
    """fp32 [..., 128] -> codes, scale, zero-point: the range is the values' own, 0 in it, times the clipping ratio.  In
    32 bits like the cache that the framework had before: the codes follow from fp32 steps, each rounded once."""
    lo, hi = x.amin(-1).clamp(max=0) * CLIP, x.amax(-1).clamp(min=0) * CLIP
    some = hi != lo
    scale = torch.where(some, (hi - lo) / torch.full_like(hi, 15.0), torch.ones_like(hi))
    zero = torch.where(some, torch.round(-lo / scale), torch.zeros_like(hi))
    code = (torch.round(x / scale[..., None]) + zero[..., None]).clamp(0, 15)
    return code.to(torch.uint8), scale, zero.to(torch.uint8)


def _as_bytes(keys, values):
    """The 138 bytes of each token and head: what _where() says the places of."""
    out = []
    for x in (keys, values):
        code, scale, zero = _quantize(x)
        out.append((code[..., 0::2] | code[..., 1::2] << 4, scale.contiguous()[..., None].view(torch.uint8), zero[..., None]))
    (kc, ks, kz), (vc, vs, vz) = out
    return torch.cat([kc, vc, ks, vs, kz, vz], dim=-1)


def _from_bytes(b):
    """Keys and values in fp32 that the bytes [..., 138] stand for."""
    out = []
    for code, scale, zero in ((b[..., :64], b[..., 128:132], b[..., 136:137]), (b[..., 64:128], b[..., 132:136], b[..., 137:138])):
        code = torch.stack([code & 15, code >> 4], dim=-1).reshape(*code.shape[:-1], D)
        out.append(scale.contiguous().view(torch.float32) * (code.float() - zero.float()))
    return out


def _plain_read(s, request, position):
    k, v = _from_bytes(s["pool"].view(-1)[_where(s, request, position)])
    return _rotate(k).to(s["dtype"]), v.to(s["dtype"])


def _plain_write(s):
    request, position = _rows(s)
    s["pool"].view(-1)[_where(s, request, position)] = _as_bytes(_rotate(s["k"][:s["used"]].float()), s["v"][:s["used"]].float())
    return request, position


def _plain_keep(s):
    """Moves the kept tokens of every request to the front of its drafted ones; returns request and place of each."""
    request = torch.bucketize(torch.arange(s["kept"], device="cuda"), s["kept_start"].long()[1:], right=True)
    i = torch.arange(s["kept"], device="cuda") - s["kept_start"].long()[request]
    to = s["first"].long()[request] + i
    source = s["first"].long()[request] + s["keep"].long()[s["row_start"].long()[request] + i]
    s["pool"].view(-1)[_where(s, request, to)] = s["pool"].view(-1)[_where(s, request, source)]
    return request, to


def _plain_attention(s):
    R, H, G = s["R"], s["H"], s["Hq"] // s["H"]
    n = s["most_rows"]
    row = s["row_start"].long()[:-1, None] + torch.arange(n, device="cuda")
    there = row < s["row_start"].long()[1:, None]                                       # [R, n]
    row = torch.where(there, row, 0)
    q = _rotate(s["q"][row].float()).reshape(R, n, H, G, D).permute(0, 2, 1, 3, 4).reshape(R, H, n * G, D)
    t = torch.arange(s["most_tokens"], device="cuda")
    request = torch.arange(R, device="cuda")[:, None].expand(R, t.numel())
    k, v = _from_bytes(s["pool"].view(-1)[_where(s, request.reshape(-1), t.expand_as(request).reshape(-1))])
    k, v = (x.reshape(R, t.numel(), H, D).transpose(1, 2) for x in (k, v))
    drafted = t - s["first"].long()[:, None]                                            # [R, T]
    word = (drafted.clamp(0, 63) >> 5)[:, None, :].expand(R, n, -1)
    word = torch.gather(s["mask"].long()[row], 2, word)
    seen = (word >> (drafted.clamp(0, 63) & 31)[:, None, :]) & 1
    seen = (drafted < 0)[:, None, :] | ((drafted < 64)[:, None, :] & (seen == 1))       # [R, n, T]
    seen = (seen & there[:, :, None])[:, None, :, None, :].expand(R, H, n, G, -1).reshape(R, H, n * G, -1)
    score = torch.matmul(q, k.transpose(2, 3)) * float(np.float32(1.0 / math.sqrt(D)))
    score = torch.where(seen, score, -math.inf)
    p = torch.exp(score - score.amax(-1, keepdim=True).clamp(min=-1e30))
    o = torch.matmul(p, v) / p.sum(-1, keepdim=True).clamp(min=1e-30)
    o = o.reshape(R, H, n, G, D).permute(0, 2, 1, 3, 4).reshape(R, n, s["Hq"], D)
    s["out"][row[there]] = o[there].to(s["dtype"])
    return s["out"]


def _plain_lora(s):
    """Every adapter's products for every row, all but the row's own masked out."""
    row = torch.arange(s["x"].shape[0], device="cuda")
    request = torch.bucketize(row, s["row_start"].long()[1:], right=True)
    mine = torch.cat([s["adapter"].long(), torch.full((1,), -1, device="cuda")])[request]
    n, rank, K = s["A"].shape
    t = torch.matmul(s["x"].float(), s["A"].float().reshape(n * rank, K).T).reshape(-1, n, rank)
    t = t * s["scaling"][:, None] * (mine[:, None] == torch.arange(n, device="cuda"))[..., None]
    add = torch.matmul(t.reshape(-1, n * rank), s["B"].float().transpose(1, 2).reshape(n * rank, -1))
    return (s["y"].float() + add).to(s["dtype"])


# -------------------------------------------------------------------------------------------------------- one pass
def run(s):
    return _own(s) if own else _plain(s)


def _plain(s):
    if s["op"] == "pages":
        return _plain_read(s, *_plain_write(s))
    if s["op"] == "history":
        return _plain_read(s, *_rows(s))
    if s["op"] == "verify":
        _plain_write(s)
        return _plain_read(s, *_plain_keep(s))
    return _plain_attention(s) if s["op"] == "attention" else _plain_lora(s)


def _own(s):
    import paper_2606_02823_b200 as qift

    if s["op"] == "lora":
        return qift.qift_lora_linear(s["x"], s["A"], s["B"], s["scaling"], s["row_start"], s["adapter"], s["y"])
    pages = qift.Kv4Pages(s["pool"], s["table"], s["page"])
    if s["op"] == "attention":
        return qift.qift_kv4_paged_attention(s["q"], pages, s["row_start"], s["first"], mask=s["mask"], q_had_block=D, out=s["out"])
    if s["op"] != "history":
        qift.qift_kv4_paged_write(s["k"], s["v"], pages, s["row_start"], s["first"], k_had_block=D, clip_ratio=CLIP)
    if s["op"] == "verify":
        qift.qift_kv4_paged_keep(pages, s["row_start"], s["first"], s["keep"], s["kept_start"])
        return qift.qift_kv4_paged_read(pages, s["kept_start"], s["first"], s["kept"], s["dtype"], k_had_block=D)
    return qift.qift_kv4_paged_read(pages, s["row_start"], s["first"], s["used"], s["dtype"], k_had_block=D)


# ------------------------------------------------------------------------------------------------------- the state
def _ints(v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype, device="cuda")


def _sums(v):
    return [0] + np.cumsum(v).tolist()


def prepare(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dtype = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    rows, first = _lengths(c)
    R, used = len(rows), sum(rows)
    s = dict(op=c["op"], dtype=dtype, R=R, used=used, row_start=_ints(_sums(rows)), first=_ints(first))

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    if c["op"] == "lora":
        r, n = random.Random(c["lens"] + 1), c["adapters"]
        s |= dict(x=normal(used, c["K"]).to(dtype), y=normal(used, c["N"]).to(dtype), adapter=_ints([r.randrange(n) for _ in rows]),
                  A=(normal(n, c["rank"], c["K"]) / math.sqrt(c["K"])).bfloat16(), B=(normal(n, c["N"], c["rank"]) / math.sqrt(c["rank"])).bfloat16(),
                  scaling=torch.rand(n, generator=g, device="cuda") + 0.5)
        return s

    H, P = c["Hkv"], c["page"]
    lengths = [n + f for n, f in zip(rows, first)]
    need = [-(-n // P) for n in lengths]
    total_pages = sum(need) + 3
    # pages in no order, as a pool that has been in use for a while hands them out
    order = torch.randperm(total_pages, generator=g, device="cuda").to(torch.int32)
    start = _ints(_sums(need), torch.int64)
    at = start[:-1, None] + torch.arange(max(need) + 1, device="cuda")
    s |= dict(H=H, page=P, table=torch.where(at < start[1:, None], order[at.clamp(max=total_pages - 1)], -1).contiguous(),
              bytes_of=torch.from_numpy(_token_bytes()).cuda(), pool=torch.zeros((total_pages, H, P // TOKENS * BLOCK), dtype=torch.uint8, device="cuda"))

    def vectors(n, shift):  # a few channels far larger than the rest, as keys have them
        x = normal(n, H, D) + shift
        x[..., 5::43] *= 6.0
        return x

    if c["op"] in ("pages", "verify"):
        s |= dict(k=vectors(used, 0.1).to(dtype), v=(normal(used, H, D) - 0.1).to(dtype))
    if c["op"] == "verify":
        paths = [_path(c, i, n) for i, n in enumerate(rows)]
        keep = [k for p, n in zip(paths, rows) for k in p + [0] * (n - len(p))]
        s |= dict(keep=_ints(keep), kept_start=_ints(_sums([len(p) for p in paths])), kept=sum(len(p) for p in paths))
    if c["op"] in ("history", "attention"):
        n = sum(lengths)
        cut = _ints(_sums(lengths), torch.int64)
        request = torch.bucketize(torch.arange(n, device="cuda"), cut[1:], right=True)
        position = torch.arange(n, device="cuda") - cut[request]
        s["pool"].view(-1)[_where(s, request, position)] = _as_bytes(_rotate(vectors(n, 0.1)), normal(n, H, D) - 0.1)
    if c["op"] == "attention":
        masks = np.zeros((used, 2), np.int64)
        at = 0
        for i, n in enumerate(rows):
            up = _parents(c, i, n) if c["tree"] else list(range(-1, n - 1))
            bits = []
            for k in range(n):
                bits.append((bits[up[k]] if up[k] >= 0 else 0) | 1 << k)
                masks[at + k] = bits[k] & 0xFFFFFFFF, bits[k] >> 32
            at += n
        s |= dict(Hq=c["Hq"], q=(normal(used, c["Hq"], D) * 1.2).to(dtype), out=torch.zeros((used, c["Hq"], D), dtype=dtype, device="cuda"),
                  mask=torch.from_numpy(masks.astype(np.uint32).view(np.int32)).cuda(), most_rows=max(rows), most_tokens=max(lengths))
    return s


# ------------------------------------------------------------------------------------- the definitions, in 64 bits
def _exact_hadamard():
    i = torch.arange(D, device="cuda")
    both = i[:, None] & i[None, :]
    odd = sum((both >> b) & 1 for b in range(7)) % 2
    return (1.0 - 2.0 * odd.double()) / math.sqrt(D)


def _exact_held(x):
    """What the cache holds of x.  The operator's definition has the range's ends, the scale and the quotients that are
    rounded to codes as fp32 numbers (equal ends, frequent among 16-bit values, put the zero-point on a border); they are
    64-bit results rounded once."""
    once = lambda v: v.float().double()  # noqa: E731
    clip, nought = float(np.float32(CLIP)), torch.zeros((), dtype=torch.float64, device="cuda")
    lo, hi = once(clip * torch.minimum(x.amin(-1), nought)), once(clip * torch.maximum(x.amax(-1), nought))
    scale = once(once(hi - lo) / 15)
    scale[hi == lo] = 1.0
    zero = torch.round(once(-lo / scale))
    code = torch.minimum(torch.maximum(torch.round(once(x / scale.unsqueeze(-1))) + zero.unsqueeze(-1), torch.zeros_like(x)), torch.full_like(x, 15.0))
    return scale.unsqueeze(-1) * (code - zero.unsqueeze(-1))


def _exact_cached(s, r, begin, end):
    """Keys and values [tokens, Hkv, 128] of a request as its pages hold them, block by block from the nibbles."""
    P, H = s["page"], s["H"]
    blocks = s["pool"][s["table"][r, :-(-end // P)].long()].reshape(-1, H, P // TOKENS, BLOCK).transpose(1, 2).reshape(-1, H, BLOCK)
    nb = blocks.shape[0]
    swap = torch.tensor([[g ^ 2 * c for g in range(8)] for c in range(4)], device="cuda").reshape(1, 1, 1, 4, 8, 1)
    nibbles = lambda b: torch.stack([b & 15, b >> 4], -1).flatten(-2)  # noqa: E731
    kc = nibbles(blocks[..., :2048].reshape(nb, H, 4, 4, 8, 16).gather(4, swap.expand(nb, H, 4, 4, 8, 16)))
    kc = kc.permute(0, 2, 4, 1, 3, 5).reshape(nb * TOKENS, H, D)                        # block, n, g | head | cq, 32 dims
    vc = blocks[..., 2048:4096].reshape(nb, H, 4, 4, 8, 16).gather(4, swap.expand(nb, H, 4, 4, 8, 16))
    vc = nibbles(vc.reshape(nb, H, 4, 4, 8, 4, 2, 2))                                   # block, head, w, cq, g, n, parity, 4 dims
    vc = vc.permute(0, 5, 3, 6, 1, 2, 4, 7).reshape(nb * TOKENS, H, D)
    out = []
    for code, at, zat in ((kc, 4096, 4352), (vc, 4224, 4384)):
        scale = blocks[..., at:at + 128].contiguous().view(torch.float32).double().transpose(1, 2).reshape(nb * TOKENS, H, 1)
        zero = blocks[..., zat:zat + 32].double().transpose(1, 2).reshape(nb * TOKENS, H, 1)
        out.append((scale * (code.double() - zero))[begin:end])
    return out


def exact(c, seed):
    s = prepare(c, seed)
    rows, first = _lengths(c)
    cut, had = _sums(rows), _exact_hadamard()
    if c["op"] == "lora":
        y = s["y"].double()
        for i, a in enumerate(s["adapter"].tolist()):
            x = s["x"][cut[i]:cut[i + 1]].double()
            y[cut[i]:cut[i + 1]] += s["scaling"][a].double() * (x @ s["A"][a].double().T) @ s["B"][a].double().T
        return y
    if c["op"] in ("pages", "verify"):
        k, v = s["k"].double(), s["v"].double()
        if c["op"] == "verify":
            at = torch.tensor([cut[i] + p for i, n in enumerate(rows) for p in _path(c, i, n)], device="cuda")
            k, v = k[at], v[at]
        return _exact_held(k @ had) @ had, _exact_held(v)
    if c["op"] == "history":
        both = [_exact_cached(s, i, f, f + n) for i, (n, f) in enumerate(zip(rows, first))]
        return torch.cat([k for k, _ in both]) @ had, torch.cat([v for _, v in both])
    out, G = torch.zeros(s["used"], c["Hq"], D, dtype=torch.float64, device="cuda"), c["Hq"] // c["Hkv"]
    for i, (n, f) in enumerate(zip(rows, first)):
        up = _parents(c, i, n) if c["tree"] else list(range(-1, n - 1))
        hidden = torch.ones(n, f + n, dtype=torch.bool)
        hidden[:, :f] = False
        for a in range(n):
            b = a
            while b >= 0:
                hidden[a, f + b] = False
                b = up[b]
        k, v = _exact_cached(s, i, 0, f + n)
        q = s["q"][cut[i]:cut[i + 1]].double() @ had
        for h in range(c["Hkv"]):
            score = torch.einsum("ngd,td->gnt", q[:, h * G:(h + 1) * G], k[:, h]) / math.sqrt(D)
            p = torch.softmax(score.masked_fill(hidden.cuda(), -math.inf), dim=-1)
            out[cut[i]:cut[i + 1], h * G:(h + 1) * G] = torch.einsum("gnt,td->ngd", p, v[:, h])
    return out
