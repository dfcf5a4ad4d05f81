"""Cases for what stands between the quantized projections of a decoder layer that serves many requests: the page tables,
positions and slots of a step, made from the requests' lengths on the device; the norms of queries and keys for each head
together with the position rotation; and the gated half of the feed-forward block, both products and the activation.

Page tables: page_table [R, max_pages] names the pages of each request (values outside 0 .. pages - 1: none), free [pages] with
count [1] is a stack of free ones.  A step adds rows[r] tokens behind first[r] cached ones and takes pages for them; it ends
with length[r] tokens that stay, and pages behind those go back.

Packed weights: tiles of 16 rows x 128 words of 16 two-bit (or 8 four-bit) codes; the three-bit set has its third bits
in words beside them.  The formulas are _word() and its neighbours.
"""
import math
import random

import numpy as np
import torch

own = False

CLIP = 0.9
BITS = dict(mnz=2, pot=2, sym=2, int4=4, int3=3)


# ---------------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # 64 requests decode one token each: the smallest tables, bound by the calls themselves
        dict(name="tables-decode-64x1", op="tables", requests=64, rows=1, ragged=False, context=8000, page=64, tree=False, short=False, lens=1),
        # a large batch drafts trees, a path of each is accepted
        dict(name="tables-verify-192x64", op="tables", requests=192, rows=64, ragged=True, context=2000, page=32, tree=True, short=False, lens=2),
        # prompts of many requests enter at once, the pool is too small for the last of them
        dict(name="tables-prompts-256x4000", op="tables", requests=256, rows=4000, ragged=True, context=500, page=64, tree=False, short=True, lens=3),
        # single tokens, grouped query heads, no norms: latency
        dict(name="rope-decode-48", op="rope", total=48, Hq=32, H=8, D=128, rot=128, norm=False, near=False, far=4000, dtype="bf16"),
        # fp32 rows in odd number with norms, neighbouring pairs, only part of a head rotated, far positions
        dict(name="rope-1237-f32", op="rope", total=1237, Hq=32, H=32, D=128, rot=96, norm=True, near=True, far=1000000, dtype="f32"),
        # prompts, with norms
        dict(name="rope-prompts-18000", op="rope", total=18000, Hq=32, H=8, D=128, rot=128, norm=True, near=False, far=32000, dtype="bf16"),
        # one token through the gated block of a 4096 -> 11008 layer, rotation and quantizer in the call
        dict(name="gated-1", op="forward", M=1, K=4096, N=11008, levels="mnz", act="silu", dtype="bf16"),
        # a few tokens, the power-of-two levels, 4096 -> 14336
        dict(name="gated-7-pot-f32", op="linear", M=7, K=4096, N=14336, levels="pot", act="silu", dtype="f32"),
        # three-bit weights
        dict(name="gated-13-int3-f32", op="linear", M=13, K=4096, N=11008, levels="int3", act="gelu", dtype="f32"),
        # a batch of decoding requests
        dict(name="gated-48", op="forward", M=48, K=4096, N=14336, levels="mnz", act="silu", dtype="bf16"),
        # a short prompt, four-bit weights
        dict(name="gated-300-int4-f32", op="linear", M=300, K=4096, N=11008, levels="int4", act="silu", dtype="f32"),
        # a long prompt
        dict(name="gated-2048", op="forward", M=2048, K=4096, N=14336, levels="mnz", act="silu", dtype="bf16"),
    ]


def draw(rng):
    def log(lo, hi):
        return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    op = rng.choice(["tables", "tables", "rope", "rope", "forward", "linear", "linear"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "tables":
        c = dict(op=op, requests=log(1, 512), ragged=rng.random() < 0.7, page=rng.choice([32, 64, 128]), tree=rng.random() < 0.4,
                 short=rng.random() < 0.2, lens=rng.randrange(1 << 30), context=rng.choice([0, log(1, 8000), log(1, 30000)]))
        c["rows"] = log(1, 64) if c["tree"] else log(1, max(1, min(8000, 600_000 // c["requests"])))
        return c
    if op == "rope":
        Hq, H = rng.choice([(32, 8), (32, 8), (32, 32), (7, 1), (12, 3)])
        D = rng.choice([128, 128, 64, 256])
        c = dict(op=op, Hq=Hq, H=H, D=D, rot=rng.choice([D, D, D // 2, D - 32]), norm=rng.random() < 0.5, near=rng.random() < 0.4,
                 far=log(100, 2_000_000), dtype=dtype)
        c["total"] = log(1, 18000 * 40 * 128 // ((Hq + H) * D) // (2 if dtype == "f32" else 1))
        return c
    c = dict(op=op, levels=rng.choice(["mnz", "mnz", "pot", "sym", "int4", "int3"]), act=rng.choice(["silu", "silu", "gelu"]), dtype=dtype)
    c["K"] = rng.choice([1024, 2048, 4096, 4096, 32 * rng.randint(8, 128)])
    c["N"] = log(100, 14336)
    c["M"] = rng.choice([1, log(2, 16), log(17, 128), log(129, 2048)])
    return c


def _lengths(c):
    """Rows and cached tokens of each request, and how many of the rows stay: from the case alone."""
    r = random.Random(c["lens"])
    rows = [r.randint(max(0, c["rows"] // 8), c["rows"]) if c["ragged"] else c["rows"] for _ in range(c["requests"])]
    first = [r.randint(c["context"] // 8, c["context"]) for _ in rows]
    rows[-1] = c["rows"]
    stay = [r.randint(0, n) for n in rows] if c["tree"] else [0] * len(rows)
    return rows, first, stay


def work(c):
    size = 2 if c.get("dtype") == "bf16" else 4
    if c["op"] == "tables":
        rows, first, stay = _lengths(c)
        P, total = c["page"], sum(rows)
        taken = sum(-(-(f + n) // P) - -(-f // P) for n, f in zip(rows, first))
        back = sum(-(-(f + n) // P) - -(-(f + k) // P) for n, f, k in zip(rows, first, stay))
        return {"bytes": 16 * len(rows) + 8 * (taken + back) + total * (12 + (8 if c["tree"] else 0)), "flops": 0}
    if c["op"] == "rope":
        x = (c["total"] - c["total"] // 9) * (c["Hq"] + c["H"]) * c["D"]                   # rows of padding are left alone
        return {"bytes": 2 * x * size + 4 * c["total"], "flops": 8 * x}
    M, N, K = c["M"], c["N"], c["K"]
    x = M * K * size if c["op"] == "forward" else M * (K + 4)
    return {"bytes": 2 * N * K * BITS[c["levels"]] // 8 + 8 * N + x + M * N * size, "flops": 4 * M * N * K}


# ------------------------------------------------------------------------------------------------ packed weights
def _word(n, j, pitch):
    """Where word j of row n stands (two- and four-bit codes)."""
    jj = j & 127
    return (n >> 4) * 16 * pitch + (j >> 7) * 2048 + ((((jj >> 4) * 2 + ((n >> 3) & 1)) * 32 + (n & 7) * 4 + ((jj >> 2) & 3)) << 2) + (jj & 3)


def _word3(n, j, pitch):
    """Where the low word j of row n stands (three-bit codes), and the word with its third bits."""
    at = (n >> 4) * 24 * pitch + (j >> 4) * 384
    quad = (n & 7) * 4 + ((j >> 2) & 3)
    half = (n >> 3) & 1
    return at + ((half * 32 + quad) << 2) + (j & 3), at + 256 + (quad << 2) + 2 * half + ((j >> 1) & 1)


def _places(N, K, levels):
    """Addresses [N, words] and the shifts of a word's codes, in ascending k; for three bits, those of the third bits too."""
    per = 8 if levels == "int4" else 16
    words = K // per
    pitch = (words + 15) // 16 * 16
    n, j = torch.arange(N, device="cuda")[:, None], torch.arange(words, device="cuda")[None, :]
    i = torch.arange(per, device="cuda")
    shift = 8 * (i % 4) + (4 if levels == "int4" else 2) * (i // 4)
    if levels != "int3":
        return _word(n, j, pitch), shift, None, None
    low, high = _word3(n, j, pitch)
    third = 4 * (j[..., None] & 1) + 8 * (i % 4) + torch.tensor([0, 2, 1, 3], device="cuda")[i // 4]
    return low, shift, high, third


def _pack(code, levels):
    N, K = code.shape
    low, shift, high, third = _places(N, K, levels)
    per, pitch = shift.numel(), (K // shift.numel() + 15) // 16 * 16
    rows = (N + 15) // 16 * 16
    out = torch.zeros(rows * pitch * 3 // 2 if levels == "int3" else rows * pitch, dtype=torch.int64, device="cuda")
    c = code.reshape(N, -1, per).long()
    out[low] = ((c & (15 if levels == "int4" else 3)) << shift).sum(-1)
    if levels == "int3":
        bits = ((c >> 2) << third).sum(-1)
        out.index_put_((high,), bits, accumulate=True)
    return torch.where(out >= 1 << 31, out - (1 << 32), out).to(torch.int32)


def _levels_of(packed, N, K, levels):
    """The levels that the codes stand for, fp32 [N, K]."""
    low, shift, high, third = _places(N, K, levels)
    shift = shift.to(torch.int32)
    if levels == "int4":
        c = ((packed[low][..., None] >> shift) & 15).reshape(N, K)
        return ((c ^ 8) - 8).float()
    c = ((packed[low][..., None] >> shift) & 3).reshape(N, K)
    if levels == "int3":
        return (c - 4 * ((packed[high][..., None] >> third.to(torch.int32)) & 1).reshape(N, K)).float()
    return (2 * c - 3 if levels == "mnz" else c - 2 if levels == "sym" else 3 * c - (c >> 1) - 4).float()


# ------------------------------------------------------------------------------------------------- the plain forms
def _plain_begin(s):
    P, total, pages = s["page"], s["total"], s["pages"]
    rows, first, table = s["rows"].long().clamp(min=0), s["first"].long(), s["table"]
    R, most = table.shape
    start = torch.nn.functional.pad(torch.cumsum(rows, 0), (1, 0)).clamp(max=total)
    n = start[1:] - start[:-1]
    i = torch.arange(most, device="cuda")
    wanted = (i >= (first // P)[:, None]) & (i < ((first + n + P - 1) // P)[:, None]) & (n > 0)[:, None]
    wanted &= (table < 0) | (table >= pages)
    k = torch.cumsum(wanted.reshape(-1), 0).reshape(R, most) - 1
    count = s["count"].long()
    page = torch.where(k < count, s["free"][(count - 1 - k).clamp(min=0)], -1)
    table.copy_(torch.where(wanted, page, table))
    s["count"].copy_((count - torch.minimum(wanted.sum(), count)).int())
    row = torch.arange(total, device="cuda")
    request = torch.bucketize(row, start[1:], right=True).clamp(max=R - 1)
    place = first[request] + row - start[request]
    held = table.reshape(-1)[request * most + (place // P).clamp(max=most - 1)].long()
    there = row < start[-1]
    some = there & (held >= 0) & (held < pages) & (place < most * P)
    slot = torch.where(some, held * P + place % P, -1)
    position = place
    if s["mask"] is not None:
        bit = torch.arange(32, device="cuda", dtype=torch.int32)
        seen = ((s["mask"][..., None] >> bit) & 1).sum((1, 2))
        position = first[request] + (seen - 1).clamp(min=0)
    lost = rows.sum() - some.sum()
    return start.int(), torch.where(there, position, -1).int(), slot, lost.int().reshape(1)


def _plain_end(s):
    P, table, pages = s["page"], s["table"], s["pages"]
    behind = torch.arange(table.shape[1], device="cuda") >= ((s["length"].long().clamp(min=0) + P - 1) // P)[:, None]
    back = behind & (table >= 0) & (table < pages)
    k = torch.cumsum(back.reshape(-1), 0).reshape(back.shape) - 1
    top = s["count"].long() + back.sum() - 1
    stack = torch.cat([s["free"], s["free"][:1]])            # one place more for what does not go back
    stack[torch.where(back, (top - k).clamp(max=pages), pages)] = table
    s["free"].copy_(stack[:-1])
    s["count"].copy_((s["count"] + back.sum()).clamp(max=pages).int())
    table.copy_(torch.where(behind, -1, table))


def _turned(x, cos, sin, rot, near):
    x, rest = x[..., :rot], x[..., rot:]
    a, b = (x[..., 0::2], x[..., 1::2]) if near else (x[..., :rot // 2], x[..., rot // 2:])
    a, b = a * cos - b * sin, b * cos + a * sin
    return torch.cat([torch.stack([a, b], -1).flatten(-2) if near else torch.cat([a, b], -1), rest], -1)


def _plain_rope(s):
    position = s["position"]
    angle = position.double()[:, None] * s["inv_freq"].double()
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    out = []
    for x, w, old in ((s["q"], s["wq"], s["q_out"]), (s["k"], s["wk"], s["k_out"])):
        y = x.float()
        if w is not None:
            y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + s["eps"]) * w.float()
        y = _turned(y, cos, sin, s["rot"], s["near"]).to(s["dtype"])
        out.append(torch.where((position >= 0)[:, None, None], y, old))
    return out


def _plain_quantize(x):
    """Rows rotated by the whole Walsh-Hadamard transform of blocks (the largest power of two in K), rounded to four bits: in
    32 bits with the steps in this order, each rounded once, as the framework's quantizer has them."""
    u, K = x.float(), x.shape[1]
    B, h = K & -K, 1
    while h < B:
        a = u.reshape(-1, K // (2 * h), 2, h)
        u = torch.stack([a[:, :, 0] + a[:, :, 1], a[:, :, 0] - a[:, :, 1]], 2).reshape(-1, K)
        h *= 2
    top = u.abs().amax(1, keepdim=True)
    step = torch.where(top > 0, top * CLIP / torch.full_like(top, 7.0), torch.ones_like(top))
    return torch.round(u / step).clamp(-8, 7), step[:, 0] * float(np.float32(1.0 / math.sqrt(B)))


def _act(g, act):
    if act == "silu":
        return g / (1 + torch.exp(-g))
    return 0.5 * g * (1 + torch.tanh(math.sqrt(2 / math.pi) * (g + 0.044715 * g * g * g)))


def _plain_gated(s):
    q, sa = _plain_quantize(s["x"]) if s["op"] == "forward" else (s["q_a"].float(), s["s_a"])
    g, u = (torch.matmul(q, _levels_of(p, sn.numel(), q.shape[1], s["levels"]).T) * sa[:, None] * sn for p, sn in (s["gate"], s["up"]))
    return (_act(g, s["act"]) * u).to(s["dtype"])


# -------------------------------------------------------------------------------------------------------- one pass
def run(s):
    if s["op"] == "tables":
        out = _own_tables(s) if own else (_plain_begin(s), _plain_end(s))[0]
        return [*out, s["table"], s["free"], s["count"]]
    if s["op"] == "rope":
        return _own_rope(s) if own else _plain_rope(s)
    return _own_gated(s) if own else _plain_gated(s)


def _own_tables(s):
    import paper_2606_02823_b200 as qift

    pages = qift.Kv4Pages(s["pool"], s["table"], s["page"])
    free = qift.Kv4FreePages(s["free"], s["count"])
    rows = qift.qift_kv4_pages_begin(pages, free, s["rows"], s["first"], s["total"], mask=s["mask"])
    qift.qift_kv4_pages_end(pages, free, s["length"])
    return rows.row_start, rows.position, rows.slot, rows.lost


def _own_rope(s):
    import paper_2606_02823_b200 as qift

    return qift.qift_qk_norm_rope(s["q"], s["k"], s["position"], s["inv_freq"], q_weight=s["wq"], k_weight=s["wk"], eps=s["eps"],
                                  pairs=qift.ROPE_NEIGHBOURS if s["near"] else qift.ROPE_HALVES, q_out=s["q_out"], k_out=s["k_out"])


def _own_gated(s):
    import paper_2606_02823_b200 as qift

    levels = dict(mnz=qift.MNZ, pot=qift.POT, sym=qift.SYM, int4=qift.INT4, int3=qift.INT3)[s["levels"]]
    act = qift.ACT_SILU if s["act"] == "silu" else qift.ACT_GELU_TANH
    if s["op"] == "forward":
        return qift.qift_gated_forward(s["x"], s["had"], s["gate"], s["up"], levels, CLIP, activation=act, out_dtype=s["dtype"])
    return qift.qift_gated_linear(s["q_a"], s["s_a"], s["gate"], s["up"], levels, activation=act, out_dtype=s["dtype"])


# ------------------------------------------------------------------------------------------------------- the state
def _ints(v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype, device="cuda")


def _masks(c, rows):
    """A tree for each request: every token's ancestors and itself, two words a row."""
    out = []
    for i, n in enumerate(rows):
        r, bits = random.Random(c["lens"] * 1000 + i), []
        for k in range(n):
            up = r.randrange(max(0, k - 12), k) if k else -1
            bits.append((bits[up] if k else 0) | 1 << k)
        out += [[b & 0xFFFFFFFF, b >> 32] for b in bits]
    return np.array(out, np.uint32).reshape(-1, 2).view(np.int32)


def prepare(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dtype = torch.bfloat16 if c.get("dtype") == "bf16" else torch.float32

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    if c["op"] == "tables":
        rows, first, stay = _lengths(c)
        P, R = c["page"], len(rows)
        # what requests hold: pages of their cached tokens, and some one more, left of an earlier draft
        held = [-(-f // P) + (i % 5 == 0) for i, f in enumerate(first)]
        taken = [max(0, -(-(f + n) // P) - h) for f, n, h in zip(first, rows, held)]
        left = sum(taken) * 9 // 10 if c["short"] else sum(taken) + 50
        pages, most = sum(held) + left, max(-(-(f + n) // P) for f, n in zip(first, rows)) + 2
        order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)      # a pool that has been in use for a while
        i, h = torch.arange(most, device="cuda"), _ints(held, torch.int64)[:, None]
        at = _ints(np.cumsum([0] + held[:-1]).tolist(), torch.int64)[:, None] + i
        free = torch.full((pages,), -1, dtype=torch.int32, device="cuda")
        free[:left] = order[sum(held):]
        total = sum(rows) + (7 if c["ragged"] else 0)                                  # a padded batch
        mask = None
        if c["tree"]:
            mask = torch.zeros((total, 2), dtype=torch.int32, device="cuda")
            mask[:sum(rows)] = torch.from_numpy(_masks(c, rows)).cuda()
        return dict(op=c["op"], page=P, pages=pages, total=total, rows=_ints(rows), first=_ints(first), mask=mask,
                    length=_ints([f + k for f, k in zip(first, stay)]), free=free, count=_ints([left]),
                    table=torch.where(i < h, order[at.clamp(max=pages - 1)], -1).contiguous(),
                    pool=torch.empty((pages, 1, P // 32 * 4416), dtype=torch.uint8, device="cuda"))

    if c["op"] == "rope":
        Hq, H, D, total = c["Hq"], c["H"], c["D"], c["total"]
        row = normal(total, Hq + 2 * H, D).to(dtype)                                   # one projection's rows: queries, keys, values
        position = torch.randint(0, c["far"], (total,), generator=g, device="cuda", dtype=torch.int32)
        position[total - total // 9:] = -1                                             # padding
        inv = 1.0 / 500000.0 ** (torch.arange(0, c["rot"], 2, device="cuda", dtype=torch.float64) / c["rot"])
        weight = lambda: (1 + 0.2 * normal(D)).to(dtype) if c["norm"] else None  # noqa: E731
        return dict(op=c["op"], dtype=dtype, rot=c["rot"], near=c["near"], eps=1e-6, q=row[:, :Hq], k=row[:, Hq:Hq + H], position=position,
                    inv_freq=inv.float(), wq=weight(), wk=weight(), q_out=torch.zeros((total, Hq, D), dtype=dtype, device="cuda"),
                    k_out=torch.zeros((total, H, D), dtype=dtype, device="cuda"))

    M, N, K, levels = c["M"], c["N"], c["K"], c["levels"]
    s = dict(op=c["op"], dtype=dtype, levels=levels, act=c["act"], had=K & -K)
    if c["op"] == "forward":
        x = normal(M, K)
        x[:, 3::97] *= 20.0                                                            # a few channels far larger than the rest
        s["x"], reach = x.to(dtype), 2.2
    else:
        s["q_a"] = torch.round(normal(M, K) * 2.3).clamp(-8, 7).to(torch.int8)
        s["s_a"], reach = torch.rand(M, generator=g, device="cuda") * 0.05 + 0.02, 0.1
    for name in ("gate", "up"):
        w = normal(N, K)
        if levels in ("mnz", "pot"):
            code = torch.bucketize(w, torch.tensor([-1.0, 0.0, 1.0], device="cuda"))
        elif levels == "sym":
            code = torch.round(w).clamp(-2, 1) + 2
        else:
            code = torch.round(w * (2.5 if levels == "int4" else 1.5)).clamp(*((-8, 7) if levels == "int4" else (-4, 3))).long() & (15 if levels == "int4" else 7)
        top = dict(mnz=1.7, pot=2.2, sym=1.0, int4=2.5, int3=1.5)[levels]
        s[name] = (_pack(code, levels), (torch.rand(N, generator=g, device="cuda") + 0.5) * 1.5 / (reach * top * math.sqrt(K)))
    return s


# ------------------------------------------------------------------------------------- the definitions, in 64 bits
def _exact_tables(c, s):
    rows, first, stay = _lengths(c)
    P, pages, table = c["page"], s["pages"], s["table"].cpu().numpy()
    stack = s["free"].cpu().tolist()[:int(s["count"])]
    free = np.array(s["free"].cpu())
    place, slot = [], []
    for r, (n, f) in enumerate(zip(rows, first)):
        for i in range(f // P, -(-(f + n) // P) if n else 0):
            if not 0 <= table[r, i] < pages:
                table[r, i] = stack.pop() if stack else -1
        p = np.arange(f, f + n)
        page = table[r, p // P].astype(np.int64)
        place.append(p)
        slot.append(np.where(page >= 0, page * P + p % P, -1))
    pad = np.full(s["total"] - sum(rows), -1)
    if s["mask"] is not None:
        words = s["mask"].cpu().numpy().view(np.uint32)[:sum(rows)]
        depth = np.unpackbits(words.view(np.uint8), axis=1).sum(1).astype(np.int64) - 1
        place = [np.repeat(first, rows) + depth]
    slot = np.concatenate(slot + [pad])
    back = []
    for r, (f, k) in enumerate(zip(first, stay)):
        keep = -(-(f + k) // P)
        back += [p for p in table[r, keep:] if 0 <= p < pages]
        table[r, keep:] = -1
    stack += back[::-1]
    free[:len(stack)] = stack
    whole = lambda v, t: torch.from_numpy(np.asarray(v).astype(t))  # noqa: E731
    return [whole(np.cumsum([0] + rows), np.int32), whole(np.concatenate(place + [pad]), np.int32), whole(slot, np.int64),
            whole([sum(rows) - (slot >= 0).sum()], np.int32), whole(table, np.int32), whole(free, np.int32), whole([len(stack)], np.int32)]


def _exact_rope(c, s):
    rot, out = c["rot"], []
    angle = s["position"].double().unsqueeze(1) * s["inv_freq"].double().unsqueeze(0)
    turn = torch.polar(torch.ones_like(angle), angle).unsqueeze(1)                     # the pairs as complex numbers
    for x, w in ((s["q"], s["wq"]), (s["k"], s["wk"])):
        y = x.double()
        if w is not None:
            y = y * (y.pow(2).sum(-1, keepdim=True) / c["D"] + s["eps"]).rsqrt() * w.double()
        head = y[..., :rot]
        head = head.reshape(*head.shape[:-1], rot // 2, 2) if c["near"] else head.reshape(*head.shape[:-1], 2, rot // 2).transpose(-1, -2)
        head = torch.view_as_real(torch.view_as_complex(head.contiguous()) * turn)
        head = head.flatten(-2) if c["near"] else head.transpose(-1, -2).flatten(-2)
        out.append(torch.cat([head, y[..., rot:]], -1) * (s["position"] >= 0).double()[:, None, None])
    return out


def _exact_codes(packed, N, K, levels):
    """Codes from the packed words, from the description of the tiles: blocks of rows, slices of 16 words, groups of four words."""
    per = 8 if levels == "int4" else 16
    bits, words = 32 // per, -(-(K // per) // 16) * 16
    w = packed.long() & 0xFFFFFFFF
    t = torch.arange(per, device="cuda")
    shift = 8 * (t & 3) + bits * (t >> 2)
    if levels == "int3":
        w = w.reshape(-1, words // 16, 384)
        low, high = w[..., :256].reshape(-1, words // 16, 2, 8, 4, 4), w[..., 256:].reshape(-1, words // 16, 8, 4, 2, 2)
        low = low.permute(0, 2, 3, 1, 4, 5).reshape(-1, words, 1)
        high = high.permute(0, 4, 2, 1, 3, 5).reshape(-1, words // 2, 1).repeat_interleave(2, 1)
        odd = (torch.arange(words, device="cuda") % 2)[:, None]
        third = 8 * (t & 3) + 4 * odd + torch.tensor([0, 2, 1, 3], device="cuda")[t >> 2]
        return ((low >> shift & 3) + 4 * (high >> third & 1)).reshape(low.shape[0], -1)[:N, :K]
    w = w.reshape(-1, words // 16, 2, 8, 4, 4) if words <= 128 else torch.cat(
        [part.reshape(-1, part.shape[1] // 256, 2, 8, 4, 4) for part in w.reshape(-1, words * 16).split(2048, 1)], 1)
    w = w.permute(0, 2, 3, 1, 4, 5).reshape(-1, words, 1)
    return (w >> shift & (2 ** bits - 1)).reshape(w.shape[0], -1)[:N, :K]


def _exact_gated(c, s):
    M, N, K = c["M"], c["N"], c["K"]
    if c["op"] == "linear":
        q, sa = s["q_a"].double(), s["s_a"].double()
    else:
        once = lambda v: v.float().double()  # noqa: E731  (the definition has the step, its products and the quotients as fp32 numbers)
        B = K & -K
        i = torch.arange(B, device="cuda")
        odd = sum(((i[:, None] & i[None, :]) >> b) & 1 for b in range(B.bit_length())) % 2
        u = (s["x"].double().reshape(M, K // B, B) @ (1.0 - 2.0 * odd.double())).reshape(M, K)
        clip = float(np.float32(CLIP))
        step = once(once(once(u.abs().amax(1)) * clip) / 7)
        q = torch.round(once(u / step[:, None])).clamp(-8, 7)
        sa = once(step * float(np.float32(1.0 / math.sqrt(B))))
    value = dict(mnz=[-3, -1, 1, 3], pot=[-4, -1, 1, 4], sym=[-2, -1, 0, 1], int4=[*range(8), *range(-8, 0)], int3=[*range(4), *range(-4, 0)])[c["levels"]]
    value = torch.tensor(value, dtype=torch.float64, device="cuda")
    g, u = ((q @ value[_exact_codes(p, N, K, c["levels"])].T) * sa.unsqueeze(1) * sn.double() for p, sn in (s["gate"], s["up"]))
    if c["act"] == "silu":
        return g * torch.sigmoid(g) * u
    return g * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (g + 0.044715 * g.pow(3))) * u


def exact(c, seed):
    s = prepare(c, seed)
    return _exact_tables(c, s) if c["op"] == "tables" else _exact_rope(c, s) if c["op"] == "rope" else _exact_gated(c, s)
