"""Plain reference of the paged KV4 cache for the tests: the block layout written out place by place from its description in
include/qift.h, and the attention of drafted trees in 64 bits."""
import numpy as np

D, TOKENS, BLOCK = 128, 32, 4416


def _places():
    """(byte, shift) of every code of a block: keys and values, [32, 128] each."""
    kb, ksh = np.zeros((TOKENS, D), np.int64), np.zeros((TOKENS, D), np.int64)
    vb, vsh = np.zeros((TOKENS, D), np.int64), np.zeros((TOKENS, D), np.int64)
    for n in range(4):
        for g in range(8):
            for cq in range(4):
                for e in range(32):                       # keys: dimensions 32cq .. 32cq + 31 in a piece
                    kb[8 * n + g, 32 * cq + e] = ((n * 4 + cq) * 8 + (g ^ 2 * cq)) * 16 + e // 2
                    ksh[8 * n + g, 32 * cq + e] = 4 * (e % 2)
    for w in range(4):
        for g in range(8):
            for cq in range(4):
                for n in range(4):
                    for h in range(2):
                        for j in range(4):                # values: four dimensions of a token in 16 bits
                            t, d = 8 * n + 2 * cq + h, 32 * w + 4 * g + j
                            vb[t, d] = 2048 + ((w * 4 + cq) * 8 + (g ^ 2 * cq)) * 16 + 4 * n + 2 * h + j // 2
                            vsh[t, d] = 4 * (j % 2)
    return kb, ksh, vb, vsh


KB, KSH, VB, VSH = _places()


def unpack_blocks(blocks):
    """uint8 [..., 4416] -> key codes, scales, zeros, value codes, scales, zeros: [..., 32, 128] and [..., 32]."""
    f = lambda at: np.ascontiguousarray(blocks[..., at:at + 128]).view(np.float32)  # noqa: E731
    return ((blocks[..., KB] >> KSH.astype(np.uint8)) & 15, f(4096), blocks[..., 4352:4384],
            (blocks[..., VB] >> VSH.astype(np.uint8)) & 15, f(4224), blocks[..., 4384:4416])


def token_bytes(t):
    """The 138 bytes of token t of a block, in the same order for every token: a byte holds two neighbouring dimensions."""
    return np.concatenate([KB[t, ::2], VB[t, ::2], 4096 + 4 * t + np.arange(4), 4224 + 4 * t + np.arange(4), [4352 + t], [4384 + t]])


def cached(pool, table, page_tokens, r, length):
    """Codes, scales and zeros of positions 0 .. length - 1 of request r, [length, H, ...]; positions without a page are NaN scales."""
    num_pages, H = pool.shape[:2]
    out = [np.zeros((length, H, D), np.uint8), np.full((length, H), np.nan, np.float32), np.zeros((length, H), np.uint8),
           np.zeros((length, H, D), np.uint8), np.full((length, H), np.nan, np.float32), np.zeros((length, H), np.uint8)]
    for i in range(-(-length // page_tokens)):
        page = int(table[r, i]) if i < table.shape[1] else -1
        if not 0 <= page < num_pages:
            continue
        parts = unpack_blocks(pool[page].reshape(H, page_tokens // TOKENS, BLOCK))
        n = min(page_tokens, length - i * page_tokens)
        for o, x in zip(out, parts):                      # [H, blocks, 32, ...] -> [tokens, H, ...]
            x = np.moveaxis(x.reshape(H, page_tokens, *x.shape[3:]), 0, 1)
            o[i * page_tokens:i * page_tokens + n] = x[:n]
    return out


def dequant(code, scale, zero):
    return scale.astype(np.float64)[..., None] * (code.astype(np.float64) - zero.astype(np.float64)[..., None])


HAD = np.array([[(-1.0) ** bin(i & j).count("1") for j in range(D)] for i in range(D)])


def rotate(x, block):
    if block <= 1:
        return x.astype(np.float64)
    return (x.reshape(*x.shape[:-1], D // block, block).astype(np.float64) @ (HAD[:block, :block] / np.sqrt(block))).reshape(x.shape)


def attention(q, pool, table, page_tokens, row_start, first, mask=None, q_had=0, scale=None):
    """-> (out fp64 [total, Hq, D], the largest sum of |q k| over a row's tokens times scale, the largest |v| it sees)."""
    total, Hq, _ = q.shape
    H = pool.shape[1]
    G = Hq // H
    scale = 1.0 / np.sqrt(D) if scale is None else scale
    qr = rotate(q, q_had)
    out, size, top = np.zeros((total, Hq, D)), np.zeros((total, Hq)), np.zeros((total, Hq))
    for r in range(len(first)):
        n, f = int(row_start[r + 1] - row_start[r]), int(first[r])
        length = max(0, min(f + n, table.shape[1] * page_tokens))
        if n <= 0 or length == 0:
            continue
        parts = cached(pool, table, page_tokens, r, length)
        have = ~np.isnan(parts[1][:, 0]) | (np.array([0 <= int(table[r, t // page_tokens]) < pool.shape[0] for t in range(length)]))
        k, v = dequant(*parts[:3]), dequant(*parts[3:])
        t = np.arange(length)
        for i in range(n):
            row = int(row_start[r]) + i
            j = t - f
            if mask is None:
                seen = j <= i
            else:
                bits = mask[row].view(np.uint32)
                jj = np.clip(j, 0, 32 * bits.size - 1)
                seen = (j < 0) | ((j < 32 * bits.size) & ((bits[jj >> 5] >> (jj & 31).astype(np.uint32)) & 1 == 1))
            seen &= have
            if not seen.any():
                continue
            for h in range(Hq):
                kk, vv = k[seen, h // G], v[seen, h // G]
                s = kk @ qr[row, h] * scale
                p = np.exp(s - s.max())
                out[row, h] = p @ vv / p.sum()
                size[row, h] = (np.abs(kk) @ np.abs(qr[row, h])).max() * scale
                top[row, h] = np.abs(vv).max()
    return out, size, top


def tree_mask(parents, words):
    """int32 [n, words]: bit j of row i when drafted token j is i or one of its ancestors."""
    m = np.zeros((len(parents), words), np.uint32)
    for i, p in enumerate(parents):
        if p >= 0:
            m[i] = m[p]
        m[i, i >> 5] |= np.uint32(1 << (i & 31))
    return m.view(np.int32)
