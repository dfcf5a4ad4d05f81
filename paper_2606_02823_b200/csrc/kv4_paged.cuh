// Paged KV4 cache of many requests: written (quantized) and read back a block of tokens at a time, and the tokens that
// survive the check of a drafted tree moved to the front.
//
// A block is 32 consecutive tokens of one KV head, 4416 contiguous bytes (138 per token):
//      0  key codes      16-byte pieces [n 4][cq 4][g ^ 2cq 8]; token 8n + g, dimensions 32cq .. 32cq + 31, 4 bits each in order
//   2048  value codes    16-byte pieces [w 4][cq 4][g ^ 2cq 8], 16-bit units [n 4][h 2]; token 8n + 2cq + h, dimensions
//                        32w + 4g .. 32w + 4g + 3, 4 bits each in order
//   4096  key scales     fp32, by token        4352  key zero-points    one byte, by token
//   4224  value scales   fp32, by token        4384  value zero-points  one byte, by token
// The order serves the attention that reads it (kv4_tree.cuh): a 16-byte piece is what one lane needs next, `word & 0x000f000f`
// of it is a pair of operands of the product it feeds (keys: two dimensions of a token, values: two tokens of a dimension), and
// the exclusive-or spreads a warp's 128-bit reads over all banks for both ways the pieces are read.  Every byte belongs to one
// token, so tokens are written without reading their neighbours.
#pragma once

#include "common.cuh"
#include "kv4.cuh"

namespace qift {

constexpr int kPgTokens = 32;        // tokens of a block
constexpr int kPgV = 2048, kPgKs = 4096, kPgVs = 4224, kPgKz = 4352, kPgVz = 4384;
constexpr int kPgBlock = 4416;
constexpr int kPgThreads = 256;
constexpr int kPgGroups = kPgThreads / 8;   // a vector is handled by eight lanes, 16 dimensions each
constexpr int kPgMaxHeads = 8;              // KV heads of one CTA

struct KvPages {
    uint8_t* pool;          // [num_pages][H][page_tokens / 32][4416]
    const int32_t* table;   // [R][max_pages]
    int num_pages, max_pages, page_tokens, H;
    // The block that holds `position` of request r and KV head h; nullptr when no page of the pool does.
    __device__ __forceinline__ uint8_t* block(int r, int position, int h) const {
        const int slot = position / page_tokens;
        const int page = table[static_cast<size_t>(r) * max_pages + slot];
        if (static_cast<unsigned>(page) >= static_cast<unsigned>(num_pages)) return nullptr;
        const int inner = (position - slot * page_tokens) / kPgTokens;
        return pool + ((static_cast<size_t>(page) * H + h) * (page_tokens / kPgTokens) + inner) * kPgBlock;
    }
    __device__ __forceinline__ int capacity() const {   // positions a request can have
        return static_cast<int>(min(static_cast<long long>(max_pages) * page_tokens, 0x7fffffe0ll));
    }
};

struct KvRows {                 // the ragged rows of a call
    const int32_t* row_start;   // [R + 1]
    const int32_t* first;       // [R] cache position of a request's first row
    int R, total;               // requests, rows that the caller's arrays hold
    __device__ __forceinline__ int begin(int r) const { return max(0, row_start[r]); }
    __device__ __forceinline__ int count(int r) const { return max(0, min(total, row_start[r + 1]) - begin(r)); }
    // positions of request r that exist in the cache: [lo, hi)
    __device__ __forceinline__ void span(int r, int capacity, int& lo, int& hi) const {
        const int f = first[r];
        const long long end = static_cast<long long>(f) + count(r);
        lo = max(f, 0);
        hi = static_cast<int>(min(end, static_cast<long long>(capacity)));
    }
};

// Which request the CTA's item belongs to, when request r has `items(r)` of them: a scan over the requests, blockDim of them a
// trip.  Returns the request (-1: no such item) and the item's number within it.
template <typename Items>
__device__ __forceinline__ int kv_find_request(int item, int R, int& inner, Items items) {
    __shared__ int warp_sum[32];
    __shared__ int found[2];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5;
    if (tid == 0) found[0] = -1;
    int before = 0;
    for (int base = 0; base < R; base += blockDim.x) {
        const int r = base + tid;
        const int n = r < R ? items(r) : 0;
        int scan = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int up = __shfl_up_sync(0xffffffffu, scan, o);
            if (lane >= o) scan += up;
        }
        if (lane == 31) warp_sum[warp] = scan;
        __syncthreads();
        int mine = before;
        for (int w = 0; w < warps; ++w) {
            if (w < warp) mine += warp_sum[w];
            before += warp_sum[w];
        }
        mine += scan - n;
        if (n > 0 && item >= mine && item < mine + n) found[0] = r, found[1] = item - mine;
        __syncthreads();
        if (before > item) break;   // the same for every thread
    }
    __syncthreads();
    inner = found[1];
    return found[0];
}

// Two fp32 operations in one instruction, each rounded on its own: a pair of values in a 64-bit register.
__device__ __forceinline__ uint64_t pair_of(float x, float y) {
    uint64_t p;
    asm("mov.b64 %0, {%1, %2};" : "=l"(p) : "f"(x), "f"(y));
    return p;
}
__device__ __forceinline__ void pair_to(uint64_t p, float& x, float& y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(p)); }
__device__ __forceinline__ uint64_t pair_add(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ uint64_t pair_mul(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ uint64_t pair_fma(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}

// In-place butterfly over the 128 values of a vector in eight lanes (value index 16 * l + e), strides below had_block; natural
// order, the same operands as everywhere else in this library.  had_block may differ between the groups of a warp.  A difference is
// taken as -1 * b + a in one rounding.
template <bool FULL>   // had_block is 128 in every lane
__device__ __forceinline__ void kv_rotate16_as(float (&v)[16], int l, int had, float inv_sqrt_b) {
    const int had_block = FULL ? kKvD : had;
    if (1 < had_block) {
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
            const float a = v[e], b = v[e + 1];
            v[e] = __fadd_rn(a, b), v[e + 1] = __fsub_rn(a, b);
        }
    }
    uint64_t p[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) p[e] = pair_of(v[2 * e], v[2 * e + 1]);
    const uint64_t minus = pair_of(-1.0f, -1.0f);
#pragma unroll
    for (int h = 1; h < 8; h <<= 1) {
        if (2 * h < had_block) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (!(e & h)) {
                    const uint64_t a = p[e], b = p[e + h];
                    p[e] = pair_add(a, b), p[e + h] = pair_fma(b, minus, a);
                }
        }
    }
#pragma unroll
    for (int h = 16; h < kKvD; h <<= 1) {
        const float sign = (l & (h >> 4)) ? -1.0f : 1.0f;   // upper element: other - v, lower: other + v, one rounding
        const uint64_t signs = pair_of(sign, sign);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint64_t other = __shfl_xor_sync(0xffffffffu, static_cast<unsigned long long>(p[e]), h >> 4);
            if (h < had_block) p[e] = pair_fma(signs, p[e], other);
        }
    }
    if (had_block > 1) {
        const uint64_t inv = pair_of(inv_sqrt_b, inv_sqrt_b);
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] = pair_mul(p[e], inv);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) pair_to(p[e], v[2 * e], v[2 * e + 1]);
}
__device__ __forceinline__ void kv_rotate16(float (&v)[16], int l, int had_block, float inv_sqrt_b) {
    if (__all_sync(0xffffffffu, had_block == kKvD)) kv_rotate16_as<true>(v, l, had_block, inv_sqrt_b);
    else if (__any_sync(0xffffffffu, had_block > 1)) kv_rotate16_as<false>(v, l, had_block, inv_sqrt_b);
}

// Sixteen values per lane of an eight-lane group -> sixteen 4-bit codes (value e at bits 4e), scale and zero-point; the fp32 steps
// of kv4_quantize_vector.  A code is rint(x / s): the quotient is taken as x times 1 / s, whose rounding can differ only within
// 2^-17 of a half for quotients up to 32 (beyond, the code is clamped either way); there, and where it is not a number, the
// division decides.
__device__ __forceinline__ uint2 kv_quantize16(const float (&v)[16], float clip, float& s, float& z) {
    float mn = 0.0f, mx = 0.0f;
#pragma unroll
    for (int e = 0; e < 16; ++e) mn = fminf(mn, v[e]), mx = fmaxf(mx, v[e]);
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) {
        mn = fminf(mn, __shfl_xor_sync(0xffffffffu, mn, o));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
    }
    const float lo = __fmul_rn(mn, clip), hi = __fmul_rn(mx, clip);
    s = 1.0f, z = 0.0f;
    if (hi != lo) {
        s = __fdiv_rn(__fsub_rn(hi, lo), 15.0f);
        if (s > 0.0f) z = rintf(__fdiv_rn(-lo, s));
        else s = 1.0f;   // a range below 15 times the smallest fp32 number has no scale: every code 0, like the empty range
    }
    const int zi = static_cast<int>(z);
    constexpr float kRound = 12582912.0f;   // 1.5 * 2^23: the sum's low mantissa bits are the nearest integer, ties to even
    const float inv = __fdiv_rn(1.0f, s);
    const int bias = zi - 0x4b400000;
    uint32_t w[2] = {0u, 0u};
    // beyond 2^21 (tiny clipping ratios, values that are no numbers) the sum's bits are not the integer's
    bool near = !(fmaxf(-mn, mx) * inv <= 0x1p21f);
    const uint64_t inv2 = pair_of(inv, inv), round2 = pair_of(kRound, kRound), back2 = pair_of(-kRound, -kRound), minus = pair_of(-1.0f, -1.0f);
#pragma unroll
    for (int e = 0; e < 16; e += 2) {
        const uint64_t y = pair_mul(pair_of(v[e], v[e + 1]), inv2), t = pair_add(y, round2);
        float t0, t1, d0, d1;
        pair_to(t, t0, t1);
        pair_to(pair_fma(pair_add(t, back2), minus, y), d0, d1);   // what the rounding took
        near |= !(fabsf(d0) <= 0.5f - 0x1p-16f) || !(fabsf(d1) <= 0.5f - 0x1p-16f);
        w[e >> 3] |= static_cast<uint32_t>(max(0, min(15, __float_as_int(t0) + bias))) << (4 * (e & 7));
        w[e >> 3] |= static_cast<uint32_t>(max(0, min(15, __float_as_int(t1) + bias))) << (4 * (e & 7) + 4);
    }
    if (near) {
        w[0] = w[1] = 0u;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int c = max(0, min(15, min(__float2int_rn(__fdiv_rn(v[e], s)), 15) + zi));   // 2^31 - 1, of any larger quotient, plus zi would wrap
            w[e >> 3] |= static_cast<uint32_t>(c) << (4 * (e & 7));
        }
    }
    return make_uint2(w[0], w[1]);
}

// Byte offsets of lane l's codes of a token in its block: keys 8 bytes; values four 16-bit units at +0, +16 * step ... (pieces
// differ in g only, so the exclusive-or is applied per unit).
__device__ __forceinline__ int kv_key_offset(int token, int l) {
    const int n = token >> 3, g = token & 7, cq = l >> 1;
    return ((n * 4 + cq) * 8 + (g ^ (2 * cq))) * 16 + (l & 1) * 8;
}
__device__ __forceinline__ int kv_value_offset(int token, int l, int u) {
    const int n = token >> 3, cq = (token >> 1) & 3, w = l >> 1, g = 4 * (l & 1) + u;
    return kPgV + ((w * 4 + cq) * 8 + (g ^ (2 * cq))) * 16 + n * 4 + (token & 1) * 2;
}

// Sixteen values of a lane as they stand in memory, and in fp32.
template <bool BF16>
struct Kv16 {
    uint4 raw[BF16 ? 2 : 4];
    __device__ __forceinline__ void load(const void* X, size_t offset) {
        const uint4* p = reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(X) + offset * (BF16 ? 2 : 4));
#pragma unroll
        for (int i = 0; i < (BF16 ? 2 : 4); ++i) raw[i] = p[i];
    }
    __device__ __forceinline__ void get(float (&v)[16]) const {
#pragma unroll
        for (int i = 0; i < (BF16 ? 2 : 4); ++i) {
            const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if constexpr (BF16) v[8 * i + 2 * k] = __uint_as_float(w[k] << 16), v[8 * i + 2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
                else v[4 * i + k] = __uint_as_float(w[k]);
            }
        }
    }
};
template <bool BF16>
__device__ __forceinline__ void kv_load16(const void* X, size_t offset, float (&v)[16]) {
    Kv16<BF16> x;
    x.load(X, offset);
    x.get(v);
}
template <bool BF16>
__device__ __forceinline__ void kv_store16(void* X, size_t offset, const float (&v)[16]) {
    if constexpr (BF16) {
        uint4* p = reinterpret_cast<uint4*>(static_cast<uint16_t*>(X) + offset);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            uint32_t w[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const __nv_bfloat162 b = __floats2bfloat162_rn(v[8 * i + 2 * k], v[8 * i + 2 * k + 1]);
                w[k] = *reinterpret_cast<const uint32_t*>(&b);
            }
            p[i] = make_uint4(w[0], w[1], w[2], w[3]);
        }
    } else {
        float4* p = reinterpret_cast<float4*>(static_cast<float*>(X) + offset);
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
    }
}

struct KvMoveParams {
    KvPages pages;
    KvRows rows;
    void* K;             // [total][H][128] with a row stride; in for the write, out for the read (either may be null there)
    void* V;
    long long k_stride, v_stride;   // elements
    int k_had, v_had;
    float k_inv_sqrt, v_inv_sqrt, clip;
    int heads;           // KV heads of a CTA
};

// An item is a block that rows of the call fall into; grid (items, H / heads).
__device__ __forceinline__ int kv_find_block(const KvMoveParams& p, int& lo, int& hi) {
    const int cap = p.pages.capacity();
    int inner;
    const int r = kv_find_request(blockIdx.x, p.rows.R, inner, [&](int q) {
        int a, b;
        p.rows.span(q, cap, a, b);
        return a < b ? (b - 1) / kPgTokens - a / kPgTokens + 1 : 0;
    });
    if (r < 0) return -1;
    int a, b;
    p.rows.span(r, cap, a, b);
    const int base = (a / kPgTokens + inner) * kPgTokens;
    lo = max(a, base), hi = min(b, base + kPgTokens);
    return r;
}

// Rows -> codes.  Groups of eight lanes take vectors (head, token; all keys, then all values).  Blocks are put together in shared
// memory: a whole one leaves in 16-byte stores, of a part the keys leave in 16 bytes, the values in pairs of tokens (4 bytes) or
// alone (2).  One or two tokens go straight to their places.
// Bound by instruction issue (68 % of the slots; about 459 warp instructions for four vectors, most of them the rotation and the
// quantizer): 9873 tokens x 8 heads, bf16: 28 us, 46 with the read of them (103 MB in all).
template <bool BF16>
__global__ void __launch_bounds__(kPgThreads)
kv4_paged_write_kernel(const KvMoveParams p) {
    __shared__ alignas(16) uint8_t image[kPgMaxHeads][kPgBlock];
    pdl_launch_dependents();
    pdl_wait();
    int lo, hi;
    const int r = kv_find_block(p, lo, hi);
    if (r < 0) return;
    const int h0 = blockIdx.y * p.heads, heads = min(p.heads, p.pages.H - h0);
    uint8_t* block0 = p.pages.block(r, lo, h0);
    if (!block0) return;
    const size_t head_step = static_cast<size_t>(p.pages.page_tokens / kPgTokens) * kPgBlock;
    const int n = hi - lo, vectors = n * heads;
    const bool whole = n == kPgTokens, direct = n < 3;
    const int l = threadIdx.x & 7, group = threadIdx.x >> 3;
    const long long row0 = p.rows.begin(r) + (static_cast<long long>(lo) - p.rows.first[r]);
    // vector i: the first half are keys, the second values; within, token by token of head by head
    auto where = [&](int i, bool& is_v, int& h, int& t) {
        is_v = i >= vectors;
        const int j = i < 2 * vectors ? (is_v ? i - vectors : i) : 0;
        h = j / n, t = j - h * n;
    };
    Kv16<BF16> ahead;                    // the next vector's values are on their way while one is quantized
    auto fetch = [&](int i) {
        bool is_v;
        int h, t;
        where(i, is_v, h, t);
        ahead.load(is_v ? p.V : p.K, static_cast<size_t>((row0 + t) * (is_v ? p.v_stride : p.k_stride)) + (h0 + h) * kKvD + 16 * l);
    };
    // the trip count is the same for the four groups of a warp: shuffles are executed by all lanes
    if ((group & ~3) < 2 * vectors) fetch(group);
    for (int base = group & ~3; base < 2 * vectors; base += kPgGroups) {
        const int i = base + (group & 3);
        const bool on = i < 2 * vectors;
        bool is_v;
        int h, t;
        where(i, is_v, h, t);
        float v[16];
        ahead.get(v);
        if (base + kPgGroups < 2 * vectors) fetch(i + kPgGroups);
        kv_rotate16(v, l, is_v ? p.v_had : p.k_had, is_v ? p.v_inv_sqrt : p.k_inv_sqrt);
        float s, z;
        const uint2 c = kv_quantize16(v, p.clip, s, z);
        if (!on) continue;
        uint8_t* dst = direct ? block0 + h * head_step : image[h];
        const int token = (lo + t) % kPgTokens;
        if (is_v) {
#pragma unroll
            for (int u = 0; u < 4; ++u)
                *reinterpret_cast<uint16_t*>(dst + kv_value_offset(token, l, u)) = static_cast<uint16_t>((u < 2 ? c.x : c.y) >> (16 * (u & 1)));
        } else {
            *reinterpret_cast<uint2*>(dst + kv_key_offset(token, l)) = c;
        }
        if (l == 0) {
            reinterpret_cast<float*>(dst + (is_v ? kPgVs : kPgKs))[token] = s;
            dst[(is_v ? kPgVz : kPgKz) + token] = static_cast<uint8_t>(static_cast<int>(z));
        }
    }
    if (direct) return;
    __syncthreads();
    if (whole) {
        for (int i = threadIdx.x; i < heads * (kPgBlock / 16); i += kPgThreads) {
            const int h = i / (kPgBlock / 16), k = i - h * (kPgBlock / 16);
            reinterpret_cast<uint4*>(block0 + h * head_step)[k] = reinterpret_cast<const uint4*>(image[h])[k];
        }
        return;
    }
    const int first = lo % kPgTokens;
    auto in = [&](int token) { return static_cast<unsigned>(token - first) < static_cast<unsigned>(n); };
    for (int h = 0; h < heads; ++h) {
        uint8_t* to = block0 + h * head_step;
        for (int i = threadIdx.x; i < 128 + 512 + 4 * kPgTokens; i += kPgThreads) {
            if (i < 128) {                       // a piece of keys: one token
                const int cq = (i >> 3) & 3, token = 8 * (i >> 5) + ((i & 7) ^ (2 * cq));
                if (in(token)) reinterpret_cast<uint4*>(to)[i] = reinterpret_cast<const uint4*>(image[h])[i];
            } else if (i < 128 + 512) {          // a word of values: two tokens
                const int k = i - 128, cq = (k >> 5) & 3, token = 8 * (k & 3) + 2 * cq;
                const uint32_t word = reinterpret_cast<const uint32_t*>(image[h] + kPgV)[k];
                if (in(token) && in(token + 1)) reinterpret_cast<uint32_t*>(to + kPgV)[k] = word;
                else if (in(token)) reinterpret_cast<uint16_t*>(to + kPgV)[2 * k] = static_cast<uint16_t>(word);
                else if (in(token + 1)) reinterpret_cast<uint16_t*>(to + kPgV)[2 * k + 1] = static_cast<uint16_t>(word >> 16);
            } else {
                const int k = (i - 128 - 512) / kPgTokens, token = i % kPgTokens;
                if (!in(token)) continue;
                if (k < 2) reinterpret_cast<uint32_t*>(to + (k ? kPgVs : kPgKs))[token] = reinterpret_cast<const uint32_t*>(image[h] + (k ? kPgVs : kPgKs))[token];
                else to[(k == 3 ? kPgVz : kPgKz) + token] = image[h][(k == 3 ? kPgVz : kPgKz) + token];
            }
        }
    }
}

// Codes -> rows: scale * (code - zero), rotated back on request.
// 3339 tokens x 32 heads, fp32 (124 MB, most of it written): 36 us, 3.5 TB/s, 64 % of the L1 and shared-memory path (the 16-bit reads of
// value codes; warps wait for its queue more than for anything else) and 41 % of the issue slots.
template <bool BF16>
__global__ void __launch_bounds__(kPgThreads)
kv4_paged_read_kernel(const KvMoveParams p) {
    __shared__ alignas(16) uint8_t image[kPgMaxHeads][kPgBlock];
    pdl_launch_dependents();
    pdl_wait();
    int lo, hi;
    const int r = kv_find_block(p, lo, hi);
    if (r < 0) return;
    const int h0 = blockIdx.y * p.heads, heads = min(p.heads, p.pages.H - h0);
    const uint8_t* block0 = p.pages.block(r, lo, h0);
    if (!block0) return;
    const size_t head_step = static_cast<size_t>(p.pages.page_tokens / kPgTokens) * kPgBlock;
    const int n = hi - lo, vectors = n * heads;
    const bool staged = n >= 8;   // below that, the tokens' own bytes are less than the block
    if (staged) {
        for (int i = threadIdx.x; i < heads * (kPgBlock / 16); i += kPgThreads) {
            const int h = i / (kPgBlock / 16), k = i - h * (kPgBlock / 16);
            reinterpret_cast<uint4*>(image[h])[k] = reinterpret_cast<const uint4*>(block0 + h * head_step)[k];
        }
        __syncthreads();
    }
    const int l = threadIdx.x & 7, group = threadIdx.x >> 3;
    const long long row0 = p.rows.begin(r) + (static_cast<long long>(lo) - p.rows.first[r]);
    for (int base = group & ~3; base < 2 * vectors; base += kPgGroups) {
        const int i = base + (group & 3);
        const bool is_v = i >= vectors;
        void* X = is_v ? p.V : p.K;
        const bool on = i < 2 * vectors && X != nullptr;
        const int j = on ? (is_v ? i - vectors : i) : 0;
        const int h = j / n, t = j - h * n, token = (lo + t) % kPgTokens;
        const uint8_t* src = staged ? image[h] : block0 + h * head_step;
        uint32_t w[2];
        if (is_v) {
            uint32_t u4[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) u4[u] = *reinterpret_cast<const uint16_t*>(src + kv_value_offset(token, l, u));
            w[0] = u4[0] | u4[1] << 16, w[1] = u4[2] | u4[3] << 16;
        } else {
            const uint2 c = *reinterpret_cast<const uint2*>(src + kv_key_offset(token, l));
            w[0] = c.x, w[1] = c.y;
        }
        const float s = reinterpret_cast<const float*>(src + (is_v ? kPgVs : kPgKs))[token];
        // a code under the exponent of 2^23 is 2^23 + code: less 2^23 + zero it is code - zero, exactly
        const float z = -(8388608.0f + static_cast<float>(src[(is_v ? kPgVz : kPgKz) + token]));
        const uint64_t z2 = pair_of(z, z), s2 = pair_of(s, s);
        float v[16];
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
            const uint32_t c0 = ((w[e >> 3] >> (4 * (e & 7))) & 15u) | 0x4b000000u, c1 = ((w[e >> 3] >> (4 * (e & 7) + 4)) & 15u) | 0x4b000000u;
            pair_to(pair_mul(pair_add(pair_of(__uint_as_float(c0), __uint_as_float(c1)), z2), s2), v[e], v[e + 1]);
        }
        kv_rotate16(v, l, is_v ? p.v_had : p.k_had, is_v ? p.v_inv_sqrt : p.k_inv_sqrt);
        if (on) kv_store16<BF16>(X, static_cast<size_t>((row0 + t) * (is_v ? p.v_stride : p.k_stride)) + (h0 + h) * kKvD + 16 * l, v);
    }
}

// Slot first + i <- slot first + keep[i], i = 0 .. kept - 1: one warp per request and head, eight tokens read before any of them
// is written.  The indices ascend, so a slot is never written before the tokens that come from it are read, and a lane only ever
// reads and writes its own share of every token.
// Bound by its chain of dependent loads (request, indices, pages, tokens), once for every eight tokens: 4 requests of up to 12 drafted
// tokens 6.1 us, 192 of up to 64 16 us.
constexpr int kPgKeepAhead = 8;
__global__ void __launch_bounds__(kPgThreads)
kv4_paged_keep_kernel(const KvPages pages, const KvRows rows, const int32_t* __restrict__ keep, const int32_t* __restrict__ kept_start) {
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31;
    const long long w = static_cast<long long>(blockIdx.x) * (kPgThreads / 32) + (threadIdx.x >> 5);
    if (w >= static_cast<long long>(rows.R) * pages.H) return;
    const int r = static_cast<int>(w / pages.H), h = static_cast<int>(w - static_cast<long long>(r) * pages.H);
    const int begin = rows.begin(r), n = rows.count(r), first = rows.first[r], cap = pages.capacity();
    const int kept = min(n, kept_start[r + 1] - kept_start[r]);
    auto place = [&](int draft) -> uint8_t* {   // the block of a drafted token, nullptr when it has no place
        const long long pos = static_cast<long long>(first) + draft;
        if (draft < 0 || draft >= n || pos < 0 || pos >= cap) return nullptr;
        return pages.block(r, static_cast<int>(pos), h);
    };
    const int l = lane >> 2, u = lane & 3;   // value unit of this lane; key bytes 2 * lane, + 1
    for (int i0 = 0; i0 < kept; i0 += kPgKeepAhead) {
        uint16_t kc[kPgKeepAhead], vc[kPgKeepAhead];
        uint32_t extra[kPgKeepAhead];
        bool have[kPgKeepAhead];
        uint8_t* to[kPgKeepAhead];   // (looked up while the indices are on their way)
        int from_of[kPgKeepAhead];
#pragma unroll
        for (int i = 0; i < kPgKeepAhead; ++i) from_of[i] = i0 + i < kept ? keep[begin + i0 + i] : -1;
#pragma unroll
        for (int i = 0; i < kPgKeepAhead; ++i) to[i] = i0 + i < kept ? place(i0 + i) : nullptr;
#pragma unroll
        for (int i = 0; i < kPgKeepAhead; ++i) {
            const int from = from_of[i];
            const uint8_t* b = place(from);
            have[i] = b != nullptr;
            kc[i] = vc[i] = 0, extra[i] = 0;
            if (!have[i]) continue;
            const int token = (first + from) % kPgTokens;
            kc[i] = *reinterpret_cast<const uint16_t*>(b + kv_key_offset(token, l) + 2 * u);
            vc[i] = *reinterpret_cast<const uint16_t*>(b + kv_value_offset(token, l, u));
            if (lane == 0) extra[i] = reinterpret_cast<const uint32_t*>(b + kPgKs)[token];
            if (lane == 1) extra[i] = reinterpret_cast<const uint32_t*>(b + kPgVs)[token];
            if (lane == 2) extra[i] = b[kPgKz + token];
            if (lane == 3) extra[i] = b[kPgVz + token];
        }
#pragma unroll
        for (int i = 0; i < kPgKeepAhead; ++i) {
            uint8_t* b = to[i];
            if (!b || !have[i]) continue;
            const int token = (first + i0 + i) % kPgTokens;
            *reinterpret_cast<uint16_t*>(b + kv_key_offset(token, l) + 2 * u) = kc[i];
            *reinterpret_cast<uint16_t*>(b + kv_value_offset(token, l, u)) = vc[i];
            if (lane == 0) reinterpret_cast<uint32_t*>(b + kPgKs)[token] = extra[i];
            if (lane == 1) reinterpret_cast<uint32_t*>(b + kPgVs)[token] = extra[i];
            if (lane == 2) b[kPgKz + token] = static_cast<uint8_t>(extra[i]);
            if (lane == 3) b[kPgVz + token] = static_cast<uint8_t>(extra[i]);
        }
    }
}

}  // namespace qift
