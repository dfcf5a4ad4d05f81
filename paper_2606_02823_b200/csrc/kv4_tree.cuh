// Attention of drafted token trees over the paged KV4 cache.
//
// The rows of a request that one KV head serves are its n drafted tokens times the G query heads of the head, in tiles of ROWS.  A
// work item is one 32-token block for one (request, KV head, row tile); the items of the whole call, in that order, are dealt to
// the warps of the grid in equal contiguous runs, whatever the requests' lengths.  A warp works alone: its own ring of blocks in
// shared memory (one 4416-byte bulk copy each), its own running maximum, sum and numerator.  A tile that lies within one warp's run
// is finished there; the pieces of the others go to the workspace -- a warp has at most two, its first and its last -- and the
// second kernel joins them, one CTA for the tile that begins in a warp and ends in a later one.
//
// Both products run on mma.sync.m16n8k16 (fp16, fp32 sums) with the codes as A and eight query rows as the columns:
//   S[token][row] = sum_d kc[token][d] q[row][d],        O[d][row] += sum_t vc[t][d] w[t][row],  w = p * vs.
// A code c in the low mantissa bits of an fp16 number is the subnormal c * 2^-24, exactly: `word & 0x000f000f` IS a pair of
// operands, `word & 0x00f000f0` one of 16 c * 2^-24 (the 16 is taken out of the query, and out of the result).  Scores come out
// with a lane holding four tokens of two rows, and movmatrix turns the packed weights into the columns of the second product.
// Zero-points enter as one more k-step (key zeros against query sums) and one more row tile (value zeros against weights), so they
// cancel against the same rounded operands.
//   q is scaled by a power of two per row (largest value 2^7 .. 2^8) and held in fp16: exact for bf16 queries that are not
//   rotated, else off by 2^-12.  fp32 calls hold q and w in two fp16 parts each (residual 2^-22), multiplied one after the other
//   into the same sums, and all codes lessened by 8 (1024 + c - 1032 in fp16, exact): the sums of an average over many tokens
//   would otherwise be far larger than the result and lose what the zero-points take away.
//   w = 2^(score - R) vs, and the sum of 2^(score - R) beside it, go by one reference point R for each row: a bound of score + log2(vs)
//   over the tokens that the row has seen, so a large value scale counts with its weight, and for the rows that see it alone.  R
//   moves (by whole binary orders, so nothing is rounded) only when a token exceeds it by more than kTreeSlack.
// Bound by latency and instruction issue: about 507 warp instructions a block with eight rows, 722 with sixteen, on 59 and 44 % of the
// issue slots, which is what 16 and 12 warps an SM (128 and 168 registers a thread) keep busy.  32 query and 8 KV heads: 64 single tokens
// over 8000 cached ones each (286 MB) 62.5 us = 4.6 TB/s; 16 trees of up to 13 tokens over 6000 (67 MB, read again by every tile) 67 us.
#pragma once

#include <type_traits>

#include "kv4_paged.cuh"

namespace qift {

struct KvTreeParams {
    KvPages pages;
    KvRows rows;
    const void* q;           // [total][Hq][128], rows q_stride elements apart
    void* out;               // [total][Hq][128], contiguous
    const int32_t* mask;     // [total][mask_words] or nullptr: a drafted token sees the drafted ones up to itself
    int mask_words;
    long long q_stride;
    int Hq, G;               // query heads, query heads per KV head
    int q_had;
    float q_inv_sqrt, scale_log2;   // score scale times log2(e)
    int4* desc;              // [warps]: tile that begins in this warp's run and ends in a later one's: request, head, tile, pieces
    float* partial;          // [2 * warps][ROWS][kTreeRow]
};

constexpr int kTreeRow = 132;        // floats of a row's piece: numerator, reference point, sum, two unused
constexpr int kTreeMinRun = 1;       // items of a run at least (mma.sync, one token over 1023 cached ones: 1: 13.4 us, 2: 15.7, 4: 21.0)
constexpr float kTreeSlack = 6.0f;   // binary orders that a weight may exceed its reference by: w * 2^8 stays below 2^14
constexpr int kTreeVexp = 40;        // exponent field that smaller value scales count with: sums of 2^(score - R) stay below 2^100 a token
constexpr int kTreeSite = 48;        // site of an expired wait

// As mbar_wait, for waits that are short and mostly over when they begin: a loop of four instructions, bounded by its trips, each of
// which the hardware parks for 4 us (measured: 64 trips 253.5 us).
constexpr uint32_t kNearTripNs = 4000;
constexpr uint32_t kNearTrips = static_cast<uint32_t>(kWaitLimitNs / kNearTripNs);
__device__ __forceinline__ bool mbar_wait_near(uint64_t* bar, uint32_t parity, unsigned int site, uint32_t trips = kNearTrips) {
    uint32_t left = trips;
    asm volatile(
        "{\n\t.reg .pred p;\n"
        "NEAR_AGAIN:\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "@p bra NEAR_DONE;\n\t"
        "add.u32 %0, %0, 0xffffffff;\n\t"
        "setp.ne.u32 p, %0, 0;\n\t"
        "@p bra NEAR_AGAIN;\n"
        "NEAR_DONE:\n\t}"
        : "+r"(left) : "r"(smem_u32(bar)), "r"(parity) : "memory");
    if (left == 0) report_timeout(site);
    return left != 0;
}

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// x * 2^d for whole d <= 0, in two steps: sums of weights go by reference points up to 212 binary orders apart (tokens whose values are
// next to nothing beside the largest), and a factor below 2^-126 would be 0.  (Numerators of that size do vanish beside the others.)
__device__ __forceinline__ float times_ex2(float x, float d) {
    const float most = fmaxf(d, -100.0f);
    return x * ex2(most) * ex2(d - most);
}

__device__ __forceinline__ uint32_t lessened(uint32_t x, uint32_t by) {   // fp16 pairs, x + by
    uint32_t y;
    asm("add.rn.f16x2 %0, %1, %2;" : "=r"(y) : "r"(x), "r"(by));
    return y;
}

// The power of two above a value scale, as its exponent.
__device__ __forceinline__ float tree_order(float vs) {
    return static_cast<float>(max(kTreeVexp, static_cast<int>(__float_as_uint(vs) >> 23 & 0xffu)) - 126);
}

// What a call makes of a request, in row tiles of ROWS and units of UNIT tokens.
struct TreeRequest {
    int n, first, len, units, tiles;   // drafted tokens, cached before them, positions in all, units and row tiles (0 without rows)
};
template <int ROWS, int UNIT>
__device__ __forceinline__ TreeRequest tree_request(const KvTreeParams& p, int r, int capacity) {
    TreeRequest q;
    q.n = p.rows.count(r), q.first = p.rows.first[r];
    const long long end = static_cast<long long>(q.first) + q.n;
    q.len = static_cast<int>(max(0ll, min(end, static_cast<long long>(capacity))));
    q.units = q.n > 0 ? (q.len - 1) / UNIT + 1 : 0;   // rows over nothing (-1 / UNIT is 0) still get their zeros; len + UNIT may not fit
    q.tiles = (q.n * p.G + ROWS - 1) / ROWS;
    return q;
}

// A run of the call's items (request, KV head, row tile, unit of tokens; in that order), tile by tile.
template <int ROWS, int UNIT>
struct TreeWalk {
    long long u0, u1, run, u, at;   // the run's items, items of a run, the current item, items before request r
    int r, capacity;
    TreeRequest q;
    int h, tile, b0, b1, begin;     // the current tile: KV head, row tile, units of it in this run, the request's first row
    // executed by whole warps
    __device__ __forceinline__ void start(const KvTreeParams& p, int me, int runs) {
        const int lane = threadIdx.x & 31, R = p.rows.R;
        capacity = p.pages.capacity();
        auto items = [&](int i) {
            if (i >= R) return 0ll;
            const TreeRequest t = tree_request<ROWS, UNIT>(p, i, capacity);
            return static_cast<long long>(t.tiles) * t.units * p.pages.H;
        };
        long long total = 0;
        for (int base = 0; base < R; base += 32) total += items(base + lane);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
        run = max(static_cast<long long>(kTreeMinRun), (total + runs - 1) / runs);
        u0 = min(total, me * run), u1 = min(total, u0 + run), u = u0;
        r = 0, at = 0, q = {};
        if (u0 >= u1) return;
        for (int base = 0;; base += 32) {
            const long long n = items(base + lane);
            long long scan = n;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const long long up = __shfl_up_sync(0xffffffffu, scan, o);
                if (lane >= o) scan += up;
            }
            const uint32_t hit = __ballot_sync(0xffffffffu, at + scan > u0);
            if (hit) {
                const int who = __ffs(hit) - 1;
                r = base + who;
                at += __shfl_sync(0xffffffffu, scan - n, who);
                break;
            }
            at += __shfl_sync(0xffffffffu, scan, 31);   // u0 < total: some request is hit before the requests end
        }
        q = tree_request<ROWS, UNIT>(p, r, capacity);
    }
    // The tile of item u; false at the run's end.
    __device__ __forceinline__ bool tile_here(const KvTreeParams& p) {
        if (u >= u1) return false;
        for (;;) {
            const long long n = static_cast<long long>(q.tiles) * q.units * p.pages.H;
            if (u - at < n) break;
            at += n;
            q = tree_request<ROWS, UNIT>(p, ++r, capacity);
        }
        const long long inner = u - at;
        const int tile_of = static_cast<int>(inner / q.units);
        b0 = static_cast<int>(inner - static_cast<long long>(tile_of) * q.units);
        b1 = static_cast<int>(min(static_cast<long long>(q.units), b0 + (u1 - u)));
        h = tile_of / q.tiles, tile = tile_of - h * q.tiles;
        begin = p.rows.begin(r);
        return true;
    }
    __device__ __forceinline__ void next() { u += b1 - b0; }
    __device__ __forceinline__ bool whole() const { return b0 == 0 && b1 == q.units; }
    // What the join needs of a tile that begins in this run and ends in a later one: request, head (and whether its first piece
    // is this run's second), row tile, pieces.
    __device__ __forceinline__ int4 unfinished(int me) const {
        return make_int4(r, h | (u != u0 ? 1 << 24 : 0), tile, static_cast<int>((u + q.units - 1) / run) - me + 1);
    }
};

template <bool BF16, int ROWS>
struct TreeShape {
    static constexpr bool kSplit = !BF16;                      // operands in two parts
    static constexpr int kParts = kSplit ? 2 : 1;
    static constexpr int kNT = ROWS / 8;                       // column tiles
    static constexpr int kWarps = kNT == 1 ? 16 : 12;          // one CTA per SM: 128 and 168 registers a thread
    static constexpr int kStages = kNT == 1 ? 2 : 3;
    static constexpr int kQuery = kNT * kParts * 4 * 512;      // query operands: tile, part, two k-steps, lane, their four registers
    static constexpr int kWarpBytes = kStages * kPgBlock + kQuery + ROWS * kParts * 16 + 64;   // ring, query, row facts, barriers
    static constexpr int kSmem = kWarps * kWarpBytes;
    static_assert(ROWS == 8 || (BF16 && ROWS == 16), "rows of a tile");
};

// Query rows of a tile -> fp16 B operands.  Dimensions 8c .. 8c + 7 of a row (c = 4 cq + i) are the pairs (0,4) (1,5)/16 of k-step
// 2i and (2,6) (3,7)/16 of k-step 2i + 1.  fact[part][row] = {-sum of the row's operands in three fp16 parts, factor from an
// accumulated product to a score}.
template <bool BF16, int ROWS>
__device__ __forceinline__ void tree_load_query(const KvTreeParams& p, int begin, int n, int h, int tile, uint8_t* operands, uint4* fact) {
    using S = TreeShape<BF16, ROWS>;
    const int lane = threadIdx.x & 31, l = lane & 7, sub = lane >> 3;
    const int valid = min(ROWS, n * p.G - tile * ROWS);
    // rows that do not exist keep what an earlier tile left, or the zeros of the start: they are columns of their own
#pragma unroll 1
    for (int base = 0; base < valid; base += 4) {
        const int row = base + sub, rho = tile * ROWS + row;
        float v[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] = 0.0f;
        if (row < valid) {
            const int i = rho / p.G, g = rho - i * p.G;
            kv_load16<BF16>(p.q, static_cast<size_t>((static_cast<long long>(begin) + i) * p.q_stride) + (h * p.G + g) * kKvD + 16 * l, v);
        }
        kv_rotate16(v, l, p.q_had, p.q_inv_sqrt);
        float top = 0.0f;
#pragma unroll
        for (int e = 0; e < 16; ++e) top = fmaxf(top, fabsf(v[e]));
#pragma unroll
        for (int o = 1; o < 8; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        // power of two that brings the largest value to 2^7 .. 2^8 (exponent field of the factor: 127 + 7 - (field - 127))
        const int field = max(16, min(254, static_cast<int>(__float_as_uint(top) >> 23)));
        const float up = __uint_as_float(static_cast<uint32_t>(min(254, 261 - field)) << 23);
        const float down = __uint_as_float(static_cast<uint32_t>(max(1, field - 7)) << 23);   // 1 / up
#pragma unroll
        for (int part = 0; part < S::kParts; ++part) {
            float sum = 0.0f;
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                uint32_t w[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float a = v[8 * c + e] * (part ? 1.0f : up), b = v[8 * c + e + 4] * (part ? 1.0f : up);
                    const float f = (e & 1) ? 0.0625f : 1.0f;
                    const __half2 hh = __floats2half2_rn(a * f, b * f);
                    const float2 back = __half22float2(hh);
                    const float ra = back.x * ((e & 1) ? 16.0f : 1.0f), rb = back.y * ((e & 1) ? 16.0f : 1.0f);
                    sum += ra + rb;
                    if (S::kSplit && part == 0) v[8 * c + e] = a - ra, v[8 * c + e + 4] = b - rb;   // the residual is the second part
                    w[e] = *reinterpret_cast<const uint32_t*>(&hh);
                }
                const int at = (((row >> 3) * S::kParts + part) * 4 + 2 * (l & 1) + c) * 512 + ((row & 7) * 4 + (l >> 1)) * 16;
                *reinterpret_cast<uint4*>(operands + at) = make_uint4(w[0], w[1], w[2], w[3]);
            }
#pragma unroll
            for (int o = 1; o < 8; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            if (l == 0) {
                const __half hi = __float2half_rn(-sum);
                const __half lo = __float2half_rn(-sum - __half2float(hi));
                const __half third = __float2half_rn((-sum - __half2float(hi)) - __half2float(lo));
                fact[part * ROWS + row] = make_uint4(static_cast<uint32_t>(__half_as_ushort(hi)) | static_cast<uint32_t>(__half_as_ushort(lo)) << 16,
                                                     __half_as_ushort(third), __float_as_uint(down * (S::kSplit ? 1.0f : 0x1p24f) * p.scale_log2), 0u);
            }
        }
    }
}

// The transpose of an 8 x 8 matrix of 16-bit values, two of them (neighbours in a row) per lane.
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

// Which tokens of block b a drafted token sees: bit k for position 32 b + k.
__device__ __forceinline__ uint32_t tree_seen(const KvTreeParams& p, int row, int i, int b, int first, int len) {
    const long long lo = static_cast<long long>(first) - static_cast<long long>(b) * kPgTokens;   // drafted token 0's bit in this block
    uint32_t seen = lo >= 32 ? 0xffffffffu : lo > 0 ? (1u << lo) - 1u : 0u;
    if (lo < 32) {
        if (p.mask) {
            const int32_t* m = p.mask + static_cast<size_t>(row) * p.mask_words;
            if (lo >= 0) {
                seen |= static_cast<uint32_t>(m[0]) << lo;
            } else {
                const long long j = -lo;
                const long long word = j >> 5;
                const int shift = static_cast<int>(j & 31);
                const uint32_t a = word < p.mask_words ? static_cast<uint32_t>(m[word]) : 0u;
                const uint32_t c = word + 1 < p.mask_words ? static_cast<uint32_t>(m[word + 1]) : 0u;
                seen |= __funnelshift_r(a, c, shift);
            }
        } else {
            const long long last = lo + i;   // bits lo .. lo + i
            const uint32_t upto = last >= 31 ? 0xffffffffu : last >= 0 ? (2u << last) - 1u : 0u;
            const uint32_t from = lo > 0 ? ~((1u << lo) - 1u) : 0xffffffffu;
            seen |= upto & from;
        }
    }
    const int left = len - b * kPgTokens;
    if (left < 32) seen &= left > 0 ? (1u << left) - 1u : 0u;
    return seen;
}

template <bool BF16, int ROWS>
__global__ void __launch_bounds__(32 * TreeShape<BF16, ROWS>::kWarps, 1)
kv4_tree_mma_kernel(const KvTreeParams p) {
    using S = TreeShape<BF16, ROWS>;
    constexpr int NT = S::kNT, ST = S::kStages;
    extern __shared__ __align__(128) uint8_t smem[];
    pdl_launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, cq = lane & 3;
    uint8_t* ring = smem + warp * S::kWarpBytes;
    uint8_t* operands = ring + ST * kPgBlock;
    uint4* fact = reinterpret_cast<uint4*>(operands + S::kQuery);
    uint64_t* bars = reinterpret_cast<uint64_t*>(fact + ROWS * S::kParts);
    if (lane < ST) mbar_init(&bars[lane], 1);
    mbar_fence_init();
    for (int i = lane; i < (S::kQuery + ROWS * S::kParts * 16) / 16; i += 32) reinterpret_cast<uint4*>(operands)[i] = make_uint4(0u, 0u, 0u, 0u);
    __syncwarp();
    pdl_wait();

    const int me = blockIdx.x * S::kWarps + warp;
    TreeWalk<ROWS, kPgTokens> walk;
    walk.start(p, me, gridDim.x * S::kWarps);
    int4 mine = make_int4(0, 0, 0, 0);   // the tile that begins here and ends later
    const int page_blocks = p.pages.page_tokens / kPgTokens;
    const uint32_t ring_at = smem_u32(ring), query = smem_u32(operands) + lane * 16;
    const uint32_t piece = static_cast<uint32_t>(cq * 8 + (g ^ (2 * cq))) * 16;
    uint32_t phases = 0;                 // parity of each stage's barrier
    bool failed = false;
    for (; !failed && walk.tile_here(p); walk.next()) {
        const TreeRequest q = walk.q;
        const int r = walk.r, h = walk.h, tile = walk.tile, b0 = walk.b0, b1 = walk.b1, begin = walk.begin;

        // ring: stage s holds block b0 + s, b0 + s + ST, ...; a block without a page is skipped (bit of `there` not set)
        const int32_t* table = p.pages.table + static_cast<size_t>(r) * p.pages.max_pages;
        int slot = b0 / page_blocks, in_page = b0 - slot * page_blocks, table_base = slot, next = b0;
        int pages32 = table_base + lane < p.pages.max_pages ? table[table_base + lane] : -1;
        uint32_t there = 0;
        const uint8_t* src = nullptr;    // next block's bytes
        auto page_of_slot = [&]() {
            const int page = __shfl_sync(0xffffffffu, pages32, slot - table_base);
            src = static_cast<unsigned>(page) < static_cast<unsigned>(p.pages.num_pages) && q.len > 0
                      ? p.pages.pool + ((static_cast<size_t>(page) * p.pages.H + h) * page_blocks + in_page) * kPgBlock : nullptr;
        };
        page_of_slot();
        auto issue = [&](int stage) {    // requests block `next` into a stage that nobody reads any more
            if (in_page == page_blocks) {
                in_page = 0, ++slot;
                if (slot - table_base == 32) {
                    table_base = slot;
                    pages32 = table_base + lane < p.pages.max_pages ? table[table_base + lane] : -1;
                }
                page_of_slot();
            }
            there &= ~(1u << stage);
            if (src) {
                if (lane == 0) {
                    mbar_expect_tx(&bars[stage], kPgBlock);
                    bulk_g2s(ring + stage * kPgBlock, src, kPgBlock, &bars[stage]);
                }
                there |= 1u << stage;
                src += kPgBlock;
            }
            ++next, ++in_page;
        };
        __syncwarp();
#pragma unroll
        for (int s = 0; s < ST; ++s)
            if (next < b1) issue(s);

        tree_load_query<BF16, ROWS>(p, begin, q.n, h, tile, operands, fact);
        __syncwarp();
        uint32_t qz[NT][S::kParts];      // B operands of the k-step of the zero-points: the sums of row g of a tile
        float factor[NT][2];             // of the lane's two rows of a tile, 2 cq and 2 cq + 1
        int token_of[NT][2];             // their drafted tokens; -1: none
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int part = 0; part < S::kParts; ++part) {
                const uint4 f = fact[part * ROWS + 8 * t + g];
                qz[t][part] = cq == 0 ? f.x : cq == 1 ? f.y : 0u;
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                factor[t][e] = __uint_as_float(fact[8 * t + 2 * cq + e].z);
                const int rho = tile * ROWS + 8 * t + 2 * cq + e;
                token_of[t][e] = rho < q.n * p.G ? rho / p.G : -1;
            }
        }

        float o[NT][8][4], z[NT][4], m_run[NT][2], l_run[NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int x = 0; x < 8; ++x)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[t][x][i] = 0.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i) z[t][i] = 0.0f;
#pragma unroll
            for (int e = 0; e < 2; ++e) m_run[t][e] = -INFINITY, l_run[t][e] = 0.0f;
        }
        const int plain_blocks = min(q.first, q.len) / kPgTokens;   // blocks that are context altogether

        int stage = 0;
        auto process = [&](int b, auto plain_tag) {
            constexpr bool kPlain = decltype(plain_tag)::value;
            const uint8_t* blk = ring + stage * kPgBlock;
            const uint32_t base = ring_at + stage * kPgBlock;
            // ---- scores: row tiles of 16 tokens (8n + g and 8(n + 1) + g), column tiles of eight query rows
            uint4 kw[4];
            uint32_t kz[4];
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                kw[n] = lds128(base + n * 512 + piece);
                kz[n] = blk[kPgKz + 8 * n + g] * 0x00010001u;
                if (S::kSplit) kz[n] = lessened(kz[n] | 0x64006400u, 0xe408e408u);   // - 1032
                kz[n] &= cq == 0 ? 0xffffffffu : cq == 1 ? 0x0000ffffu : 0u;
            }
            float sc[NT][2][4];
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int n = 0; n < 2; ++n) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) sc[t][n][i] = 0.0f;
#pragma unroll
                    for (int part = 0; part < S::kParts; ++part) mma_f16(sc[t][n], kz[2 * n], kz[2 * n + 1], 0u, 0u, qz[t][part], 0u);
                }
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                uint4 qb[NT][S::kParts];   // query operands come from shared memory every time: the registers go to the sums
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int part = 0; part < S::kParts; ++part) qb[t][part] = lds128(query + ((t * S::kParts + part) * 4 + c) * 512);
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    uint32_t r[2][4];      // the lane's word of two 8-token groups as four operand pairs each
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const uint4& x = kw[2 * n + i];
                        const uint32_t w = c == 0 ? x.x : c == 1 ? x.y : c == 2 ? x.z : x.w, y = w >> 8;
                        r[i][0] = w & 0x000f000fu, r[i][1] = w & 0x00f000f0u, r[i][2] = y & 0x000f000fu, r[i][3] = y & 0x00f000f0u;
                        if (S::kSplit) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) r[i][e] = lessened(r[i][e] | 0x64006400u, (e & 1) ? 0xe480e480u : 0xe408e408u);   // - 1152 : - 1032
                        }
                    }
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int part = 0; part < S::kParts; ++part) {
                            mma_f16(sc[t][n], r[0][0], r[1][0], r[0][1], r[1][1], qb[t][part].x, qb[t][part].y);
                            mma_f16(sc[t][n], r[0][2], r[1][2], r[0][3], r[1][3], qb[t][part].z, qb[t][part].w);
                        }
                }
            }
            float ks[4], vs[4];            // of the lane's tokens 8n + g
            uint32_t vz[4];
            uint4 vw[4];
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                ks[n] = *reinterpret_cast<const float*>(blk + kPgKs + (8 * n + g) * 4);
                // an infinite scale stands for a vector that is no number; the codes' product, 0, is exact without the 8 only
                if (S::kSplit) ks[n] = fmaf(ks[n], 0.0f, ks[n]);
                vs[n] = *reinterpret_cast<const float*>(blk + kPgVs + (8 * n + g) * 4);
                vz[n] = __byte_perm(*reinterpret_cast<const uint16_t*>(blk + kPgVz + 8 * n + 2 * cq), 0u, 0x4140u);
                if (S::kSplit) vz[n] = lessened(vz[n] | 0x64006400u, 0xe408e408u);   // - 1032
                vw[n] = lds128(base + kPgV + n * 512 + piece);
            }
            __syncwarp();                 // the stage has been read: its next block may come
            if (next < b1) issue(stage);

            // ---- which tokens are seen; slots that hold nothing may hold anything, NaN included
            uint32_t seen[NT][2];
            if (!kPlain) {
                const int left = q.len - b * kPgTokens;
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        seen[t][e] = token_of[t][e] >= 0 ? tree_seen(p, begin + token_of[t][e], token_of[t][e], b, q.first, q.len) >> g : 0u;
#pragma unroll
                for (int n = 0; n < 4; ++n)
                    if (8 * n + g >= left) vs[n] = 0.0f;
            }
            // ---- vectors of zeros: scale 1, whatever the others' are, and codes and zero-point 0 (in lane cq of token 8n + 2cq + h).  They
            // add nothing, so a scale of 0 does as well, which neither moves R nor leaves a rounding error of the codes less 8
            auto drop_zero_vectors = [&]() {
                if (!__any_sync(0xffffffffu, vs[0] == 1.0f || vs[1] == 1.0f || vs[2] == 1.0f || vs[3] == 1.0f)) return;
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                    uint32_t x = vz[n] ^ (S::kSplit ? 0xc800c800u : 0u);   // - 8
#pragma unroll
                    for (int w = 0; w < 4; ++w) x |= n == 0 ? vw[w].x : n == 1 ? vw[w].y : n == 2 ? vw[w].z : vw[w].w;
#pragma unroll
                    for (int i = 4; i < 32; i <<= 1) x |= __shfl_xor_sync(0xffffffffu, x, i);
                    x = __shfl_sync(0xffffffffu, x, g >> 1);
                    if (vs[n] == 1.0f && ((g & 1) ? x >> 16 : x & 0xffffu) == 0u) vs[n] = 0.0f;
                }
            };
            if (S::kSplit) drop_zero_vectors();
            // ---- scores, and whether one may exceed its row's reference point: by the lane's largest score and value scale, of whatever
            // tokens they are
            const float order = tree_order(fmaxf(fmaxf(vs[0], vs[1]), fmaxf(vs[2], vs[3])));
            bool raise = false;
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float top = -INFINITY;
#pragma unroll
                    for (int n = 0; n < 4; ++n) {
                        float& x = sc[t][n >> 1][2 * (n & 1) + e];
                        x *= ks[n];
                        if (!kPlain && !(seen[t][e] >> (8 * n) & 1)) x = -INFINITY;
                        top = fmaxf(top, x);
                    }
                    raise |= fmaf(top, factor[t][e], order) > m_run[t][e] + kTreeSlack;
                }
            if (__any_sync(0xffffffffu, raise)) {   // token by token
                if (!S::kSplit) drop_zero_vectors();
                float of[4];
#pragma unroll
                for (int n = 0; n < 4; ++n) of[n] = tree_order(vs[n]);
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float top = -INFINITY;
#pragma unroll
                        for (int n = 0; n < 4; ++n) top = fmaxf(top, fmaf(sc[t][n >> 1][2 * (n & 1) + e], factor[t][e], of[n]));
#pragma unroll
                        for (int x = 4; x < 32; x <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
                        const float to = fmaxf(ceilf(top), m_run[t][e]);
                        const float d = to > m_run[t][e] ? m_run[t][e] - to : 0.0f, corr = ex2(d);   // from -inf: 0
                        m_run[t][e] = to;
                        if (b != b0) {    // (nothing to scale before the first block)
                            l_run[t][e] = times_ex2(l_run[t][e], d);
                            z[t][e] *= corr;
#pragma unroll
                            for (int x = 0; x < 8; ++x) o[t][x][e] *= corr, o[t][x][2 + e] *= corr;
                        }
                    }
            }
            uint32_t wb[NT][S::kParts][4];   // weights as B operands: tokens of group n, columns = rows
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                float w[2][4];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float at = 8.0f - m_run[t][e];   // weights and their sum carry 2^8
#pragma unroll
                    for (int n = 0; n < 4; ++n) {
                        const bool on = kPlain || (seen[t][e] >> (8 * n) & 1);
                        const float pr = on ? ex2(fmaf(sc[t][n >> 1][2 * (n & 1) + e], factor[t][e], at)) : 0.0f;
                        l_run[t][e] += pr;
                        w[e][n] = on ? pr * vs[n] : 0.0f;
                    }
                }
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                    if constexpr (S::kSplit) {
                        uint32_t hi, lo;
                        split_half2(w[0][n], w[1][n], hi, lo);
                        wb[t][0][n] = transpose8(hi), wb[t][1][n] = transpose8(lo);
                    } else {
                        const __half2 hw = __floats2half2_rn(w[0][n], w[1][n]);
                        wb[t][0][n] = transpose8(*reinterpret_cast<const uint32_t*>(&hw));
                    }
                }
            }
            // ---- O += codes . w: row tile 2w + j of dimensions 32w + 4g + {j, j + 2}
            // The matrix instruction cuts its sums off instead of rounding them, always towards zero, which a long run of blocks
            // would add up (fp32, 3087 tokens a tile: 2.7e-6 of the output's norm): there each block's sum starts from zero and
            // joins the others by an fp32 addition.  To bf16's 2^-9 it is nothing.
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                float sum[4] = {};
#pragma unroll
                for (int part = S::kParts - 1; part >= 0; --part)
#pragma unroll
                    for (int k = 0; k < 2; ++k) mma_f16(S::kSplit ? sum : z[t], vz[2 * k], 0u, vz[2 * k + 1], 0u, wb[t][part][2 * k], wb[t][part][2 * k + 1]);
                if (S::kSplit) z[t][0] += sum[0], z[t][1] += sum[1];
            }
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const uint32_t x[4] = {vw[w].x, vw[w].y, vw[w].z, vw[w].w};
                float sum[2][4] = {};
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const uint32_t select = j ? 0x00f000f0u : 0x000f000fu;
                        uint32_t v[4] = {x[2 * k] & select, (x[2 * k] >> 8) & select, x[2 * k + 1] & select, (x[2 * k + 1] >> 8) & select};
                        if (S::kSplit) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) v[e] = lessened(v[e] | 0x64006400u, j ? 0xe480e480u : 0xe408e408u);   // - 1152 : - 1032
                        }
#pragma unroll
                        for (int t = 0; t < NT; ++t)
#pragma unroll
                            for (int part = S::kParts - 1; part >= 0; --part)
                                mma_f16(S::kSplit ? sum[j] : o[t][2 * w + j], v[0], v[1], v[2], v[3], wb[t][part][2 * k], wb[t][part][2 * k + 1]);
                    }
                if (S::kSplit)            // one column tile
#pragma unroll
                    for (int j = 0; j < 2; ++j)
#pragma unroll
                        for (int i = 0; i < 4; ++i) o[0][2 * w + j][i] += sum[j][i];
            }
        };
        for (int b = b0; b < b1; ++b, stage = stage + 1 == ST ? 0 : stage + 1) {
            if (!(there >> stage & 1)) {
                if (next < b1) issue(stage);
                continue;
            }
            if (!mbar_wait_near(&bars[stage], phases >> stage & 1, kTreeSite)) {
                failed = true;
                break;
            }
            phases ^= 1u << stage;
            if (b < plain_blocks) process(b, std::true_type{});
            else process(b, std::false_type{});
        }
        if (failed) break;

        // ---- the tile, or this warp's piece of it
        const bool whole = walk.whole();
        float* piece_at = p.partial + static_cast<size_t>(2 * me + (walk.u == walk.u0 ? 0 : 1)) * ROWS * kTreeRow;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float l = l_run[t][e];
#pragma unroll
                for (int x = 4; x < 32; x <<= 1) l += __shfl_xor_sync(0xffffffffu, l, x);
                if (token_of[t][e] < 0) continue;
                const int row = 8 * t + 2 * cq + e, hq = h * p.G + tile * ROWS + row - token_of[t][e] * p.G;
                const size_t out_at = (static_cast<size_t>(begin + token_of[t][e]) * p.Hq + hq) * kKvD;
                const float inv = whole ? (l == 0.0f ? 0.0f : 1.0f / l) : 1.0f;   // 0: nothing was seen
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    float y[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        y[j] = fmaf(o[t][2 * w + (j & 1)][(j & 2) + e], (j & 1) ? 0.0625f : 1.0f, -z[t][e]) * (S::kSplit ? 1.0f : 0x1p24f) * inv;
                    const int d = 32 * w + 4 * g;
                    if (!whole) {
                        *reinterpret_cast<float4*>(piece_at + row * kTreeRow + d) = make_float4(y[0], y[1], y[2], y[3]);
                    } else if constexpr (BF16) {
                        const __nv_bfloat162 u0 = __floats2bfloat162_rn(y[0], y[1]), u1 = __floats2bfloat162_rn(y[2], y[3]);
                        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.out) + out_at + d) =
                            make_uint2(*reinterpret_cast<const uint32_t*>(&u0), *reinterpret_cast<const uint32_t*>(&u1));
                    } else {
                        *reinterpret_cast<float4*>(static_cast<float*>(p.out) + out_at + d) = make_float4(y[0], y[1], y[2], y[3]);
                    }
                }
                if (!whole && g == 0) *reinterpret_cast<float2*>(piece_at + row * kTreeRow + kKvD) = make_float2(m_run[t][e], l);
            }
        if (b0 == 0 && !whole) mine = walk.unfinished(me);
    }
    if (failed) {   // copies in flight end (or are given up) before the shared memory does; whoever waits for this run's piece skips it
        mine = make_int4(0, 0, 0, 0);
        for (int s = 0; s < ST; ++s) mbar_wait(&bars[s], phases >> s & 1, kTreeSite, 1000000ull);
    }
    if (lane == 0) p.desc[me] = mine;
}

// Joins the pieces of the tile that begins in run blockIdx.x and ends in a later one.  The CTA's warps are shared out over the
// tile's rows; the warps of a row take its pieces in turn and meet in shared memory.
constexpr int kTreeJoinWarps = 8;
template <bool BF16, int ROWS>
__global__ void __launch_bounds__(32 * kTreeJoinWarps)
kv4_tree_join_kernel(const KvTreeParams p) {
    __shared__ float4 num[kTreeJoinWarps][32];
    __shared__ float2 ml[kTreeJoinWarps];
    pdl_launch_dependents();
    pdl_wait();
    const int4 d = p.desc[blockIdx.x];
    if (d.w == 0) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int r = d.x, h = d.y & 0xffffff, tile = d.z, pieces = d.w;
    const int begin = p.rows.begin(r), n = p.rows.count(r);
    const int row0 = 8 * blockIdx.y;     // rows of the tile for this CTA: eight
    const int valid = min(8, min(ROWS, n * p.G - tile * ROWS) - row0);
    if (valid <= 0) return;
    int share = kTreeJoinWarps;          // warps of a row: a power of two
    while (share > 1 && (kTreeJoinWarps / share < valid || share > pieces)) share >>= 1;
    const int rows_at_once = kTreeJoinWarps / share, sub = warp % share;
    const size_t step = static_cast<size_t>(2) * ROWS * kTreeRow;
    const float* first = p.partial + static_cast<size_t>(2 * blockIdx.x + (d.y >> 24)) * ROWS * kTreeRow;
    const float* rest = p.partial + static_cast<size_t>(blockIdx.x) * step;   // piece s > 0: rest + s * step
    for (int base = 0; base < valid; base += rows_at_once) {
        const int local = base + warp / share, row = row0 + local;
        float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        float m = -INFINITY, l = 0.0f;
        if (local < valid) {
            constexpr int kAhead = 4;
            for (int s0 = sub; s0 < pieces; s0 += share * kAhead) {
                float4 x[kAhead];
                float2 t[kAhead];
#pragma unroll
                for (int i = 0; i < kAhead; ++i) {
                    const int s = s0 + i * share;
                    const float* at = (s == 0 ? first : rest + s * step) + row * kTreeRow;
                    t[i] = make_float2(-INFINITY, 0.0f), x[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                    if (s < pieces) x[i] = *reinterpret_cast<const float4*>(at + 4 * lane), t[i] = *reinterpret_cast<const float2*>(at + kKvD);
                }
#pragma unroll
                for (int i = 0; i < kAhead; ++i) {
                    if (t[i].y == 0.0f) continue;   // saw nothing; scores that are no numbers leave a sum that is none, which stays
                    const float to = fmaxf(m, t[i].x), a = ex2(m - to), c = ex2(t[i].x - to);
                    acc.x = fmaf(acc.x, a, x[i].x * c), acc.y = fmaf(acc.y, a, x[i].y * c);
                    acc.z = fmaf(acc.z, a, x[i].z * c), acc.w = fmaf(acc.w, a, x[i].w * c);
                    l = times_ex2(l, m - to) + times_ex2(t[i].y, t[i].x - to), m = to;
                }
            }
        }
        if (share > 1) {
            __syncthreads();
            num[warp][lane] = acc;
            if (lane == 0) ml[warp] = make_float2(m, l);
            __syncthreads();
            if (sub == 0) {
                for (int s = 1; s < share; ++s) {
                    const float2 t = ml[warp + s];
                    if (t.y == 0.0f) continue;
                    const float4 x = num[warp + s][lane];
                    const float to = fmaxf(m, t.x), a = ex2(m - to), c = ex2(t.x - to);
                    acc.x = fmaf(acc.x, a, x.x * c), acc.y = fmaf(acc.y, a, x.y * c);
                    acc.z = fmaf(acc.z, a, x.z * c), acc.w = fmaf(acc.w, a, x.w * c);
                    l = times_ex2(l, m - to) + times_ex2(t.y, t.x - to), m = to;
                }
            }
        }
        if (local < valid && sub == 0) {
            const int rho = tile * ROWS + row, i = rho / p.G, hq = h * p.G + rho - i * p.G;
            const float inv = l == 0.0f ? 0.0f : 1.0f / l;
            const size_t at = (static_cast<size_t>(begin + i) * p.Hq + hq) * kKvD + 4 * lane;
            if constexpr (BF16) {
                const __nv_bfloat162 a = __floats2bfloat162_rn(acc.x * inv, acc.y * inv), c = __floats2bfloat162_rn(acc.z * inv, acc.w * inv);
                *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.out) + at) =
                    make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&c));
            } else {
                *reinterpret_cast<float4*>(static_cast<float*>(p.out) + at) = make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
            }
        }
    }
}

}  // namespace qift
