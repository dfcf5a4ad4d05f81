// Attention of drafted token trees with many rows per KV head (bf16 calls): the tcgen05 form of kv4_tree.cuh, on the same runs of
// items and the same pieces, joined by the same kernel.  An item is 64 tokens (two blocks) of one row tile.
//
//   S[128 rows][64 tokens] = Q (tensor memory) x K^T (shared memory),     O[128 rows][128 dims] += P (tensor memory) x V
// Rows are the lanes of tensor memory, so a thread has a row: maximum, sum and rescaling stay in it.
//   warps 0-7    softmax, two warps for 32 rows, which take the items in turn: while one is at the exponentials of its item (the
//                special-function pipe is the limit), the other scales the scores of the next and finds their maximum.  A row's
//                reference point goes from item to item through shared memory
//   warps 8-12   conversion: codes less their zero-points become fp16 (exactly: (c - z) * 2^-24, odd dimensions * 2^-20) in the
//                128-byte-swizzled tiles that the products read.  A task is the keys or the values of one block; they are dealt out
//                in the order in which the products need them (keys run three items ahead of values), so no task waits behind one
//                that is needed later
//   warp 13      fetches the blocks, one 4416-byte bulk copy each, up to twenty ahead (a lane looks up one block's page, 32 blocks at
//                a time)
//   warp 14      issues O as the weights and values of an item are there
//   warp 15      tensor memory; issues S.  Two warps issue because a wait, the instructions and their commits take one several
//                hundred cycles per item.  There are four S: a weight's way -- S, softmax, O -- takes about 2000 cycles, an item's
//                share of the tensor cores 512.  The weights take the place of their S
// What bounds it, per item: the tensor cores (8 instructions of 32 cycles, 4 of 64), the exponentials (128 rows x 64 at 16 a cycle) and
// shared memory (32 KB of tiles written, 32 KB read) each take about 512 cycles.
// Measured it is the hand-overs between the roles: about 1700 cycles an item, and 20000 a tile for its query, its results and the refill.
// 8 trees of 64 tokens over up to 32000, 32 query and 8 KV heads: 260 us (85 at the tensor cores' rate).  Value scales more than 2^12
// apart within 64 tokens take longer (2^-8 to 2^8 487 us), vectors of zeros too (a fifth of the tokens 359 us).
#pragma once

#include "kv4_tree.cuh"
#include "decode_tc.cuh"
#include "prefill.cuh"

namespace qift {

constexpr int kTtRows = 128;                 // rows of a tile
constexpr int kTtUnit = 64;                  // tokens of an item
constexpr int kTtDepth = 4;                  // S under way
constexpr int kTtTiles = 3;                  // tiles of keys, and of values
constexpr int kTtTile = 16384;               // bytes of a tile
constexpr int kTtConvert = 5;                // conversion warps
constexpr int kTtThreads = 32 * (8 + kTtConvert + 3);
constexpr int kTtRing = 20;                  // blocks on their way to the conversion; three items of them wait for their values to be due
constexpr int kTtScaleBytes = 2 * kTtUnit * 4 + 16;   // scales of keys and values; largest and smallest value scale of both blocks (0: no such block)
constexpr int kTtStage = 8 * 4096;           // 4 KB of a softmax warp: query operands on their way in, results on their way out
constexpr int kTtSmem = 1024 + 2 * kTtTiles * kTtTile + kTtRing * kPgBlock + 2 * kTtDepth * kTtScaleBytes + kTtStage + 2 * 128 * 4 + 768;
// Binary orders between the value scales of an item up to which the largest stands for all in the bound on a row's weights.  The
// largest weight is then 2^(6 - 12) at least, and fp16's smallest step, 2^-24, is still 2^-18 of it.
constexpr float kTtAlike = 12.0f;
constexpr uint32_t kTtS = 0, kTtO = 256, kTtQ = 384;   // tensor-memory columns: four S (the weights take the place of the first half), O, Q

// D[tmem] (+)= A[tmem] * B[smem descriptor], fp16 operands, fp32 sums
__device__ __forceinline__ void tc_mma_f16_ts(uint32_t tmem_d, uint32_t tmem_a, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(tmem_d),
        "r"(tmem_a), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
}
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void sts128(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ void tc_ld4(uint32_t taddr, uint32_t (&v)[4]) {   // and waits for it
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0,%1,%2,%3}, [%4];\n\ttcgen05.wait::ld.sync.aligned;"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tc_st16(uint32_t taddr, const uint32_t (&v)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
        "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]),
        "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
        : "memory");
}
// Pairs of fp32 values (bit patterns, neighbouring registers) in one instruction, in place: x = x * y, x = x * y + z.
__device__ __forceinline__ void mul2(uint32_t& x0, uint32_t& x1, uint32_t y0, uint32_t y1) {
    asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%0, %1};\n\tmov.b64 y, {%2, %3};\n\tmul.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "+r"(x0), "+r"(x1) : "r"(y0), "r"(y1));
}
__device__ __forceinline__ void fma2(uint32_t& x0, uint32_t& x1, uint64_t y, uint64_t z) {
    asm("{\n\t.reg .b64 x;\n\tmov.b64 x, {%0, %1};\n\tfma.rn.f32x2 x, x, %2, %3;\n\tmov.b64 {%0, %1}, x;\n\t}" : "+r"(x0), "+r"(x1) : "l"(y), "l"(z));
}
__device__ __forceinline__ void add2(uint64_t& sum, uint32_t x0, uint32_t x1) {
    asm("{\n\t.reg .b64 x;\n\tmov.b64 x, {%1, %2};\n\tadd.rn.f32x2 %0, %0, x;\n\t}" : "+l"(sum) : "r"(x0), "r"(x1));
}
__device__ __forceinline__ uint64_t both(float x) { return static_cast<uint64_t>(__float_as_uint(x)) << 32 | __float_as_uint(x); }
__device__ __forceinline__ float sum2(uint64_t x) { return __uint_as_float(static_cast<uint32_t>(x)) + __uint_as_float(static_cast<uint32_t>(x >> 32)); }

// Items of a run one by one: a tile's units are consecutive.
struct TtItems {
    TreeWalk<kTtRows, kTtUnit> w;
    int unit;          // the item's unit within its tile
    uint32_t n;        // items of this run before it
    bool valid;
    __device__ __forceinline__ void start(const KvTreeParams& p) {
        w.start(p, blockIdx.x, gridDim.x);
        n = 0, valid = w.tile_here(p), unit = valid ? w.b0 : 0;
    }
    __device__ __forceinline__ void to(const KvTreeParams& p, uint32_t item) {
        while (valid && n < item) {
            ++n;
            if (++unit == w.b1) {
                w.next();
                valid = w.tile_here(p);
                if (valid) unit = w.b0;
            }
        }
    }
};

__global__ void __launch_bounds__(kTtThreads, 1)
kv4_tree_tc_kernel(const KvTreeParams p) {
    // fp32 sums, fp16 operands, K-major, M = 128; N = 64 tokens or 128 dimensions
    constexpr uint32_t S_IDESC = (1u << 4) | ((64u / 8) << 17) | ((128u / 16) << 24), O_IDESC = (1u << 4) | ((128u / 8) << 17) | ((128u / 16) << 24);
    extern __shared__ __align__(128) uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    uint8_t* k_tiles = smem;                       // [kTtTiles] two halves of 64 dimensions, 64 rows (tokens) of 128 bytes
    uint8_t* v_tiles = smem + kTtTiles * kTtTile;  // [kTtTiles] 128 rows (dimensions) of 128 bytes, 64 tokens
    uint8_t* raw = smem + 2 * kTtTiles * kTtTile;  // ring of blocks
    uint8_t* scales = raw + kTtRing * kPgBlock;    // [2 * kTtDepth] items
    uint8_t* stage = scales + 2 * kTtDepth * kTtScaleBytes;
    float* marks = reinterpret_cast<float*>(stage + kTtStage);     // [item parity][row] reference points
    uint64_t* bars = reinterpret_cast<uint64_t*>(marks + 2 * 128);
    uint64_t* raw_full = bars;                     // [kTtRing] fetch -> conversion
    uint64_t* raw_free = raw_full + kTtRing;       // [kTtRing] conversion -> fetch
    uint64_t* k_full = raw_free + kTtRing;         // [kTtTiles] conversion -> products
    uint64_t* k_free = k_full + kTtTiles;          // [2 * kTtTiles] products -> conversion, by item
    uint64_t* v_free = k_free + 2 * kTtTiles;      // [2 * kTtTiles]
    uint64_t* scale_full = v_free + 2 * kTtTiles;      // [2 * kTtDepth] conversion -> softmax
    uint64_t* s_full = scale_full + 2 * kTtDepth;  // [kTtDepth] products -> softmax
    uint64_t* p_full = s_full + kTtDepth;          // [kTtDepth] softmax (weights) and conversion (values) -> products
    uint64_t* o_done = p_full + kTtDepth;          // [kTtDepth] products -> softmax
    uint64_t* q_full = o_done + kTtDepth;          // softmax -> products
    uint64_t* mark_full = q_full + 1;              // [2][4] reference points of an item, by lane quarter
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(mark_full + 8);
    int* raw_tokens = reinterpret_cast<int*>(tmem_slot + 1);   // [kTtRing] tokens of a block that hold something; 0: no such block
    static_assert((2 * kTtRing + 5 * kTtTiles + 5 * kTtDepth + 9) * 8 + 4 + 4 * kTtRing <= 768, "barriers");

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    pdl_launch_dependents();
    if (tid == 0) {
        for (int i = 0; i < kTtRing; ++i) mbar_init(&raw_full[i], 1), mbar_init(&raw_free[i], 2);
        for (int i = 0; i < kTtDepth; ++i) {
            mbar_init(&p_full[i], 4 + 2), mbar_init(&s_full[i], 1), mbar_init(&o_done[i], 1);
        }
        for (int i = 0; i < kTtTiles; ++i) mbar_init(&k_full[i], 2);
        for (int i = 0; i < 2 * kTtTiles; ++i) mbar_init(&k_free[i], 1), mbar_init(&v_free[i], 1);
        for (int i = 0; i < 2 * kTtDepth; ++i) mbar_init(&scale_full[i], 2);
        mbar_init(q_full, 8);
        for (int i = 0; i < 8; ++i) mbar_init(&mark_full[i], 1);
        mbar_fence_init();
    }
    if (warp == 15) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    pdl_wait();

    // registers move to the softmax: 128 a thread at the launch, then 2 x 184 + 2 x 72 = 4 x 128 in the four warpgroups
    if (warp < 8) asm volatile("setmaxnreg.inc.sync.aligned.u32 184;");
    else asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    if (warp < 8) {
        // ------------------------------------------------------------------ softmax: a thread per row, items in turn
        const int quarter = warp & 3, turn = warp >> 2;       // items n with (n & 1) == turn; half of the columns of Q and O
        const uint32_t lanes = tmem + (static_cast<uint32_t>(quarter * 32) << 16);
        const int row = quarter * 32 + lane;                  // row of the tile
        // the two warps of a lane quarter meet here; a warp that has given up waiting still comes
        auto meet = [&]() { asm volatile("bar.sync %0, 64;" ::"r"(1 + quarter) : "memory"); };
        TreeWalk<kTtRows, kTtUnit> walk;
        walk.start(p, blockIdx.x, gridDim.x);
        int4 mine = make_int4(0, 0, 0, 0);
        uint32_t n = 0;                                       // items done
        bool ok = true;
        for (; walk.tile_here(p); walk.next()) {
            const TreeRequest q = walk.q;
            const int begin = walk.begin, rows = q.n * p.G - walk.tile * kTtRows;   // rows from this tile on
            const bool have = row < rows;                     // this row exists
            const bool active = quarter * 32 < rows;          // some row of the warp does
            const int token = have ? (walk.tile * kTtRows + row) / p.G : -1;
            // ---- the query rows: rotated, scaled by a power of two each (largest value 2^7 .. 2^8), fp16, pairs (0,4) (1,5)/16 (2,6)
            // (3,7)/16 of every eight dimensions -- the order of the codes in a word of the cache.  Eight lanes make a row; the rows
            // of the quarter, sixteen per warp, meet in shared memory and go to the lanes that own them, half of the columns per warp
            float factor = 0.0f;
            if (active) {
                uint8_t* here = stage + quarter * 8192;
                const int l = lane & 7, sub = lane >> 3;
                uint4 in[2];                                  // the next four rows are on their way while these are rotated
                auto fetch = [&](int pass) {
                    in[0] = in[1] = make_uint4(0u, 0u, 0u, 0u);
                    const int at = quarter * 32 + 16 * turn + 4 * pass + sub;
                    if (pass < 4 && at < rows) {
                        const int rho = walk.tile * kTtRows + at, t = rho / p.G;
                        const uint4* src = reinterpret_cast<const uint4*>(
                            static_cast<const uint16_t*>(p.q) + static_cast<size_t>((static_cast<long long>(begin) + t) * p.q_stride) + (walk.h * p.G + rho - t * p.G) * kKvD + 16 * l);
                        in[0] = src[0], in[1] = src[1];
                    }
                };
                fetch(0);
#pragma unroll 1
                for (int pass = 0; pass < 4; ++pass) {
                    const int row32 = 16 * turn + 4 * pass + sub;
                    float v[16];
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const uint32_t w[4] = {in[c].x, in[c].y, in[c].z, in[c].w};
#pragma unroll
                        for (int e = 0; e < 4; ++e) v[8 * c + 2 * e] = __uint_as_float(w[e] << 16), v[8 * c + 2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
                    }
                    fetch(pass + 1);
                    kv_rotate16(v, l, p.q_had, p.q_inv_sqrt);
                    float top = 0.0f;
#pragma unroll
                    for (int e = 0; e < 16; ++e) top = fmaxf(top, fabsf(v[e]));
#pragma unroll
                    for (int o = 1; o < 8; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                    const int field = max(16, min(254, static_cast<int>(__float_as_uint(top) >> 23)));
                    const float up = __uint_as_float(static_cast<uint32_t>(min(254, 261 - field)) << 23);
                    if (l == 0) marks[quarter * 32 + row32] = __uint_as_float(static_cast<uint32_t>(max(1, field - 7)) << 23) * 0x1p24f * p.scale_log2;
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        uint32_t x[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float f = (e & 1) ? 0.0625f * up : up;
                            const __half2 hh = __floats2half2_rn(v[8 * c + e] * f, v[8 * c + e + 4] * f);
                            x[e] = *reinterpret_cast<const uint32_t*>(&hh);
                        }
                        *reinterpret_cast<uint4*>(here + row32 * 256 + (((2 * l + c) ^ (row32 & 15)) << 4)) = make_uint4(x[0], x[1], x[2], x[3]);
                    }
                }
                meet();
                factor = marks[row];
                uint32_t w[32];
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    const uint4 x = *reinterpret_cast<const uint4*>(here + lane * 256 + (((8 * turn + c) ^ (lane & 15)) << 4));
                    w[4 * c] = x.x, w[4 * c + 1] = x.y, w[4 * c + 2] = x.z, w[4 * c + 3] = x.w;
                }
                meet();
                tc_st32(lanes + kTtQ + 32 * turn, w);
                tc_wait_st();
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(q_full);

            float m = -INFINITY;                              // reference point as of an item
            float l_m = -INFINITY;                            // the one that this warp's sum of weights goes by
            uint64_t l2 = 0;                                  // two sums of weights
            const uint32_t n0 = n;
            n += walk.b1 - walk.b0;
            for (uint32_t i = n0 + ((n0 ^ turn) & 1); i < n; i += 2) {
                const int unit = walk.b0 + static_cast<int>(i - n0);
                const uint32_t buf = i % kTtDepth, s_at = lanes + kTtS + buf * kTtUnit;
                if (ok) ok = mbar_wait_near(&s_full[buf], (i / kTtDepth) & 1, kTreeSite + 1) &&
                             mbar_wait_near(&scale_full[i % (2 * kTtDepth)], (i / (2 * kTtDepth)) & 1, kTreeSite + 2);
                tc_fence_after();
                if (active) {
                    const uint32_t sl = smem_u32(scales + (i % (2 * kTtDepth)) * kTtScaleBytes);
                    const uint4 info = lds128(sl + 2 * kTtUnit * 4);   // largest and smallest value scale of the two blocks (0: not there)
                    const float order = tree_order(__uint_as_float(max(info.x, info.y)));
                    const bool alike = order - tree_order(__uint_as_float(min(info.z - 1, info.w - 1))) <= kTtAlike;   // (a block that is not there: 0 - 1)
                    const bool plain = unit < min(q.first, q.len) / kTtUnit && info.z && info.w && alike;
                    auto weigh = [&](auto plain_tag) {        // scores -> weights
                        constexpr bool kPlain = decltype(plain_tag)::value;
                        uint32_t x[2][32], seen[2];           // of tokens 32 b + 0 .. 31
                        tc_ld32(s_at, x[0]);
                        tc_ld32(s_at + 32, x[1]);
                        if (!kPlain) {
                            const bool context = unit < min(q.first, q.len) / kTtUnit;
                            seen[0] = !have || !info.z ? 0u : context ? 0xffffffffu : tree_seen(p, begin + token, token, 2 * unit, q.first, q.len);
                            seen[1] = !have || !info.w ? 0u : context ? 0xffffffffu : tree_seen(p, begin + token, token, 2 * unit + 1, q.first, q.len);
                        }
                        tc_wait_ld();
                        // ---- the largest score
                        float best[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                        for (int b = 0; b < 2; ++b) {
#pragma unroll
                            for (int c = 0; c < 8; ++c) {
                                const uint4 k4 = lds128(sl + 128 * b + 16 * c);
                                mul2(x[b][4 * c], x[b][4 * c + 1], k4.x, k4.y), mul2(x[b][4 * c + 2], x[b][4 * c + 3], k4.z, k4.w);
                            }
                            if (!kPlain) {
#pragma unroll
                                for (int c = 0; c < 32; ++c)
                                    if (!(seen[b] >> c & 1)) x[b][c] = 0xff800000u;   // -inf
                            }
#pragma unroll
                            for (int c = 0; c < 32; c += 2)
                                best[(c >> 1) & 3] = fmaxf(best[(c >> 1) & 3], fmaxf(__uint_as_float(x[b][c]), __uint_as_float(x[b][c + 1])));
                        }
                        const float top = fmaxf(fmaxf(best[0], best[1]), fmaxf(best[2], best[3]));
                        // ---- the row's reference point: the one of the item before, raised if need be
                        float m_old = -INFINITY;
                        if (i != n0) {
                            if (ok) ok = mbar_wait_near(&mark_full[((i - 1) & 1) * 4 + quarter], ((i - 1) >> 1) & 1, kTreeSite + 12);
                            m_old = marks[((i - 1) & 1) * 128 + row];
                        }
                        m = m_old;
                        const float bound = fmaf(top, factor, order);   // by the largest value scale of any token
                        if (__any_sync(0xffffffffu, bound > m_old + kTreeSlack)) {
                            float highest = bound;
                            if (!kPlain && !alike) {          // token by token, of those that are seen
                                highest = -INFINITY;
#pragma unroll 1
                                for (int c = 0; c < kTtUnit; c += 4) {   // (short code: 64 tokens at once slow the whole kernel, 258 -> 280 us)
                                    uint32_t y[4];
                                    tc_ld4(s_at + c, y);
                                    const uint32_t on = (c < 32 ? seen[0] : seen[1]) >> (c & 31);
                                    const uint4 k4 = lds128(sl + 4 * c), v4 = lds128(sl + 4 * (kTtUnit + c));
                                    const uint32_t k[4] = {k4.x, k4.y, k4.z, k4.w}, v[4] = {v4.x, v4.y, v4.z, v4.w};
#pragma unroll
                                    for (int e = 0; e < 4; ++e)
                                        if (on >> e & 1)
                                            highest = fmaxf(highest, fmaf(__uint_as_float(y[e]) * __uint_as_float(k[e]), factor, tree_order(__uint_as_float(v[e]))));
                                }
                            }
                            if (highest > m_old + kTreeSlack) m = ceilf(highest);   // whole binary orders
                        }
                        marks[(i & 1) * 128 + row] = m;
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&mark_full[(i & 1) * 4 + quarter]);
                        if (i != n0 && __any_sync(0xffffffffu, m != m_old)) {
                            // O of the item before times what the references differ by, row by row
                            const float corr = m != m_old ? ex2(m_old - m) : 1.0f;
                            if (ok) ok = mbar_wait_near(&o_done[(i - 1) % kTtDepth], ((i - 1) / kTtDepth) & 1, kTreeSite + 3);
                            tc_fence_after();
#pragma unroll 1
                            for (int c = 0; c < 8; ++c) {
                                uint32_t y[16];
                                tc_ld16(lanes + kTtO + 16 * c, y);
                                tc_wait_ld();
#pragma unroll
                                for (int e = 0; e < 16; ++e) y[e] = __float_as_uint(__uint_as_float(y[e]) * corr);
                                tc_st16(lanes + kTtO + 16 * c, y);
                            }
                            tc_wait_st();
                        }
                        if (__any_sync(0xffffffffu, m != l_m)) {
                            l2 = __float_as_uint(times_ex2(sum2(l2), m != l_m ? l_m - m : 0.0f));
                            l_m = m;
                        }
                        // ---- weights
                        const uint64_t f2 = both(factor);
                        const uint64_t r2 = both(8.0f - m);   // weights and their sum carry 2^8
                        uint64_t l3 = 0;
#pragma unroll
                        for (int b = 0; b < 2; ++b) {
                            uint32_t out[16];
#pragma unroll
                            for (int c = 0; c < 8; ++c) {
                                const uint4 v4 = lds128(sl + kTtUnit * 4 + 128 * b + 16 * c);
#pragma unroll
                                for (int e = 0; e < 2; ++e) {
                                    const int j = 2 * c + e;   // tokens 2 j, 2 j + 1 of the 32
                                    uint32_t &y0 = x[b][2 * j], &y1 = x[b][2 * j + 1];
                                    fma2(y0, y1, f2, r2);
                                    y0 = __float_as_uint(ex2(__uint_as_float(y0))), y1 = __float_as_uint(ex2(__uint_as_float(y1)));
                                    if (!kPlain) {
                                        if (!(seen[b] >> (2 * j) & 1)) y0 = 0u;
                                        if (!(seen[b] >> (2 * j + 1) & 1)) y1 = 0u;
                                    }
                                    add2(e ? l3 : l2, y0, y1);
                                    mul2(y0, y1, e ? v4.z : v4.x, e ? v4.w : v4.y);
                                    if (!kPlain) {             // a slot that is not seen may hold anything
                                        if (!(seen[b] >> (2 * j) & 1)) y0 = 0u;
                                        if (!(seen[b] >> (2 * j + 1) & 1)) y1 = 0u;
                                    }
                                    const __half2 hw = __floats2half2_rn(__uint_as_float(y0), __uint_as_float(y1));
                                    // token 32 b + 8 n + 2 cq + h stands at position 32 b + 8 cq + 2 n + h of the second product
                                    out[(j & 3) * 4 + (j >> 2)] = *reinterpret_cast<const uint32_t*>(&hw);
                                }
                            }
                            // the weights take the place of scores that have been read
                            tc_st16(s_at + 16 * b, out);
                        }
                        add2(l2, static_cast<uint32_t>(l3), static_cast<uint32_t>(l3 >> 32));
                        tc_wait_st();
                    };
                    if (plain) weigh(std::true_type{});
                    else weigh(std::false_type{});
                } else if (lane == 0) {
                    mbar_arrive(&mark_full[(i & 1) * 4 + quarter]);   // keeps the barrier in step with the items
                }
                tc_fence_before();
                ok = __all_sync(0xffffffffu, ok);
                if (lane == 0) mbar_arrive(&p_full[buf]);
            }
            // ---- the tile, or this run's piece of it: half of the columns per warp
            if (ok) ok = mbar_wait_near(&o_done[(n - 1) % kTtDepth], ((n - 1) / kTtDepth) & 1, kTreeSite + 3);
            ok = __all_sync(0xffffffffu, ok);
            tc_fence_after();
            if (active) {
                const bool whole = walk.whole();
                // the last item's reference point, and this warp's sum brought to it
                if (ok) ok = mbar_wait_near(&mark_full[((n - 1) & 1) * 4 + quarter], ((n - 1) >> 1) & 1, kTreeSite + 12);
                m = marks[((n - 1) & 1) * 128 + row];
                float l = sum2(l2);  // without a reference point: 0, or no number when no score was one
                if (l_m > -INFINITY) l = times_ex2(l, l_m - m);
                meet();              // the reference points have been read by both
                marks[turn * 128 + row] = l;
                meet();
                l += marks[(turn ^ 1) * 128 + row];
                const float inv = whole ? (l == 0.0f ? 0.0f : 1.0f / l) : 1.0f;
                float* piece = p.partial + (static_cast<size_t>(2 * blockIdx.x + (walk.u == walk.u0 ? 0 : 1)) * kTtRows + quarter * 32) * kTreeRow;
                float4* own = reinterpret_cast<float4*>(stage + quarter * 8192 + turn * 4096);   // the quarter's own, as for the query
#pragma unroll 1
                for (int part = 2 * turn; part < 2 * turn + 2; ++part) {
                    uint32_t a[32];
                    tc_ld32(lanes + kTtO + 32 * part, a);
                    tc_wait_ld();
                    // column 32 w + 8 j + g is dimension 32 w + 4 g + j; odd ones carry 16.  32 rows of 32 dimensions go through shared
                    // memory, so that eight lanes write 128 bytes of a row together
                    __syncwarp();
#pragma unroll
                    for (int g = 0; g < 8; ++g) {
                        float y[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) y[j] = __uint_as_float(a[8 * j + g]) * ((j & 1) ? 0x1p20f : 0x1p24f) * inv;
                        own[lane * 8 + (g ^ (lane & 7))] = make_float4(y[0], y[1], y[2], y[3]);
                    }
                    __syncwarp();
#pragma unroll 1
                    for (int i = 0; i < 8; ++i) {
                        const int r32 = 4 * i + (lane >> 3), c = lane & 7, at = quarter * 32 + r32;
                        const float4 y = own[r32 * 8 + (c ^ (r32 & 7))];
                        if (!ok || at >= rows) continue;
                        if (whole) {
                            const int rho = walk.tile * kTtRows + at, t = rho / p.G;
                            const __nv_bfloat162 u0 = __floats2bfloat162_rn(y.x, y.y), u1 = __floats2bfloat162_rn(y.z, y.w);
                            *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.out) + (static_cast<size_t>(begin + t) * p.Hq + walk.h * p.G + rho - t * p.G) * kKvD + 32 * part + 4 * c) =
                                make_uint2(*reinterpret_cast<const uint32_t*>(&u0), *reinterpret_cast<const uint32_t*>(&u1));
                        } else {
                            *reinterpret_cast<float4*>(piece + r32 * kTreeRow + 32 * part + 4 * c) = y;
                        }
                    }
                }
                if (ok && have && turn == 0 && !whole) *reinterpret_cast<float2*>(piece + lane * kTreeRow + kKvD) = make_float2(m, l);
                meet();              // the sums have been read before the next tile's factors come
            }
            tc_fence_before();       // O has been read: the next tile's products may write
            if (walk.b0 == 0 && !walk.whole()) mine = walk.unfinished(blockIdx.x);
        }
        if (tid == 0) p.desc[blockIdx.x] = ok ? mine : make_int4(0, 0, 0, 0);
    } else if (warp < 8 + kTtConvert) {
        // ------------------------------------------------------------------ conversion: every fifth task
        const int cq = lane >> 3, g = lane & 7;
        const uint32_t piece = static_cast<uint32_t>(cq * 8 + (g ^ (2 * cq))) * 16;
        const uint32_t raw_at = smem_u32(raw), k_at = smem_u32(k_tiles) + (cq >> 1) * 8192 + g * 128, v_at = smem_u32(v_tiles) + g * 128;
        TreeWalk<kTtRows, kTtUnit> walk;
        walk.start(p, blockIdx.x, gridDim.x);
        const uint32_t items = static_cast<uint32_t>(walk.u1 - walk.u0);   // (an item's number fits: 2^32 of them take days)
        // pairs of tasks: keys of items 0 .. 2, then values of item i and keys of item i + 3 in turn
        for (uint32_t task = warp - 8; task < 2 * (2 * items + kTtTiles - 1); task += kTtConvert) {
            const uint32_t pair = task >> 1, blk = task & 1;
            const bool values = pair >= kTtTiles && !((pair - kTtTiles) & 1);
            const uint32_t item = pair < kTtTiles ? pair : values ? (pair - kTtTiles) >> 1 : ((pair - kTtTiles) >> 1) + kTtTiles;
            if (item >= items) continue;
            const uint32_t buf = item % kTtTiles;
            const uint32_t block = 2 * item + blk, slot = block % kTtRing;
            const uint8_t* src = raw + slot * kPgBlock;
            const uint32_t base = raw_at + slot * kPgBlock + piece;
            if (!mbar_wait_near(&raw_full[slot], (block / kTtRing) & 1, kTreeSite + 4)) break;
            // The item that had the tile before is done with it.  Tasks are waited for out of step -- this warp may come here while the
            // products of earlier items are under way -- and a parity cannot tell a phase from the second next: with two barriers
            // per tile, the phase before is the one of item - 9, over when this warp's last task began
            if (item >= kTtTiles) {
                const uint32_t before = item - kTtTiles;
                uint64_t* bar = (values ? v_free : k_free) + before % (2 * kTtTiles);
                if (!mbar_wait_near(bar, before / (2 * kTtTiles) & 1, kTreeSite + 5)) break;
            }
            const int tokens = raw_tokens[slot];
            const bool have = tokens > 0;
            if (!values) {
                // ---- row = token, 16-byte chunk = eight dimensions
                const uint32_t ktile = k_at + buf * kTtTile + blk * 4096;
                if (have) {
#pragma unroll
                    for (int n = 0; n < 4; ++n) {
                        const uint4 x4 = lds128(base + n * 512);
                        const uint32_t x[4] = {x4.x, x4.y, x4.z, x4.w};
                        const uint32_t z = src[kPgKz + 8 * n + g] * 0x00010001u;
                        const uint32_t z1 = z ^ 0x80008000u, z16 = (z << 4) ^ 0x80008000u;   // minus the zero-point, and 16 times it
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint32_t y = x[i] >> 8;
                            sts128(ktile + n * 1024 + ((((cq & 1) * 4 + i) ^ g) << 4), lessened(x[i] & 0x000f000fu, z1), lessened(x[i] & 0x00f000f0u, z16),
                                   lessened(y & 0x000f000fu, z1), lessened(y & 0x00f000f0u, z16));
                        }
                    }
                }
                uint8_t* sl = scales + (item % (2 * kTtDepth)) * kTtScaleBytes;
                const bool in = lane < tokens;
                const float ksc = in ? reinterpret_cast<const float*>(src + kPgKs)[lane] : 0.0f;
                float vsc = in ? reinterpret_cast<const float*>(src + kPgVs)[lane] : 0.0f;
                const bool suspect = vsc == 1.0f && src[kPgVz + lane] == 0;   // a vector of zeros?  It adds nothing, and its scale says nothing
                if (__any_sync(0xffffffffu, suspect)) {
                    uint32_t codes = 0;      // of this lane's token: 16 bits (lane & 1) of word lane / 8 of all pieces with cq = lane / 2 % 4
#pragma unroll 1
                    for (int n = 0; n < 4; ++n) {
                        uint32_t x = 0;
#pragma unroll
                        for (int w = 0; w < 4; ++w) x |= *reinterpret_cast<const uint32_t*>(src + kPgV + w * 512 + piece + 4 * n);
#pragma unroll
                        for (int o = 1; o < 8; o <<= 1) x |= __shfl_xor_sync(0xffffffffu, x, o);
                        x = __shfl_sync(0xffffffffu, x, (lane >> 1 & 3) * 8);
                        if (lane >> 3 == n) codes = x >> (16 * (lane & 1)) & 0xffffu;
                    }
                    if (suspect && codes == 0) vsc = 0.0f;
                }
                reinterpret_cast<float*>(sl)[32 * blk + lane] = ksc;
                reinterpret_cast<float*>(sl + kTtUnit * 4)[32 * blk + lane] = vsc;
                const uint32_t bits = __float_as_uint(vsc);
                const bool counts = bits - 1u < 0x7f7fffffu;   // finite, not 0
                const uint32_t top = __reduce_max_sync(0xffffffffu, counts ? bits : 0u), least = __reduce_min_sync(0xffffffffu, counts ? bits : in ? 1u : 0x7f7fffffu);   // (nothing: unlike any)
                uint32_t* info = reinterpret_cast<uint32_t*>(sl + 2 * kTtUnit * 4);
                if (lane == 0) info[blk] = top, info[2 + blk] = have ? least : 0u;
                fence_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(&k_full[buf]), mbar_arrive(&scale_full[item % (2 * kTtDepth)]), mbar_arrive(&raw_free[slot]);
            } else {
                // ---- row = dimension, 16-byte chunk = eight tokens
                const uint32_t vtile = v_at + buf * kTtTile + (((blk * 4 + cq) ^ g) << 4);
                if (have) {
                    uint32_t z1[4], z16[4];
#pragma unroll
                    for (int n = 0; n < 4; ++n) {
                        const uint32_t z = __byte_perm(*reinterpret_cast<const uint16_t*>(src + kPgVz + 8 * n + 2 * cq), 0u, 0x4140u);
                        z1[n] = z ^ 0x80008000u, z16[n] = (z << 4) ^ 0x80008000u;
                    }
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const uint4 x4 = lds128(base + kPgV + w * 512);
                        const uint32_t x[4] = {x4.x, x4.y, x4.z, x4.w};
                        const uint32_t y[4] = {x4.x >> 8, x4.y >> 8, x4.z >> 8, x4.w >> 8};
                        sts128(vtile + (w * 4) * 1024, lessened(x[0] & 0x000f000fu, z1[0]), lessened(x[1] & 0x000f000fu, z1[1]),
                               lessened(x[2] & 0x000f000fu, z1[2]), lessened(x[3] & 0x000f000fu, z1[3]));
                        sts128(vtile + (w * 4 + 1) * 1024, lessened(x[0] & 0x00f000f0u, z16[0]), lessened(x[1] & 0x00f000f0u, z16[1]),
                               lessened(x[2] & 0x00f000f0u, z16[2]), lessened(x[3] & 0x00f000f0u, z16[3]));
                        sts128(vtile + (w * 4 + 2) * 1024, lessened(y[0] & 0x000f000fu, z1[0]), lessened(y[1] & 0x000f000fu, z1[1]),
                               lessened(y[2] & 0x000f000fu, z1[2]), lessened(y[3] & 0x000f000fu, z1[3]));
                        sts128(vtile + (w * 4 + 3) * 1024, lessened(y[0] & 0x00f000f0u, z16[0]), lessened(y[1] & 0x00f000f0u, z16[1]),
                               lessened(y[2] & 0x00f000f0u, z16[2]), lessened(y[3] & 0x00f000f0u, z16[3]));
                    }
                } else {   // no such block: its weights are zero, and zero times what was left there must be zero
#pragma unroll 1
                    for (int w = 0; w < 16; ++w) sts128(vtile + w * 1024, 0u, 0u, 0u, 0u);
                }
                fence_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(&p_full[item % kTtDepth]), mbar_arrive(&raw_free[slot]);
            }
        }
    } else if (warp == 13) {
        // ------------------------------------------------------------------ fetch: lane i looks up block 32 j + i
        TtItems items;
        items.start(p);
        const int page_blocks = p.pages.page_tokens / kPgTokens;
        const uint32_t blocks = 2 * static_cast<uint32_t>(items.w.u1 - items.w.u0);
        uint32_t slot = 0, round = 0;
        bool ok = true;
        for (uint32_t base = 0; base < blocks && ok; base += 32) {
            const uint8_t* src = nullptr;
            int tokens = 0;
            items.to(p, (base + lane) >> 1);
            if (items.valid) {
                const int b = 2 * items.unit + (lane & 1);
                tokens = items.w.q.len - b * kPgTokens;
                if (tokens > 0) {
                    const int at = b / page_blocks;
                    const int page = p.pages.table[static_cast<size_t>(items.w.r) * p.pages.max_pages + at];
                    if (static_cast<unsigned>(page) < static_cast<unsigned>(p.pages.num_pages))
                        src = p.pages.pool + ((static_cast<size_t>(page) * p.pages.H + items.w.h) * page_blocks + (b - at * page_blocks)) * kPgBlock;
                }
            }
            for (uint32_t i = 0; i < 32 && base + i < blocks; ++i) {
                if (round > 0) ok = __all_sync(0xffffffffu, mbar_wait_near(&raw_free[slot], (round - 1) & 1, kTreeSite + 8));
                if (!ok) break;
                if (lane == static_cast<int>(i)) {
                    raw_tokens[slot] = src ? tokens : 0;
                    if (src) {
                        mbar_expect_tx(&raw_full[slot], kPgBlock);
                        bulk_g2s(raw + slot * kPgBlock, src, kPgBlock, &raw_full[slot]);
                    } else {
                        mbar_arrive(&raw_full[slot]);
                    }
                }
                __syncwarp();
                if (++slot == kTtRing) slot = 0, ++round;
            }
        }
        if (!ok)   // copies in flight end (or are given up) before the shared memory does
            for (uint32_t i = 0; i < kTtRing; ++i)
                if (i < slot || round > 0) mbar_wait(&raw_full[i], (i < slot ? round : round - 1) & 1, kTreeSite + 4, 1000000ull);
    } else if (warp == 14) {
        // ------------------------------------------------------------------ O
        // the whole warp follows the loop, so that descriptors stay in uniform registers; one elected lane issues
        TreeWalk<kTtRows, kTtUnit> walk;
        walk.start(p, blockIdx.x, gridDim.x);
        const uint64_t vdesc = make_kmajor_sw128_desc(smem_u32(v_tiles));
        uint32_t n = 0;
        bool ok = true;
        for (; ok && walk.tile_here(p); walk.next()) {
            const uint32_t n0 = n;
            for (const uint32_t end = n + (walk.b1 - walk.b0); n < end; ++n) {
                const uint32_t buf = n % kTtDepth, tile = n % kTtTiles;
                ok = __all_sync(0xffffffffu, mbar_wait_near(&p_full[buf], (n / kTtDepth) & 1, kTreeSite + 11));
                if (!ok) break;
                tc_fence_after();
                const uint32_t a = tmem + kTtS + buf * kTtUnit, more = n != n0;
                const uint64_t b = vdesc + tile * (kTtTile >> 4);
                if (elect_one()) {
#pragma unroll
                    for (int ks = 0; ks < 4; ++ks) tc_mma_f16_ts(tmem + kTtO, a + 8 * ks, b + 2 * ks, O_IDESC, ks != 0 ? 1u : more);
                    tc_commit(&v_free[n % (2 * kTtTiles)]);
                    tc_commit(&o_done[buf]);
                }
                __syncwarp();
            }
        }
    } else {
        // ------------------------------------------------------------------ S
        TreeWalk<kTtRows, kTtUnit> walk;
        walk.start(p, blockIdx.x, gridDim.x);
        const uint64_t kdesc = make_kmajor_sw128_desc(smem_u32(k_tiles));
        uint32_t n = 0, tiles = 0;
        bool ok = true;
        for (; ok && walk.tile_here(p); walk.next(), ++tiles) {
            ok = __all_sync(0xffffffffu, mbar_wait_near(q_full, tiles & 1, kTreeSite + 9));
            for (const uint32_t end = n + (walk.b1 - walk.b0); n < end && ok; ++n) {
                const uint32_t buf = n % kTtDepth, use = n / kTtDepth, tile = n % kTtTiles;
                // the place is free when the weights of item n - 4 have been used
                ok = mbar_wait_near(&k_full[tile], (n / kTtTiles) & 1, kTreeSite + 7) && (use == 0 || mbar_wait_near(&o_done[buf], (use - 1) & 1, kTreeSite + 10));
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                tc_fence_after();
                const uint32_t d = tmem + kTtS + buf * kTtUnit;
                const uint64_t b = kdesc + tile * (kTtTile >> 4);
                if (elect_one()) {
#pragma unroll
                    for (int ks = 0; ks < 8; ++ks) tc_mma_f16_ts(d, tmem + kTtQ + 8 * ks, b + (ks >> 2) * (8192 >> 4) + 2 * (ks & 3), S_IDESC, ks != 0);
                    tc_commit(&k_free[n % (2 * kTtTiles)]);
                    tc_commit(&s_full[buf]);
                }
                __syncwarp();
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 15) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    }
}

}  // namespace qift
