// Attention of drafted token trees with many rows per KV head (bf16 calls): the tcgen05 form of kv4_tree.cuh, on the same runs of
// items and the same pieces, joined by the same kernel.  An item is 128 tokens (four blocks) of one row tile.
//
//   S[128 rows][128 tokens] = Q (tensor memory) x K^T (shared memory),     O[128 rows][128 dims] += P (tensor memory) x V
// Rows are the lanes of tensor memory, so a thread has a row: maximum, sum and rescaling stay in it.
//   warps 0-7    softmax, two warps for 32 rows: scores of 64 of the item's tokens each, weights back as fp16.  The two agree on the
//                row's reference point through shared memory, once per item
//   warps 8-14   conversion, block by block in turn: codes less their zero-points become fp16 (exactly: (c - z) * 2^-24, odd
//                dimensions * 2^-20) in the 128-byte-swizzled tiles that the products read.  A warp fetches its own blocks two
//                ahead, 4416-byte bulk copies
//   warp 15      tensor memory and the two products: S of the next item is issued before O of this one, so the tensor cores
//                work while the softmax does
// What bounds it, per item of 128 tokens: the tensor cores (2 x 8 instructions of 64 cycles), the exponentials (128 rows x 128 at 16
// a cycle) and shared memory (64 KB of tiles written, 64 KB read) each take about 1024 cycles.
#pragma once

#include "kv4_tree.cuh"
#include "decode_tc.cuh"
#include "prefill.cuh"

namespace qift {

constexpr int kTtRows = 128;                 // rows of a tile
constexpr int kTtUnit = 128;                 // tokens of an item
constexpr int kTtConvert = 7;                // conversion warps
constexpr int kTtThreads = 32 * (8 + kTtConvert + 1);
constexpr int kTtRing = 2;                   // raw blocks of a conversion warp
constexpr int kTtScaleBytes = 2 * kTtUnit * 4 + 32;   // scales of keys and values; per block: largest value scale, whether it is there
constexpr int kTtStage = 4 * 16 * 256;       // query operands on their way to tensor memory: 16 rows of each lane quarter
constexpr int kTtSmem = 1024 + 4 * 32768 + kTtConvert * kTtRing * kPgBlock + 4 * kTtScaleBytes + kTtStage + 2 * 8 * 32 * 4 + 512;
constexpr uint32_t kTtS = 0, kTtO = 256, kTtP = 384, kTtQ = 448;   // tensor-memory columns: two S, O, P, Q

// As mbar_wait, polling without a time hint: these waits are short and mostly over when they begin.
__device__ __forceinline__ bool mbar_wait_near(uint64_t* bar, uint32_t parity, unsigned int site) {
    const uint32_t at = smem_u32(bar);
    uint64_t t0 = 0;
    for (uint32_t tries = 0;; ++tries) {
        uint32_t done;
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(done) : "r"(at), "r"(parity) : "memory");
        if (done) return true;
        if ((tries & 63) == 63) {
            const uint64_t t = global_timer_ns();
            if (t0 == 0) t0 = t;
            else if (t - t0 > kWaitLimitNs) break;
        }
    }
    report_timeout(site);
    return false;
}

// D[tmem] (+)= A[tmem] * B[smem descriptor], fp16 operands, fp32 sums
__device__ __forceinline__ void tc_mma_f16_ts(uint32_t tmem_d, uint32_t tmem_a, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(tmem_d),
        "r"(tmem_a), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void sts128(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
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
    constexpr uint32_t IDESC = (1u << 4) | ((128u / 8) << 17) | ((128u / 16) << 24);   // fp32 sums, fp16 operands, K-major, N = M = 128
    extern __shared__ __align__(128) uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    uint8_t* k_tiles = smem;                       // two, 32 KB each: two halves of 64 dimensions, 128 rows (tokens) of 128 bytes
    uint8_t* v_tiles = smem + 2 * 32768;           // two: two halves of 64 tokens, 128 rows (dimensions) of 128 bytes
    uint8_t* raw = smem + 4 * 32768;               // conversion warp, slot
    uint8_t* scales = raw + kTtConvert * kTtRing * kPgBlock;   // four items
    uint8_t* stage = scales + 4 * kTtScaleBytes;
    float* tops = reinterpret_cast<float*>(stage + kTtStage);   // [item parity][softmax warp][lane]
    uint64_t* bars = reinterpret_cast<uint64_t*>(tops + 2 * 8 * 32);
    uint64_t* raw_full = bars;                     // [kTtConvert * kTtRing]
    uint64_t* k_full = raw_full + kTtConvert * kTtRing;   // [2] conversion -> products
    uint64_t* k_free = k_full + 2;                 // [2] products -> conversion
    uint64_t* v_full = k_free + 2;
    uint64_t* v_free = v_full + 2;
    uint64_t* scale_full = v_free + 2;             // [4] conversion -> softmax
    uint64_t* s_full = scale_full + 4;             // [2] products -> softmax
    uint64_t* s_free = s_full + 2;                 // [2] softmax -> products
    uint64_t* p_full = s_free + 2;                 // softmax -> products
    uint64_t* o_done = p_full + 1;                 // products -> softmax
    uint64_t* q_full = o_done + 1;                 // softmax -> products
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(q_full + 1);
    static_assert((kTtConvert * kTtRing + 19) * 8 + 4 <= 512, "barriers");

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    pdl_launch_dependents();
    if (tid == 0) {
        for (int i = 0; i < kTtConvert * kTtRing; ++i) mbar_init(&raw_full[i], 1);
        for (int i = 0; i < 2; ++i) {
            mbar_init(&k_full[i], 4), mbar_init(&v_full[i], 4), mbar_init(&s_free[i], 8);
            mbar_init(&k_free[i], 1), mbar_init(&v_free[i], 1), mbar_init(&s_full[i], 1);
        }
        for (int i = 0; i < 4; ++i) mbar_init(&scale_full[i], 4);
        mbar_init(p_full, 8), mbar_init(o_done, 1), mbar_init(q_full, 8);
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

    // registers move to the softmax: 128 a thread at the launch, then 2 x 168 + 2 x 88 = 4 x 128 in the four warpgroups
    if (warp < 8) asm volatile("setmaxnreg.inc.sync.aligned.u32 168;");
    else asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    if (warp < 8) {
        // ------------------------------------------------------------------ softmax: a thread per row and half of the tokens
        const int quarter = warp & 3, half = warp >> 2;
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
            const int hq = have ? walk.h * p.G + walk.tile * kTtRows + row - token * p.G : 0;
            // ---- the query rows: rotated, scaled by a power of two each (largest value 2^7 .. 2^8), fp16, pairs (0,4) (1,5)/16 (2,6)
            // (3,7)/16 of every eight dimensions -- the order of the codes in a word of the cache.  Eight lanes make a row; sixteen
            // rows of the quarter at a time meet in shared memory and go to the lanes that own them, half of the columns per warp
            float factor = 0.0f;
            if (active) {
                uint8_t* here = stage + quarter * 16 * 256;
                const int l = lane & 7, sub = lane >> 3;
                uint32_t w[32];
#pragma unroll
                for (int i = 0; i < 32; ++i) w[i] = 0u;
#pragma unroll 1
                for (int round = 0; round < 2; ++round) {
#pragma unroll 1
                    for (int pass = 0; pass < 2; ++pass) {
                        const int row16 = 8 * half + 4 * pass + sub, at = quarter * 32 + 16 * round + row16;
                        float v[16];
#pragma unroll
                        for (int e = 0; e < 16; ++e) v[e] = 0.0f;
                        if (at < rows) {
                            const int rho = walk.tile * kTtRows + at, t = rho / p.G;
                            kv_load16<true>(p.q, static_cast<size_t>((static_cast<long long>(begin) + t) * p.q_stride) + (walk.h * p.G + rho - t * p.G) * kKvD + 16 * l, v);
                        }
                        kv_rotate16(v, l, p.q_had, p.q_inv_sqrt);
                        float top = 0.0f;
#pragma unroll
                        for (int e = 0; e < 16; ++e) top = fmaxf(top, fabsf(v[e]));
#pragma unroll
                        for (int o = 1; o < 8; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                        const int field = max(16, min(254, static_cast<int>(__float_as_uint(top) >> 23)));
                        const float up = __uint_as_float(static_cast<uint32_t>(min(254, 261 - field)) << 23);
                        if (l == 0) tops[(4 * round + quarter) * 32 + row16] = __uint_as_float(static_cast<uint32_t>(max(1, field - 7)) << 23) * 0x1p24f * p.scale_log2;
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            uint32_t x[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const float f = (e & 1) ? 0.0625f * up : up;
                                const __half2 hh = __floats2half2_rn(v[8 * c + e] * f, v[8 * c + e + 4] * f);
                                x[e] = *reinterpret_cast<const uint32_t*>(&hh);
                            }
                            *reinterpret_cast<uint4*>(here + row16 * 256 + (((2 * l + c) ^ row16) << 4)) = make_uint4(x[0], x[1], x[2], x[3]);
                        }
                    }
                    meet();
                    if ((lane >> 4) == round) {
                        factor = tops[(4 * round + quarter) * 32 + (lane & 15)];
#pragma unroll
                        for (int c = 0; c < 8; ++c) {
                            const uint4 x = *reinterpret_cast<const uint4*>(here + (lane & 15) * 256 + (((8 * half + c) ^ (lane & 15)) << 4));
                            w[4 * c] = x.x, w[4 * c + 1] = x.y, w[4 * c + 2] = x.z, w[4 * c + 3] = x.w;
                        }
                    }
                    meet();
                }
                tc_st32(lanes + kTtQ + 32 * half, w);
                tc_wait_st();
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(q_full);

            float m = -INFINITY;
            uint64_t l2 = 0;                                  // two sums of weights
            int vexp = kTreeVexp;
            for (int unit = walk.b0; unit < walk.b1; ++unit, ++n) {
                const bool fresh = unit == walk.b0;           // O holds nothing of this tile yet
                if (ok) ok = mbar_wait_near(&s_full[n & 1], (n >> 1) & 1, kTreeSite + 1) && mbar_wait_near(&scale_full[n & 3], (n >> 2) & 1, kTreeSite + 2);
                tc_fence_after();
                bool o_waited = n == 0;                       // O of the item before is done, and its P has been read
                auto wait_o = [&]() {
                    if (!o_waited && ok) ok = mbar_wait_near(o_done, (n - 1) & 1, kTreeSite + 3);
                    o_waited = true;
                    tc_fence_after();
                };
                if (active) {
                    const uint32_t sl = smem_u32(scales + (n & 3) * kTtScaleBytes);
                    const uint4 vtops = lds128(sl + 2 * kTtUnit * 4), info = lds128(sl + 2 * kTtUnit * 4 + 16);
                    const uint32_t vt = max(max(vtops.x, vtops.y), max(vtops.z, vtops.w));
                    const bool plain = (unit + 1) * kTtUnit <= min(q.first, q.len) && (info.x & info.y & info.z & info.w);
                    auto weigh = [&](auto plain_tag) {        // 64 tokens: scores -> weights
                        constexpr bool kPlain = decltype(plain_tag)::value;
                        uint32_t x[2][32];                    // scores, then weights, of tokens 32 i + 0 .. 31
                        tc_ld32(lanes + kTtS + (n & 1) * 128 + 64 * half, x[0]);
                        tc_ld32(lanes + kTtS + (n & 1) * 128 + 64 * half + 32, x[1]);
                        tc_wait_ld();
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&s_free[n & 1]);   // S may be written again
                        uint32_t seen[2];
                        if (!kPlain) {
                            const uint32_t i0 = half ? info.z : info.x, i1 = half ? info.w : info.y;
                            seen[0] = have && i0 ? tree_seen(p, begin + token, token, 4 * unit + 2 * half, q.first, q.len) : 0u;
                            seen[1] = have && i1 ? tree_seen(p, begin + token, token, 4 * unit + 2 * half + 1, q.first, q.len) : 0u;
                        }
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const uint4 k4 = lds128(sl + 256 * half + 16 * i);
                            uint32_t* y = &x[i >> 3][4 * (i & 7)];
                            mul2(y[0], y[1], k4.x, k4.y), mul2(y[2], y[3], k4.z, k4.w);
                        }
                        if (!kPlain) {
#pragma unroll
                            for (int i = 0; i < 64; ++i)
                                if (!(seen[i >> 5] >> (i & 31) & 1)) x[i >> 5][i & 31] = 0xff800000u;   // -inf
                        }
                        float best[4];
#pragma unroll
                        for (int c = 0; c < 4; ++c) best[c] = __uint_as_float(x[0][c]);
#pragma unroll
                        for (int i = 4; i < 64; i += 2)
                            best[(i >> 1) & 3] = fmaxf(best[(i >> 1) & 3], fmaxf(__uint_as_float(x[i >> 5][i & 31]), __uint_as_float(x[i >> 5][(i & 31) + 1])));
                        float top = fmaxf(fmaxf(best[0], best[1]), fmaxf(best[2], best[3])) * factor;
                        // the row's reference point, the same in both warps
                        float* told = tops + (n & 1) * 256;
                        told[warp * 32 + lane] = top;
                        meet();
                        top = fmaxf(top, told[(warp ^ 4) * 32 + lane]);
                        const bool vgrew = static_cast<int>(vt >> 23) > vexp;   // the same for all rows
                        if (vgrew || __any_sync(0xffffffffu, top > m + kTreeSlack)) {
                            const float to = top > m + kTreeSlack ? ceilf(top) : m;
                            float corr = to > m ? ex2(m - to) : 1.0f;
                            m = to;
                            if (vgrew) {
                                const int v = static_cast<int>(vt >> 23);
                                corr *= __uint_as_float(static_cast<uint32_t>(max(1, 127 + vexp - v)) << 23);
                                vexp = v;
                            }
                            l2 = both(0.0f) | __float_as_uint(sum2(l2) * corr);
                            if (!fresh) {
                                wait_o();
#pragma unroll 1
                                for (int c = 0; c < 4; ++c) {   // O times corr, row by row; half of the columns per warp
                                    uint32_t x[16];
                                    tc_ld16(lanes + kTtO + 64 * half + 16 * c, x);
                                    tc_wait_ld();
#pragma unroll
                                    for (int i = 0; i < 16; ++i) x[i] = __float_as_uint(__uint_as_float(x[i]) * corr);
                                    tc_st16(lanes + kTtO + 64 * half + 16 * c, x);
                                }
                                tc_wait_st();
                            }
                        }
                        const uint64_t f2 = both(factor);
                        const uint64_t r2 = both(static_cast<float>(134 - vexp) - m);   // weights and their sum carry 2^8 / 2^(vexp - 126)
                        uint64_t l3 = 0;
#pragma unroll
                        for (int b = 0; b < 2; ++b) {
                            uint32_t out[16];
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                const uint4 v4 = lds128(sl + kTtUnit * 4 + 256 * half + 128 * b + 16 * i);
#pragma unroll
                                for (int e = 0; e < 2; ++e) {
                                    const int j = 2 * i + e;   // tokens 2 j, 2 j + 1 of the 32
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
                            if (b == 0) wait_o();
                            tc_st16(lanes + kTtP + 32 * half + 16 * b, out);
                        }
                        add2(l2, static_cast<uint32_t>(l3), static_cast<uint32_t>(l3 >> 32));
                        tc_wait_st();
                    };
                    if (plain) weigh(std::true_type{});
                    else weigh(std::false_type{});
                } else {
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&s_free[n & 1]);
                    wait_o();
                }
                tc_fence_before();
                ok = __all_sync(0xffffffffu, ok);
                if (lane == 0) mbar_arrive(p_full);
            }
            // ---- the tile, or this run's piece of it: half of the columns per warp
            if (ok) ok = mbar_wait_near(o_done, (n - 1) & 1, kTreeSite + 3);
            ok = __all_sync(0xffffffffu, ok);
            tc_fence_after();
            if (active) {
                const bool whole = walk.whole();
                const float c1 = __uint_as_float(static_cast<uint32_t>(vexp) << 23);
                float l = (sum2(l2) * 0x1p-7f) * c1;
                float* told = tops + (n & 1) * 256;
                told[warp * 32 + lane] = l;
                meet();
                l += told[(warp ^ 4) * 32 + lane];
                const float inv = whole ? (l == 0.0f ? 0.0f : 1.0f / l) : 1.0f;
                float* piece = p.partial + (static_cast<size_t>(2 * blockIdx.x + (walk.u == walk.u0 ? 0 : 1)) * kTtRows + row) * kTreeRow;
                const size_t out_at = (static_cast<size_t>(begin + token) * p.Hq + hq) * kKvD;
#pragma unroll 1
                for (int part = 2 * half; part < 2 * half + 2; ++part) {
                    uint32_t a[32];
                    float y[32];
                    tc_ld32(lanes + kTtO + 32 * part, a);
                    tc_wait_ld();
#pragma unroll
                    for (int i = 0; i < 32; ++i)   // column 32 w + 8 j + g is dimension 32 w + 4 g + j; odd ones carry 16
                        y[4 * (i & 7) + (i >> 3)] = (__uint_as_float(a[i]) * (((i >> 3) & 1) ? 0x1p13f : 0x1p17f)) * c1 * inv;
                    if (!ok || !have) continue;
                    if (whole) {
                        uint4* dst = reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.out) + out_at + 32 * part);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            uint32_t bits[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const __nv_bfloat162 t = __floats2bfloat162_rn(y[8 * i + 2 * e], y[8 * i + 2 * e + 1]);
                                bits[e] = *reinterpret_cast<const uint32_t*>(&t);
                            }
                            dst[i] = make_uint4(bits[0], bits[1], bits[2], bits[3]);
                        }
                    } else {
                        float4* dst = reinterpret_cast<float4*>(piece + 32 * part);
#pragma unroll
                        for (int i = 0; i < 8; ++i) dst[i] = make_float4(y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]);
                    }
                }
                if (ok && have && half == 0 && !whole) *reinterpret_cast<float2*>(piece + kKvD) = make_float2(m, l);
                meet();              // the sums have been read before the next tile's factors come
            }
            tc_fence_before();       // O has been read: the next tile's products may write
            if (walk.b0 == 0 && !walk.whole()) mine = walk.unfinished(blockIdx.x);
        }
        if (tid == 0) p.desc[blockIdx.x] = ok ? mine : make_int4(0, 0, 0, 0);
    } else if (warp < 8 + kTtConvert) {
        // ------------------------------------------------------------------ conversion: every seventh block
        const int k = warp - 8;
        const int cq = lane >> 3, g = lane & 7;
        const int page_blocks = p.pages.page_tokens / kPgTokens;
        uint8_t* my_raw = raw + k * kTtRing * kPgBlock;
        TtItems ahead, now;
        now.start(p);
        ahead = now;
        uint32_t want = k, block = k;                         // numbers of the next block to ask for and to convert
        uint32_t there = 0;                                   // which ring slots got one
        int slot_in = 0, slot = 0, page = -1;
        auto look_up = [&]() {                                // the page of block `want`: used when it is asked for, later
            ahead.to(p, want >> 2);
            page = -1;
            if (!ahead.valid) return;
            const int b = 4 * ahead.unit + (want & 3);
            if (b * kPgTokens < ahead.w.q.len) page = p.pages.table[static_cast<size_t>(ahead.w.r) * p.pages.max_pages + b / page_blocks];
        };
        auto ask = [&]() {
            const int b = 4 * ahead.unit + (want & 3);
            const bool have = ahead.valid && static_cast<unsigned>(page) < static_cast<unsigned>(p.pages.num_pages);
            there = have ? there | (1u << slot_in) : there & ~(1u << slot_in);
            if (have && lane == 0) {
                uint64_t* bar = &raw_full[k * kTtRing + slot_in];
                mbar_expect_tx(bar, kPgBlock);
                bulk_g2s(my_raw + slot_in * kPgBlock, p.pages.pool + ((static_cast<size_t>(page) * p.pages.H + ahead.w.h) * page_blocks + b % page_blocks) * kPgBlock,
                         kPgBlock, bar);
            }
            slot_in ^= 1, want += kTtConvert;
            look_up();
        };
        static_assert(kTtRing == 2, "slots alternate");
        look_up();
        ask(), ask();
        uint32_t phases = 0;
        bool ok = true;
        for (now.to(p, block >> 2); now.valid; block += kTtConvert, now.to(p, block >> 2), slot ^= 1) {
            const int buf = now.n & 1, blk = block & 3;
            const uint32_t use = now.n >> 1;                  // how often this pair of tiles has been used before
            const bool have = there >> slot & 1;
            const uint8_t* src = my_raw + slot * kPgBlock;
            const uint32_t base = smem_u32(src);
            if (have) {
                if (!mbar_wait_near(&raw_full[k * kTtRing + slot], phases >> slot & 1, kTreeSite + 4)) {
                    ok = false;
                    break;
                }
                phases ^= 1u << slot;
                there &= ~(1u << slot);
            }
            if (use > 0 && !mbar_wait_near(&k_free[buf], (use - 1) & 1, kTreeSite + 5)) {
                ok = false;
                break;
            }
            // ---- keys: row = token, 16-byte chunk = eight dimensions
            const uint32_t ktile = smem_u32(k_tiles + buf * 32768) + (cq >> 1) * 16384 + blk * 4096 + g * 128;
            if (have) {
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                    const uint4 x4 = lds128(base + (n * 32 + cq * 8 + (g ^ (2 * cq))) * 16);
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
            {
                uint8_t* sl = scales + (now.n & 3) * kTtScaleBytes;
                const bool in = have && (4 * now.unit + blk) * kPgTokens + lane < now.w.q.len;
                const float ksc = in ? reinterpret_cast<const float*>(src + kPgKs)[lane] : 0.0f;
                const float vsc = in ? reinterpret_cast<const float*>(src + kPgVs)[lane] : 0.0f;
                reinterpret_cast<float*>(sl)[32 * blk + lane] = ksc;
                reinterpret_cast<float*>(sl + kTtUnit * 4)[32 * blk + lane] = vsc;
                const uint32_t bits = __float_as_uint(vsc);
                const uint32_t top = __reduce_max_sync(0xffffffffu, bits < 0x7f800000u ? bits : 0u);
                uint32_t* info = reinterpret_cast<uint32_t*>(sl + 2 * kTtUnit * 4);
                if (lane == 0) info[blk] = top, info[4 + blk] = have;
            }
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&k_full[buf]), mbar_arrive(&scale_full[now.n & 3]);
            // ---- values: row = dimension, 16-byte chunk = eight tokens
            if (use > 0 && !mbar_wait_near(&v_free[buf], (use - 1) & 1, kTreeSite + 6)) {
                ok = false;
                break;
            }
            const uint32_t vtile = smem_u32(v_tiles + buf * 32768) + (blk >> 1) * 16384 + g * 128 + ((((blk & 1) * 4 + cq) ^ g) << 4);
            if (have) {
                uint32_t z1[4], z16[4];
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                    const uint32_t z = __byte_perm(*reinterpret_cast<const uint16_t*>(src + kPgVz + 8 * n + 2 * cq), 0u, 0x4140u);
                    z1[n] = z ^ 0x80008000u, z16[n] = (z << 4) ^ 0x80008000u;
                }
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const uint4 x4 = lds128(base + kPgV + (w * 32 + cq * 8 + (g ^ (2 * cq))) * 16);
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
#pragma unroll
                for (int w = 0; w < 16; ++w) sts128(vtile + w * 1024, 0u, 0u, 0u, 0u);
            }
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&v_full[buf]);
            ask();
        }
        if (!ok)   // copies in flight end (or are given up) before the shared memory does
            for (int s = 0; s < kTtRing; ++s)
                if (there >> s & 1) mbar_wait(&raw_full[k * kTtRing + s], phases >> s & 1, kTreeSite + 4);
    } else {
        // ------------------------------------------------------------------ products
        TreeWalk<kTtRows, kTtUnit> walk;
        walk.start(p, blockIdx.x, gridDim.x);
        if (lane == 0) {
            const uint64_t kdesc = make_kmajor_sw128_desc(smem_u32(k_tiles)), vdesc = make_kmajor_sw128_desc(smem_u32(v_tiles));
            uint32_t n = 0, tiles = 0;
            bool ok = true;
            auto scores = [&](uint32_t i) {                   // S of item i
                const uint32_t buf = i & 1, use = i >> 1;
                if (!mbar_wait_near(&k_full[buf], use & 1, kTreeSite + 7)) return false;
                if (use > 0 && !mbar_wait_near(&s_free[buf], (use - 1) & 1, kTreeSite + 8)) return false;
                tc_fence_after();
#pragma unroll
                for (int ks = 0; ks < 8; ++ks)
                    tc_mma_f16_ts(tmem + kTtS + buf * 128, tmem + kTtQ + 8 * ks, kdesc + buf * (32768 >> 4) + (ks >> 2) * (16384 >> 4) + 2 * (ks & 3), IDESC, ks != 0);
                tc_commit(&k_free[buf]);
                tc_commit(&s_full[buf]);
                return true;
            };
            for (; ok && walk.tile_here(p); walk.next(), ++tiles) {
                if (!mbar_wait_near(q_full, tiles & 1, kTreeSite + 9)) break;
                tc_fence_after();
                if (!scores(n)) break;
                for (int unit = walk.b0; unit < walk.b1; ++unit, ++n) {
                    const uint32_t buf = n & 1, use = n >> 1;
                    if (unit + 1 < walk.b1 && !scores(n + 1)) {
                        ok = false;
                        break;
                    }
                    if (!mbar_wait_near(p_full, n & 1, kTreeSite + 10) || !mbar_wait_near(&v_full[buf], use & 1, kTreeSite + 11)) {
                        ok = false;
                        break;
                    }
                    tc_fence_after();
#pragma unroll
                    for (int ks = 0; ks < 8; ++ks)
                        tc_mma_f16_ts(tmem + kTtO, tmem + kTtP + 8 * ks, vdesc + buf * (32768 >> 4) + (ks >> 2) * (16384 >> 4) + 2 * (ks & 3), IDESC,
                                      (unit != walk.b0 || ks != 0) ? 1u : 0u);
                    tc_commit(&v_free[buf]);
                    tc_commit(o_done);
                }
            }
        }
        __syncwarp();
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 15) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    }
}

}  // namespace qift
