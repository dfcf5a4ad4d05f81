// Attention of drafted token trees with many rows per KV head (bf16 calls): the tcgen05 form of kv4_tree.cuh, on the same runs of
// items and the same pieces, joined by the same kernel.  An item is 128 tokens (four blocks) of one row tile.
//
//   S[128 rows][128 tokens] = Q (tensor memory) x K^T (shared memory),     O[128 rows][128 dims] += P (tensor memory) x V
// Rows are the lanes of tensor memory, so a thread owns a row: maximum, sum and rescaling stay in it.
//   warps 0-3    softmax, one thread per lane: scores from tensor memory in two halves of 64 tokens, weights back as fp16
//   warps 4-11   conversion: every warp has one of the four blocks of every other item; codes less their zero-points become fp16
//                (exactly: (c - z) * 2^-24, odd dimensions * 2^-20) in the 128-byte-swizzled tiles that the products read.  A warp
//                fetches its own blocks two items ahead, 4416-byte bulk copies
//   warp 12      tensor memory and the two products: S of the next item is issued before O of this one, so the tensor cores
//                work while the softmax does
// REP = 2 serves tiles of up to 64 rows: lanes 64 .. 127 hold the same rows as 0 .. 63 and take the second 64 tokens of an item (the
// other half of their P stays zero), which halves the softmax per warp; the two halves of O meet in shared memory at the end.
// What bounds it, per item of 128 tokens: the tensor cores (2 x 8 instructions of 64 cycles), the exponentials (128 rows x 128 at 16
// a cycle) and shared memory (64 KB of tiles written, 64 KB read) each take about 1024 cycles.
#pragma once

#include "kv4_tree.cuh"
#include "decode_tc.cuh"
#include "prefill.cuh"

namespace qift {

constexpr int kTtUnit = 128;                 // tokens of an item
constexpr int kTtThreads = 32 * 13;
constexpr int kTtRing = 2;                   // raw blocks of a conversion warp
constexpr int kTtScaleBytes = 2 * kTtUnit * 4 + 32;   // scales of keys and values; per block: largest value scale, whether it is there
constexpr int kTtMeet = 68;                  // floats of a row where the halves meet (64 of a numerator, reference point, sum)
constexpr uint32_t kTtS = 0, kTtO = 256, kTtP = 384, kTtQ = 448;   // tensor-memory columns: two S, O, P, Q

template <int REP>
struct TtShape {
    static constexpr int kRows = 128 / REP;
    static constexpr int kSmem = 1024 + 4 * 32768 + 8 * kTtRing * kPgBlock + 4 * kTtScaleBytes + (REP == 2 ? 64 * kTtMeet * 4 : 0) + 512;
};

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
// Pairs of fp32 values in one instruction.
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    float2 d;
    asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmul.rn.f32x2 z, x, y;\n\tmov.b64 {%0, %1}, z;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 d;
    asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tadd.rn.f32x2 z, x, y;\n\tmov.b64 {%0, %1}, z;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 d;
    asm("{\n\t.reg .b64 x, y, z, w;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmov.b64 z, {%6, %7};\n\tfma.rn.f32x2 w, x, y, z;\n\tmov.b64 {%0, %1}, w;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}

// Items of a run one by one: a tile's units are consecutive.
template <int ROWS>
struct TtItems {
    TreeWalk<ROWS, kTtUnit> w;
    int unit;          // the item's unit within its tile
    uint32_t n;        // items of this run before it
    bool valid;
    __device__ __forceinline__ void start(const KvTreeParams& p) {
        w.start(p, blockIdx.x, gridDim.x);
        n = 0, valid = w.tile_here(p), unit = valid ? w.b0 : 0;
    }
    __device__ __forceinline__ void next(const KvTreeParams& p) {
        ++n;
        if (++unit == w.b1) {
            w.next();
            valid = w.tile_here(p);
            if (valid) unit = w.b0;
        }
    }
};

template <int REP>
__global__ void __launch_bounds__(kTtThreads, 1)
kv4_tree_tc_kernel(const KvTreeParams p) {
    using S = TtShape<REP>;
    constexpr int ROWS = S::kRows;
    constexpr uint32_t IDESC = (1u << 4) | ((128u / 8) << 17) | ((128u / 16) << 24);   // fp32 sums, fp16 operands, K-major, N = M = 128
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    uint8_t* k_tiles = smem;                       // two, 32 KB each: two halves of 64 dimensions, 128 rows (tokens) of 128 bytes
    uint8_t* v_tiles = smem + 2 * 32768;           // two: two halves of 64 tokens, 128 rows (dimensions) of 128 bytes
    uint8_t* raw = smem + 4 * 32768;               // conversion warp, slot
    uint8_t* scales = raw + 8 * kTtRing * kPgBlock;   // four items
    float* meet = reinterpret_cast<float*>(scales + 4 * kTtScaleBytes);
    uint64_t* bars = reinterpret_cast<uint64_t*>(reinterpret_cast<uint8_t*>(meet) + (REP == 2 ? 64 * kTtMeet * 4 : 0));
    uint64_t* raw_full = bars;                     // [8 * kTtRing]
    uint64_t* k_full = raw_full + 8 * kTtRing;     // [2] conversion -> products
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

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    pdl_launch_dependents();
    if (tid == 0) {
        for (int i = 0; i < 8 * kTtRing; ++i) mbar_init(&raw_full[i], 1);
        for (int i = 0; i < 2; ++i) {
            mbar_init(&k_full[i], 4), mbar_init(&v_full[i], 4), mbar_init(&s_free[i], 4);
            mbar_init(&k_free[i], 1), mbar_init(&v_free[i], 1), mbar_init(&s_full[i], 1);
        }
        for (int i = 0; i < 4; ++i) mbar_init(&scale_full[i], 4);
        mbar_init(p_full, 4), mbar_init(o_done, 1), mbar_init(q_full, 4);
        mbar_fence_init();
    }
    if (warp == 12) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    pdl_wait();

    if (warp < 4) {
        // ------------------------------------------------------------------ softmax: a thread per lane
        const uint32_t lanes = tmem + (static_cast<uint32_t>(warp * 32) << 16);
        const int row = (warp * 32 + lane) & (ROWS - 1);      // row of the tile
        const int half = REP == 2 ? warp >> 1 : 0;            // REP = 2: the 64 tokens of an item that these lanes take
        if (REP == 2) {                                       // the others' weights stay zero
            tc_zero16(lanes + kTtP + 32 * (1 - half)), tc_zero16(lanes + kTtP + 32 * (1 - half) + 16);
            tc_wait_st();
        }
        TreeWalk<ROWS, kTtUnit> walk;
        walk.start(p, blockIdx.x, gridDim.x);
        int4 mine = make_int4(0, 0, 0, 0);
        uint32_t n = 0;                                       // items done
        bool ok = true;   // once false the warp only keeps the barriers that the four share
        for (; walk.tile_here(p); walk.next()) {
            const TreeRequest q = walk.q;
            const int begin = walk.begin, rho = walk.tile * ROWS + row;
            const bool have = rho < q.n * p.G;                // this row exists
            const bool active = walk.tile * ROWS + (warp * 32 & (ROWS - 1)) < q.n * p.G;   // some row of the warp does
            const int token = have ? rho / p.G : -1, hq = have ? walk.h * p.G + rho - token * p.G : 0;
            float factor = 0.0f;
            if (ok) {   // the query row: rotated, scaled by a power of two (largest value 2^7 .. 2^8), fp16, pairs (0,4) (1,5)/16 (2,6) (3,7)/16
                // of every eight dimensions -- the order of the codes in a word of the cache
                float v[128];
#pragma unroll
                for (int i = 0; i < 128; ++i) v[i] = 0.0f;
                if (have) {
                    const uint4* src = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p.q) +
                                                                      static_cast<size_t>((static_cast<long long>(begin) + token) * p.q_stride) + hq * kKvD);
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const uint4 x = src[i];
                        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            v[8 * i + 2 * k] = __uint_as_float(w[k] << 16), v[8 * i + 2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
                    }
                }
#pragma unroll
                for (int h = 1; h < kKvD; h <<= 1) {
                    if (h < p.q_had) {
#pragma unroll
                        for (int i = 0; i < 128; ++i)
                            if (!(i & h)) {
                                const float a = v[i], b = v[i + h];
                                v[i] = a + b, v[i + h] = a - b;
                            }
                    }
                }
                float top = 0.0f;
#pragma unroll
                for (int i = 0; i < 128; ++i) v[i] *= p.q_inv_sqrt, top = fmaxf(top, fabsf(v[i]));
                const int field = max(16, min(254, static_cast<int>(__float_as_uint(top) >> 23)));
                const float up = __uint_as_float(static_cast<uint32_t>(min(254, 261 - field)) << 23);
                factor = __uint_as_float(static_cast<uint32_t>(max(1, field - 7)) << 23) * 0x1p24f * p.scale_log2;
#pragma unroll
                for (int part = 0; part < 2; ++part) {
                    uint32_t w[32];
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        const int d = 64 * part + 8 * (i >> 2) + (i & 3);
                        const float f = (i & 1) ? 0.0625f * up : up;
                        const __half2 hh = __floats2half2_rn(v[d] * f, v[d + 4] * f);
                        w[i] = *reinterpret_cast<const uint32_t*>(&hh);
                    }
                    tc_st32(lanes + kTtQ + 32 * part, w);
                }
                tc_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(q_full);
            }
            float m = -INFINITY, vexp_f = 0.0f;
            float2 l2 = make_float2(0.0f, 0.0f);
            int vexp = kTreeVexp;
            for (int unit = walk.b0; unit < walk.b1 && ok; ++unit, ++n) {
                const bool fresh = unit == walk.b0;           // O holds nothing of this tile yet
                if (!mbar_wait(&s_full[n & 1], (n >> 1) & 1, kTreeSite + 1) || !mbar_wait(&scale_full[n & 3], (n >> 2) & 1, kTreeSite + 2)) {
                    ok = false;
                    break;
                }
                tc_fence_after();
                bool o_waited = n == 0;                       // O of the item before is done
                const uint8_t* sl = scales + (n & 3) * kTtScaleBytes;
                const uint32_t* info = reinterpret_cast<const uint32_t*>(sl + 2 * kTtUnit * 4);
                const uint32_t s_at = lanes + kTtS + (n & 1) * 128;
                auto rescale = [&](float corr, int p_done) {  // O (and the weights of this item already given) times corr, row by row
                    if (!fresh) {
                        if (!o_waited) {
                            if (!mbar_wait(o_done, (n - 1) & 1, kTreeSite + 3)) ok = false;
                            o_waited = true;
                            tc_fence_after();
                        }
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            uint32_t x[32];
                            tc_ld32(lanes + kTtO + 32 * c, x);
                            tc_wait_ld();
#pragma unroll
                            for (int i = 0; i < 32; ++i) x[i] = __float_as_uint(__uint_as_float(x[i]) * corr);
                            tc_st32(lanes + kTtO + 32 * c, x);
                        }
                    }
                    if (p_done) {
                        uint32_t x[32];
                        tc_ld32(lanes + kTtP, x);
                        tc_wait_ld();
                        const __half2 c2 = __float2half2_rn(corr);
#pragma unroll
                        for (int i = 0; i < 32; ++i) {
                            const __half2 y = __hmul2(*reinterpret_cast<const __half2*>(&x[i]), c2);
                            x[i] = *reinterpret_cast<const uint32_t*>(&y);
                        }
                        tc_st32(lanes + kTtP, x);
                    }
                    tc_wait_st();
                    l2.x *= corr, l2.y *= corr;
                };
                if (active) {
                    // the power of two of the value scales, over the four blocks
                    const uint32_t vt = max(max(info[0], info[1]), max(info[2], info[3]));
                    if (static_cast<int>(vt >> 23) > vexp) {   // the same for all rows
                        const int to = static_cast<int>(vt >> 23);
                        rescale(__uint_as_float(static_cast<uint32_t>(max(1, 127 + vexp - to)) << 23), 0);
                        vexp = to;
                    }
                    vexp_f = static_cast<float>(134 - vexp);
                    const bool plain = (unit + 1) * kTtUnit <= min(q.first, q.len) && (info[4] & info[5] & info[6] & info[7]);
#pragma unroll
                    for (int sub = 0; sub < (REP == 2 ? 1 : 2); ++sub) {
                        const int c0 = 64 * (REP == 2 ? half : sub);   // tokens of the item
                        float2 s[32];
                        {
                            uint32_t x[32], y[32];
                            tc_ld32(s_at + c0, x);
                            tc_ld32(s_at + c0 + 32, y);
                            tc_wait_ld();
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                s[i] = make_float2(__uint_as_float(x[2 * i]), __uint_as_float(x[2 * i + 1]));
                                s[16 + i] = make_float2(__uint_as_float(y[2 * i]), __uint_as_float(y[2 * i + 1]));
                            }
                        }
                        if (REP == 2 || sub == 1) {            // S may be written again
                            tc_fence_before();
                            __syncwarp();
                            if (lane == 0) mbar_arrive(&s_free[n & 1]);
                        }
                        const float4* ks = reinterpret_cast<const float4*>(sl) + c0 / 4;
                        const float4* vs = reinterpret_cast<const float4*>(sl + kTtUnit * 4) + c0 / 4;
                        uint32_t seen[2] = {0xffffffffu, 0xffffffffu};
                        if (!plain) {
#pragma unroll
                            for (int b = 0; b < 2; ++b)
                                seen[b] = have && info[4 + c0 / 32 + b] ? tree_seen(p, begin + token, token, 4 * unit + c0 / 32 + b, q.first, q.len) : 0u;
                        }
                        float top = -INFINITY;
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const float4 k4 = ks[i];
                            s[2 * i] = mul2(s[2 * i], make_float2(k4.x, k4.y));
                            s[2 * i + 1] = mul2(s[2 * i + 1], make_float2(k4.z, k4.w));
                        }
                        if (!plain) {
#pragma unroll
                            for (int i = 0; i < 32; ++i) {
                                if (!(seen[i >> 4] >> (2 * (i & 15)) & 1)) s[i].x = -INFINITY;
                                if (!(seen[i >> 4] >> (2 * (i & 15) + 1) & 1)) s[i].y = -INFINITY;
                            }
                        }
#pragma unroll
                        for (int i = 0; i < 32; ++i) top = fmaxf(top, fmaxf(s[i].x, s[i].y));
                        top *= factor;
                        if (__any_sync(0xffffffffu, top > m + kTreeSlack)) {
                            const float to = top > m ? ceilf(top) : m;   // whole binary orders: the correction is exact
                            const float corr = to > m ? ex2(m - to) : 1.0f;
                            rescale(corr, sub);
                            m = to;
                        }
                        const float2 f2 = make_float2(factor, factor);
                        const float ref = vexp_f - m;
                        const float2 r2 = make_float2(ref, ref);
                        uint32_t out[32];
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const float4 v4 = vs[i];
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                const int j = 2 * i + e;       // tokens 2 j, 2 j + 1 of the 64
                                const float2 a = fma2(s[j], f2, r2);
                                float2 pr = make_float2(ex2(a.x), ex2(a.y));
                                if (!plain) {
                                    if (!(seen[j >> 4] >> (2 * (j & 15)) & 1)) pr.x = 0.0f;
                                    if (!(seen[j >> 4] >> (2 * (j & 15) + 1) & 1)) pr.y = 0.0f;
                                }
                                l2 = add2(l2, pr);
                                float2 w = mul2(pr, e ? make_float2(v4.z, v4.w) : make_float2(v4.x, v4.y));
                                if (!plain) {                  // a slot that is not seen may hold anything
                                    if (!(seen[j >> 4] >> (2 * (j & 15)) & 1)) w.x = 0.0f;
                                    if (!(seen[j >> 4] >> (2 * (j & 15) + 1) & 1)) w.y = 0.0f;
                                }
                                const __half2 hw = __floats2half2_rn(w.x, w.y);
                                // token 32 b + 8 n + 2 cq + h stands at position 32 b + 8 cq + 2 n + h of the second product
                                out[(j >> 4) * 16 + (j & 3) * 4 + ((j >> 2) & 3)] = *reinterpret_cast<const uint32_t*>(&hw);
                            }
                        }
                        if (!o_waited) {                       // P of the item before has been read
                            if (!mbar_wait(o_done, (n - 1) & 1, kTreeSite + 3)) ok = false;
                            o_waited = true;
                            tc_fence_after();
                        }
                        tc_st32(lanes + kTtP + c0 / 2, out);
                    }
                    tc_wait_st();
                } else {
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&s_free[n & 1]);
                    if (!o_waited && !mbar_wait(o_done, (n - 1) & 1, kTreeSite + 3)) ok = false;
                }
                tc_fence_before();
                __syncwarp();
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                if (lane == 0) mbar_arrive(p_full);
            }
            // ---- the tile, or this run's piece of it
            if (ok && !mbar_wait(o_done, (n - 1) & 1, kTreeSite + 3)) ok = false;
            ok = __all_sync(0xffffffffu, ok);
            tc_fence_after();
            const bool whole = walk.whole();
            const float c1 = __uint_as_float(static_cast<uint32_t>(vexp) << 23);
            float l = ((l2.x + l2.y) * 0x1p-7f) * c1, own = 1.0f, other = 0.0f;
            float* piece = p.partial + (static_cast<size_t>(2 * blockIdx.x + (walk.u == walk.u0 ? 0 : 1)) * ROWS + row) * kTreeRow;
            if (REP == 2) {
                // the second half hands over its numerator in two parts of 64 columns, its reference point and sum with each
                m = l == 0.0f ? -INFINITY : m;
            }
#pragma unroll
            for (int part = 0; part < 2; ++part) {
                float y[64];
                {
                    uint32_t a[32], b[32];
                    tc_ld32(lanes + kTtO + 64 * part, a);
                    tc_ld32(lanes + kTtO + 64 * part + 32, b);
                    tc_wait_ld();
                    // column 32 w + 8 j + g is dimension 32 w + 4 g + j; odd ones carry 16
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        const int at = 4 * (i & 7) + (i >> 3);
                        const float f = ((i >> 3) & 1) ? 0.0625f : 1.0f;
                        y[at] = (__uint_as_float(a[i]) * f * 0x1p17f) * c1;
                        y[32 + at] = (__uint_as_float(b[i]) * f * 0x1p17f) * c1;
                    }
                }
                if (REP == 2) {
                    float* mt = meet + row * kTtMeet;
                    if (half == 1) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) reinterpret_cast<float4*>(mt)[i] = make_float4(y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]);
                        mt[64] = m, mt[65] = l;
                    }
                    asm volatile("bar.sync 1, 128;" ::: "memory");
                    if (half == 0) {
                        if (part == 0) {
                            const float mo = mt[64], lo = mt[65], to = fmaxf(m, mo);
                            own = m > -INFINITY ? ex2(m - to) : 0.0f, other = mo > -INFINITY ? ex2(mo - to) : 0.0f;
                            l = l * own + lo * other, m = to;
                        }
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const float4 x = reinterpret_cast<const float4*>(mt)[i];
                            const float xs[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                            for (int e = 0; e < 4; ++e) y[4 * i + e] = fmaf(y[4 * i + e], own, xs[e] * other);
                        }
                    }
                    asm volatile("bar.sync 1, 128;" ::: "memory");
                }
                if (ok && have && half == 0) {
                    if (whole) {
                        const float inv = l > 0.0f ? 1.0f / l : 0.0f;
                        uint4* dst = reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.out) + (static_cast<size_t>(begin + token) * p.Hq + hq) * kKvD + 64 * part);
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            uint32_t bits[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const __nv_bfloat162 t = __floats2bfloat162_rn(l > 0.0f ? y[8 * i + 2 * e] * inv : 0.0f, l > 0.0f ? y[8 * i + 2 * e + 1] * inv : 0.0f);
                                bits[e] = *reinterpret_cast<const uint32_t*>(&t);
                            }
                            dst[i] = make_uint4(bits[0], bits[1], bits[2], bits[3]);
                        }
                    } else {
                        float4* dst = reinterpret_cast<float4*>(piece + 64 * part);
#pragma unroll
                        for (int i = 0; i < 16; ++i) dst[i] = make_float4(y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]);
                    }
                }
            }
            if (ok && have && half == 0 && !whole) *reinterpret_cast<float2*>(piece + kKvD) = make_float2(m, l);
            tc_fence_before();   // O and Q have been read: the next tile's products may write
            if (walk.b0 == 0 && !whole) mine = walk.unfinished(blockIdx.x);
        }
        if (tid == 0) p.desc[blockIdx.x] = ok ? mine : make_int4(0, 0, 0, 0);
    } else if (warp < 12) {
        // ------------------------------------------------------------------ conversion: block `blk` of the items of one parity
        const int k = warp - 4, blk = k & 3, par = k >> 2;
        const int cq = lane >> 3, g = lane & 7;
        const int page_blocks = p.pages.page_tokens / kPgTokens;
        uint8_t* my_raw = raw + k * kTtRing * kPgBlock;
        TtItems<ROWS> ahead, now;
        now.start(p);
        if (now.valid && par == 1) now.next(p);
        ahead = now;
        uint32_t asked = 0, there = 0;                        // blocks asked for; which ring slots got one
        int page = -1;
        auto look_up = [&]() {                                // the page of `ahead`'s block: used when it is asked for, later
            page = -1;
            if (!ahead.valid) return;
            const int b = 4 * ahead.unit + blk, slot = b / page_blocks;
            if (b * kPgTokens < ahead.w.q.len) page = p.pages.table[static_cast<size_t>(ahead.w.r) * p.pages.max_pages + slot];
        };
        auto ask = [&]() {
            const int slot = asked % kTtRing;
            const int b = 4 * ahead.unit + blk;
            const bool have = ahead.valid && static_cast<unsigned>(page) < static_cast<unsigned>(p.pages.num_pages);
            there = have ? there | (1u << slot) : there & ~(1u << slot);
            if (have && lane == 0) {
                mbar_expect_tx(&raw_full[k * kTtRing + slot], kPgBlock);
                bulk_g2s(my_raw + slot * kPgBlock, p.pages.pool + ((static_cast<size_t>(page) * p.pages.H + ahead.w.h) * page_blocks + b % page_blocks) * kPgBlock,
                         kPgBlock, &raw_full[k * kTtRing + slot]);
            }
            ++asked;
            if (ahead.valid) ahead.next(p);
            if (ahead.valid) ahead.next(p);
            look_up();
        };
        look_up();
        for (int i = 0; i < kTtRing; ++i) ask();
        uint32_t phases = 0, used = 0;
        bool ok = true;
        while (now.valid && ok) {
            const int buf = par;                              // items of one parity use one pair of tiles
            const int slot = used % kTtRing;
            const bool have = there >> slot & 1;
            const uint8_t* src = my_raw + slot * kPgBlock;
            const uint32_t base = smem_u32(src);
            const uint32_t use = now.n >> 1;                  // how often this pair of tiles has been used before
            if (have) {
                if (!mbar_wait(&raw_full[k * kTtRing + slot], phases >> slot & 1, kTreeSite + 4)) {
                    ok = false;
                    break;
                }
                phases ^= 1u << slot;
                there &= ~(1u << slot);
            }
            if (use > 0 && !mbar_wait(&k_free[buf], (use - 1) & 1, kTreeSite + 5)) {
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
            if (use > 0 && !mbar_wait(&v_free[buf], (use - 1) & 1, kTreeSite + 6)) {
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
            ++used;
            ask();
            now.next(p);
            if (now.valid) now.next(p);
        }
        if (!ok)   // copies in flight end (or are given up) before the shared memory does
            for (int s = 0; s < kTtRing; ++s)
                if (there >> s & 1) mbar_wait(&raw_full[k * kTtRing + s], phases >> s & 1, kTreeSite + 4);
    } else {
        // ------------------------------------------------------------------ products
        TreeWalk<ROWS, kTtUnit> walk;
        walk.start(p, blockIdx.x, gridDim.x);
        if (lane == 0) {
            const uint64_t kdesc = make_kmajor_sw128_desc(smem_u32(k_tiles)), vdesc = make_kmajor_sw128_desc(smem_u32(v_tiles));
            uint32_t n = 0, tiles = 0;
            bool ok = true;
            auto scores = [&](uint32_t i) {                   // S of item i
                const uint32_t buf = i & 1, use = i >> 1;
                if (!mbar_wait(&k_full[buf], use & 1, kTreeSite + 7)) return false;
                if (use > 0 && !mbar_wait(&s_free[buf], (use - 1) & 1, kTreeSite + 8)) return false;
                tc_fence_after();
#pragma unroll
                for (int ks = 0; ks < 8; ++ks)
                    tc_mma_f16_ts(tmem + kTtS + buf * 128, tmem + kTtQ + 8 * ks, kdesc + buf * (32768 >> 4) + (ks >> 2) * (16384 >> 4) + 2 * (ks & 3), IDESC, ks != 0);
                tc_commit(&k_free[buf]);
                tc_commit(&s_full[buf]);
                return true;
            };
            for (; ok && walk.tile_here(p); walk.next(), ++tiles) {
                if (!mbar_wait(q_full, tiles & 1, kTreeSite + 9)) break;
                tc_fence_after();
                if (!scores(n)) break;
                for (int unit = walk.b0; unit < walk.b1; ++unit, ++n) {
                    const uint32_t buf = n & 1, use = n >> 1;
                    if (unit + 1 < walk.b1 && !scores(n + 1)) {
                        ok = false;
                        break;
                    }
                    if (!mbar_wait(p_full, n & 1, kTreeSite + 10) || !mbar_wait(&v_full[buf], use & 1, kTreeSite + 11)) {
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
    if (warp == 12) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    }
}

}  // namespace qift
