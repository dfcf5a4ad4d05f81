// Low-rank adapters of many requests beside a shared projection: out[m] = y[m] + scaling_a * B_a (A_a x[m]).
//
// Two launches: t = A x (sums over K, split over CTAs) and out = y + scaling * B t.  Both are bound by memory -- the adapters of the
// requests for single tokens, x, y and out for prompts -- so they run on mma.sync (bf16, fp32 sums): which k stands at which place
// of an instruction is free as long as both operands agree, so a lane reads 16 contiguous bytes of x and of A (eight k of a row:
// two k-steps) and 8 of B.
//   lora_down_kernel, lora_up_kernel             requests of few rows: a CTA's item is up to 16 rows of a request, its eight warps share
//                                                out K or N; everything comes straight from global memory
//   lora_down_wide_kernel, lora_up_wide_kernel   longer ones: up to 128 rows, 16 per warp; the adapter's rows, which all warps need, are
//                                                staged in shared memory three steps deep (read by every warp through L1 instead, the
//                                                second kernel took 147 us for 3259 rows, rank 64, N = 14336)
// fp32 rows enter in three bf16 parts (exact to 2^-25; an infinite value leaves NaN parts, its row no numbers), t in two beside bf16 results
// (2^-17 of t, next to a result rounded at 2^-9) and in three beside fp32 ones.  fp32 results over K = 11008 are within 3.4e-7 of 64 bits.
// 7 requests of up to 11 fp32 rows, rank 24, 4096 -> 1024: 9.9 us; 5 of up to 800, rank 64, 4096 -> 4096: 86 us.
#pragma once

#include "common.cuh"
#include "decode_tc.cuh"
#include "kv4_paged.cuh"

namespace qift {

struct LoraParams {
    const void* x;            // [M][K]
    const uint16_t* A;        // bf16 [adapters][rank][K]
    const uint16_t* B;        // bf16 [adapters][N][rank]
    const float* scaling;     // [adapters]
    const int32_t* row_start; // [R + 1]
    const int32_t* adapter;   // [R]
    const void* y;            // [M][N] or nullptr (zeros)
    void* out;                // [M][N]
    float* t;                 // workspace: fp32 [splits][M][rank]
    int M, N, K, rank, adapters, R;
    int splits, k_slice;      // slices of K, each k_slice long (a multiple of 32)
    int n_slice;              // columns of a CTA of the second kernel (a multiple of 256)
};

constexpr int kLoraThreads = 256;
constexpr int kLoraWarps = kLoraThreads / 32;
constexpr int kLoraMaxRank = 128;
constexpr int kLoraMaxRows = 0x7fffff00;   // a row index and a tile more fit 32 bits
constexpr int kLoraMaxSize = 0x7ff00000;   // N, K: an index and all slices' roundings (592 x 256, 16 x 64) and steps more fit 32 bits

__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Takes the nearest bf16 pair off (x, y).
__device__ __forceinline__ uint32_t take_bf16(float& x, float& y) {
    const __nv_bfloat162 b = __floats2bfloat162_rn(x, y);
    const uint32_t bits = *reinterpret_cast<const uint32_t*>(&b);
    x -= __uint_as_float(bits << 16), y -= __uint_as_float(bits & 0xffff0000u);
    return bits;
}

// acc += 32 k of fp32 rows in three parts.  The matrix instruction cuts its sums off instead of rounding them, always towards zero: one
// accumulator through all of K = 11008 ended up to 5e-5 short.  So 32 k are summed from zero, the small parts first, and join by a rounded
// addition.  (bf16 rows, two instructions per 32 k, lose 2e-5 at that length beside the 2^-9 of their result.)
__device__ __forceinline__ void lora_add_parts(float (&acc)[4], const uint32_t (&a)[3][2][4], const uint4& b) {
    float sum[4] = {};
#pragma unroll
    for (int part = 2; part >= 0; --part) {
        mma_bf16(sum, a[part][0], b.x, b.y);
        mma_bf16(sum, a[part][1], b.z, b.w);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i] += sum[i];
}

// The CTA's item: rows [m0, m1) of a request and its adapter (-1: none); false when there is no such item.
template <int WM>
__device__ __forceinline__ bool lora_item(const LoraParams& p, int& m0, int& m1, int& adapter) {
    constexpr int kRows = 16 * WM;
    auto span = [&](int r, int& a, int& b) { a = max(0, p.row_start[r]), b = min(p.M, p.row_start[r + 1]); };
    int inner;
    const int r = kv_find_request(blockIdx.x, p.R, inner, [&](int q) {
        int a, b;
        span(q, a, b);
        return b > a ? (b - a + kRows - 1) / kRows : 0;
    });
    if (r < 0) return false;
    int a, b;
    span(r, a, b);
    m0 = a + inner * kRows, m1 = min(b, m0 + kRows);
    const int id = p.adapter[r];
    adapter = id >= 0 && id < p.adapters ? id : -1;
    return true;
}

// ---- t[split][m][j] = sum over the slice of x[m][k] A[j][k].  RS: rank in steps of 16, rounded up
template <bool BF16, int RS>
__global__ void __launch_bounds__(kLoraThreads)
lora_down_kernel(const LoraParams p) {
    constexpr int kParts = BF16 ? 1 : 3;
    __shared__ float red[kLoraWarps / 2][16][16 * RS + 4];   // of half of the warps
    pdl_launch_dependents();
    pdl_wait();
    int m0, m1, id;
    if (!lora_item<1>(p, m0, m1, id) || id < 0) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, cq = lane & 3;
    const int k0 = blockIdx.y * p.k_slice, k1 = min(p.K, k0 + p.k_slice);
    const int row[2] = {m0 + g, m0 + g + 8};
    const bool have[2] = {row[0] < m1, row[1] < m1};
    const uint16_t* A = p.A + static_cast<size_t>(id) * p.rank * p.K;
    float acc[2 * RS][4];
#pragma unroll
    for (int j = 0; j < 2 * RS; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[j][i] = 0.0f;
    constexpr int kStep = 32;                               // k of a trip: eight per lane of a row
    constexpr int kStride = kStep * kLoraWarps;
    constexpr int kX = BF16 ? 1 : 2;                        // 16-byte pieces of a lane's eight values
    constexpr int kAhead = 2;                               // trips that x is asked for ahead (A comes from L2, x from memory)
    uint4 x[kAhead][2][kX];
    auto fetch = [&](uint4 (&to)[2][kX], int k) {
        const int kk = k + 8 * cq;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < kX; ++i) {
                to[h][i] = make_uint4(0u, 0u, 0u, 0u);
                if (kk < k1 && have[h])
                    to[h][i] = reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(p.x) + (static_cast<size_t>(row[h]) * p.K + kk) * (BF16 ? 2 : 4))[i];
            }
    };
    const int begin = k0 + kStep * warp;
#pragma unroll
    for (int i = 0; i < kAhead; ++i) fetch(x[i], begin + i * kStride);
    auto trip = [&](int k, uint4 (&now)[2][kX]) {
        const int kk = k + 8 * cq;
        const bool in = kk < k1;                            // K is a multiple of eight
        uint4 b[2 * RS];
#pragma unroll
        for (int j = 0; j < 2 * RS; ++j) {
            b[j] = make_uint4(0u, 0u, 0u, 0u);
            if (in && 8 * j < p.rank) b[j] = *reinterpret_cast<const uint4*>(A + static_cast<size_t>(8 * j + g) * p.K + kk);
        }
        uint4 mine[2][kX];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < kX; ++i) mine[h][i] = now[h][i];
        fetch(now, k + kAhead * kStride);
        if constexpr (BF16) {
            const uint32_t a0[4] = {mine[0][0].x, mine[1][0].x, mine[0][0].y, mine[1][0].y}, a1[4] = {mine[0][0].z, mine[1][0].z, mine[0][0].w, mine[1][0].w};
#pragma unroll
            for (int j = 0; j < 2 * RS; ++j) {
                if (8 * j >= p.rank) break;
                mma_bf16(acc[j], a0, b[j].x, b[j].y);
                mma_bf16(acc[j], a1, b[j].z, b[j].w);
            }
        } else {
            float v[2][8];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < kX; ++i) {
                    v[h][4 * i] = __uint_as_float(mine[h][i].x), v[h][4 * i + 1] = __uint_as_float(mine[h][i].y);
                    v[h][4 * i + 2] = __uint_as_float(mine[h][i].z), v[h][4 * i + 3] = __uint_as_float(mine[h][i].w);
                }
            uint32_t a[kParts][2][4];                       // part, k-step
#pragma unroll
            for (int part = 0; part < kParts; ++part)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int e = 0; e < 4; ++e) a[part][e >> 1][2 * (e & 1) + h] = take_bf16(v[h][2 * e], v[h][2 * e + 1]);
#pragma unroll
            for (int j = 0; j < 2 * RS; ++j) {
                if (8 * j >= p.rank) break;
                lora_add_parts(acc[j], a, b[j]);
            }
        }
    };
    for (int k = begin; k < k1; k += kAhead * kStride) {
        trip(k, x[0]);
        if (k + kStride < k1) trip(k + kStride, x[1]);
    }
    float* t = p.t + static_cast<size_t>(blockIdx.y) * p.M * p.rank;
    constexpr int kHalf = kLoraWarps / 2;
    if (warp >= kHalf) {
#pragma unroll
        for (int j = 0; j < 2 * RS; ++j) {
            *reinterpret_cast<float2*>(&red[warp - kHalf][g][8 * j + 2 * cq]) = make_float2(acc[j][0], acc[j][1]);
            *reinterpret_cast<float2*>(&red[warp - kHalf][g + 8][8 * j + 2 * cq]) = make_float2(acc[j][2], acc[j][3]);
        }
    }
    __syncthreads();
    if (warp < kHalf) {
#pragma unroll
        for (int j = 0; j < 2 * RS; ++j) {
            float2* at = reinterpret_cast<float2*>(&red[warp][g][8 * j + 2 * cq]);
            float2* at8 = reinterpret_cast<float2*>(&red[warp][g + 8][8 * j + 2 * cq]);
            *at = make_float2(at->x + acc[j][0], at->y + acc[j][1]);
            *at8 = make_float2(at8->x + acc[j][2], at8->y + acc[j][3]);
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < (m1 - m0) * p.rank; i += kLoraThreads) {
        const int m = i / p.rank, j = i - m * p.rank;
        float s = 0.0f;
#pragma unroll
        for (int w = 0; w < kHalf; ++w) s += red[w][m][j];
        t[static_cast<size_t>(m0 + m) * p.rank + j] = s;
    }
}

// The sums over the slices of t, scaled, as A operands in kParts bf16 parts: step s of 16 ranks, lane cq has ranks 16 s + 4 cq .. + 3 of
// rows g and g + 8.
template <int RS, int kParts>
__device__ __forceinline__ void lora_load_t(const LoraParams& p, int id, const int (&row)[2], const bool (&have)[2], int cq, uint32_t (&ta)[kParts][RS][4]) {
    float t[RS][2][4];
#pragma unroll
    for (int s = 0; s < RS; ++s)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < 4; ++e) t[s][h][e] = 0.0f;
    if (id >= 0) {
        const float scale = p.scaling[id];
#pragma unroll 4
        for (int sp = 0; sp < p.splits; ++sp) {
            const float* src = p.t + static_cast<size_t>(sp) * p.M * p.rank;
#pragma unroll
            for (int s = 0; s < RS; ++s)
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    if (have[h] && 16 * s + 4 * cq < p.rank) {
                        const float4 v = *reinterpret_cast<const float4*>(src + static_cast<size_t>(row[h]) * p.rank + 16 * s + 4 * cq);
                        t[s][h][0] += v.x, t[s][h][1] += v.y, t[s][h][2] += v.z, t[s][h][3] += v.w;
                    }
        }
#pragma unroll
        for (int s = 0; s < RS; ++s)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 4; ++e) t[s][h][e] *= scale;
    }
#pragma unroll
    for (int part = 0; part < kParts; ++part)
#pragma unroll
        for (int s = 0; s < RS; ++s)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                ta[part][s][h] = take_bf16(t[s][h][0], t[s][h][1]);
                ta[part][s][2 + h] = take_bf16(t[s][h][2], t[s][h][3]);
            }
}

// out of eight neighbouring columns of the lane's two rows: y plus the four column tiles' sums.
template <bool BF16>
__device__ __forceinline__ void lora_finish(const LoraParams& p, const int (&row)[2], const bool (&have)[2], int n, float (&y)[2][8], const float (&acc)[4][4]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        if (!have[h]) continue;
        const size_t at = static_cast<size_t>(row[h]) * p.N + n;
#pragma unroll
        for (int i = 0; i < 4; ++i) y[h][2 * i] += acc[i][2 * h], y[h][2 * i + 1] += acc[i][2 * h + 1];
        if constexpr (BF16) {
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const __nv_bfloat162 v = __floats2bfloat162_rn(y[h][2 * e], y[h][2 * e + 1]);
                w[e] = *reinterpret_cast<const uint32_t*>(&v);
            }
            *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.out) + at) = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
            float4* dst = reinterpret_cast<float4*>(static_cast<float*>(p.out) + at);
            dst[0] = make_float4(y[h][0], y[h][1], y[h][2], y[h][3]), dst[1] = make_float4(y[h][4], y[h][5], y[h][6], y[h][7]);
        }
    }
}

// ---- out[m][n] = y[m][n] + sum_j (scaling * sum over the slices of t)[m][j] B[n][j]
template <bool BF16, int RS>
__global__ void __launch_bounds__(kLoraThreads)
lora_up_kernel(const LoraParams p) {
    constexpr int kParts = BF16 ? 2 : 3;
    pdl_launch_dependents();
    pdl_wait();
    int m0, m1, id;
    if (!lora_item<1>(p, m0, m1, id)) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, cq = lane & 3;
    const int row[2] = {m0 + g, m0 + g + 8};
    const bool have[2] = {row[0] < m1, row[1] < m1};
    const int n_end = min(p.N, (blockIdx.y + 1) * p.n_slice);
    constexpr int kY = BF16 ? 1 : 2;                        // 16-byte pieces of a lane's eight columns
    constexpr int kStride = 32 * kLoraWarps;
    const int n_begin = blockIdx.y * p.n_slice + 32 * warp;
    uint4 yq[2][kY];                                        // y of the next trip
    auto fetch = [&](int n) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < kY; ++i) {
                yq[h][i] = make_uint4(0u, 0u, 0u, 0u);
                if (p.y && have[h] && n < n_end)
                    yq[h][i] = reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(p.y) + (static_cast<size_t>(row[h]) * p.N + n) * (BF16 ? 2 : 4))[i];
            }
    };
    fetch(n_begin + 8 * cq);
    uint32_t ta[kParts][RS][4];
    lora_load_t<RS, kParts>(p, id, row, have, cq, ta);
    const uint16_t* B = p.B + static_cast<size_t>(max(id, 0)) * p.N * p.rank;
    // 32 columns a trip, as four column tiles: column c of tile i is n0 + 8 (c / 2) + 2 i + c % 2, so that a lane ends up with eight
    // neighbouring columns of its two rows
    for (int n0 = n_begin; n0 < n_end; n0 += kStride) {
        const int n = n0 + 8 * cq;
        float y[2][8];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < kY; ++i) {
                const uint32_t w[4] = {yq[h][i].x, yq[h][i].y, yq[h][i].z, yq[h][i].w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if constexpr (BF16) y[h][2 * e] = __uint_as_float(w[e] << 16), y[h][2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
                    else y[h][4 * i + e] = __uint_as_float(w[e]);
                }
            }
        fetch(n + kStride);
        float acc[4][4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[i][e] = 0.0f;
        if (id >= 0) {
            const int nb = n0 + 8 * (g >> 1) + (g & 1);
            const bool in = n0 + 8 * (g >> 1) < n_end;
#pragma unroll
            for (int s = 0; s < RS; ++s) {
                if (16 * s >= p.rank) break;
                uint2 b[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    b[i] = make_uint2(0u, 0u);
                    if (in && 16 * s + 4 * cq < p.rank) b[i] = *reinterpret_cast<const uint2*>(B + static_cast<size_t>(nb + 2 * i) * p.rank + 16 * s + 4 * cq);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int part = 0; part < kParts; ++part) mma_bf16(acc[i], ta[part][s], b[i].x, b[i].y);
            }
        }
        if (n < n_end) lora_finish<BF16>(p, row, have, n, y, acc);
    }
}

// ------------------------------------------------------------------------------------------------ requests of many rows
constexpr int kLoraStages = 3;
__device__ __forceinline__ void cp_async16_or_zero(uint32_t dst_smem, const void* src, bool there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst_smem), "l"(src), "r"(there ? 16 : 0) : "memory");
}

// Rows of A in steps of 64 k: 128 bytes a row, 192 apart (the two rows of a quarter-warp's 128-bit reads fill all banks).
template <bool BF16, int RS>
struct LoraDownWide {
    static constexpr int kPitch = 192, kStage = 16 * RS * kPitch, kSmem = kLoraStages * kStage;
};
template <bool BF16, int RS>
__global__ void __launch_bounds__(kLoraThreads)
lora_down_wide_kernel(const LoraParams p) {
    using S = LoraDownWide<BF16, RS>;
    constexpr int kParts = BF16 ? 1 : 3;
    extern __shared__ __align__(128) uint8_t smem[];
    pdl_launch_dependents();
    pdl_wait();
    int m0, m1, id;
    if (!lora_item<kLoraWarps>(p, m0, m1, id) || id < 0) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, cq = lane & 3;
    const int k0 = blockIdx.y * p.k_slice, k1 = min(p.K, k0 + p.k_slice);
    const int row[2] = {m0 + 16 * warp + g, m0 + 16 * warp + g + 8};
    const bool have[2] = {row[0] < m1, row[1] < m1};
    const bool active = m0 + 16 * warp < m1;                // the others only help to stage
    const uint16_t* A = p.A + static_cast<size_t>(id) * p.rank * p.K;
    auto stage = [&](int trip) {
        const int k = k0 + 64 * trip;
        const uint32_t to = smem_u32(smem) + (trip % kLoraStages) * S::kStage;
        for (int i = threadIdx.x; i < 16 * RS * 8; i += kLoraThreads) {
            const int j = i >> 3, piece = i & 7, kk = k + 8 * piece;
            const bool there = j < p.rank && kk < k1;
            cp_async16_or_zero(to + j * S::kPitch + 16 * piece, there ? A + static_cast<size_t>(j) * p.K + kk : A, there);
        }
        cp_async_commit();
    };
    constexpr int kX = BF16 ? 1 : 2;
    uint4 x[2][2][kX];                                      // half of the step, row
    auto fetch = [&](int trip) {
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < kX; ++i) {
                    const int kk = k0 + 64 * trip + 32 * half + 8 * cq;
                    x[half][h][i] = make_uint4(0u, 0u, 0u, 0u);
                    if (kk < k1 && have[h])
                        x[half][h][i] = reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(p.x) + (static_cast<size_t>(row[h]) * p.K + kk) * (BF16 ? 2 : 4))[i];
                }
    };
    float acc[2 * RS][4];
#pragma unroll
    for (int j = 0; j < 2 * RS; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[j][i] = 0.0f;
    const int trips = (k1 - k0 + 63) / 64;
    fetch(0);
#pragma unroll
    for (int i = 0; i < kLoraStages - 1; ++i) stage(i);     // (steps behind the end are zeros)
    for (int trip = 0; trip < trips; ++trip) {
        cp_async_wait<kLoraStages - 2>();
        __syncthreads();                                    // this step is there, and the one before it has been read by all
        stage(trip + kLoraStages - 1);
        uint4 mine[2][2][kX];
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < kX; ++i) mine[half][h][i] = x[half][h][i];
        fetch(trip + 1);
        if (!active) continue;
        const uint32_t from = smem_u32(smem) + (trip % kLoraStages) * S::kStage + g * S::kPitch + 16 * cq;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            uint32_t a[kParts][2][4];                       // part, k-step
            if constexpr (BF16) {
                const uint4 u = mine[half][0][0], v = mine[half][1][0];
                a[0][0][0] = u.x, a[0][0][1] = v.x, a[0][0][2] = u.y, a[0][0][3] = v.y;
                a[0][1][0] = u.z, a[0][1][1] = v.z, a[0][1][2] = u.w, a[0][1][3] = v.w;
            } else {
                float v[2][8];
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < kX; ++i) {
                        v[h][4 * i] = __uint_as_float(mine[half][h][i].x), v[h][4 * i + 1] = __uint_as_float(mine[half][h][i].y);
                        v[h][4 * i + 2] = __uint_as_float(mine[half][h][i].z), v[h][4 * i + 3] = __uint_as_float(mine[half][h][i].w);
                    }
#pragma unroll
                for (int part = 0; part < kParts; ++part)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int e = 0; e < 4; ++e) a[part][e >> 1][2 * (e & 1) + h] = take_bf16(v[h][2 * e], v[h][2 * e + 1]);
            }
#pragma unroll
            for (int j = 0; j < 2 * RS; ++j) {
                if (8 * j >= p.rank) break;
                const uint4 b = lds128(from + 8 * j * S::kPitch + 64 * half);
                if constexpr (BF16) {
                    mma_bf16(acc[j], a[0][0], b.x, b.y);
                    mma_bf16(acc[j], a[0][1], b.z, b.w);
                } else {
                    lora_add_parts(acc[j], a, b);
                }
            }
        }
    }
    cp_async_wait<0>();
    float* t = p.t + static_cast<size_t>(blockIdx.y) * p.M * p.rank;
#pragma unroll
    for (int j = 0; j < 2 * RS; ++j) {
        if (8 * j >= p.rank) break;
#pragma unroll
        for (int h = 0; h < 2; ++h)
            if (have[h]) *reinterpret_cast<float2*>(t + static_cast<size_t>(row[h]) * p.rank + 8 * j + 2 * cq) = make_float2(acc[j][2 * h], acc[j][2 * h + 1]);
    }
}

// Rows of B in steps of 64 columns, in the order in which a lane group reads them: row 32 q + 8 i + g is column 32 q + 8 (g / 2) + 2 i +
// g % 2.  Rows are a multiple of 128 bytes plus 32 apart (rank 16: 32), so that the 64-bit reads of a half-warp fill all banks.
template <bool BF16, int RS>
struct LoraUpWide {
    static constexpr int kPitch = RS == 1 ? 32 : 32 * RS + 32, kStage = 64 * kPitch, kSmem = kLoraStages * kStage;
};
template <bool BF16, int RS>
__global__ void __launch_bounds__(kLoraThreads)
lora_up_wide_kernel(const LoraParams p) {
    using S = LoraUpWide<BF16, RS>;
    constexpr int kParts = BF16 ? 2 : 3;
    extern __shared__ __align__(128) uint8_t smem[];
    pdl_launch_dependents();
    pdl_wait();
    int m0, m1, id;
    if (!lora_item<kLoraWarps>(p, m0, m1, id)) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, cq = lane & 3;
    const int row[2] = {m0 + 16 * warp + g, m0 + 16 * warp + g + 8};
    const bool have[2] = {row[0] < m1, row[1] < m1};
    const bool active = m0 + 16 * warp < m1;                // the others only help to stage
    const int n_begin = blockIdx.y * p.n_slice, n_end = min(p.N, n_begin + p.n_slice);
    const uint16_t* B = p.B + static_cast<size_t>(max(id, 0)) * p.N * p.rank;
    auto stage = [&](int trip) {
        const uint32_t to = smem_u32(smem) + (trip % kLoraStages) * S::kStage;
        for (int i = threadIdx.x; i < 64 * 2 * RS; i += kLoraThreads) {
            const int c = i / (2 * RS), piece = i - c * (2 * RS), n = n_begin + 64 * trip + c;
            const int at = (c & 32) + 8 * ((c >> 1) & 3) + 2 * ((c >> 3) & 3) + (c & 1);
            const bool there = id >= 0 && n < n_end && 8 * piece < p.rank;
            cp_async16_or_zero(to + at * S::kPitch + 16 * piece, there ? B + static_cast<size_t>(n) * p.rank + 8 * piece : B, there);
        }
        cp_async_commit();
    };
    constexpr int kY = BF16 ? 1 : 2;
    uint4 yq[2][2][kY];                                     // y of the next step: half, row
    auto fetch = [&](int trip) {
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < kY; ++i) {
                    const int n = n_begin + 64 * trip + 32 * half + 8 * cq;
                    yq[half][h][i] = make_uint4(0u, 0u, 0u, 0u);
                    if (p.y && have[h] && n < n_end)
                        yq[half][h][i] = reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(p.y) + (static_cast<size_t>(row[h]) * p.N + n) * (BF16 ? 2 : 4))[i];
                }
    };
    fetch(0);
#pragma unroll
    for (int i = 0; i < kLoraStages - 1; ++i) stage(i);     // (steps behind the end are zeros)
    uint32_t ta[kParts][RS][4];
    lora_load_t<RS, kParts>(p, id, row, have, cq, ta);
    const int trips = (n_end - n_begin + 63) / 64;
    for (int trip = 0; trip < trips; ++trip) {
        cp_async_wait<kLoraStages - 2>();
        __syncthreads();                                    // this step is there, and the one before it has been read by all
        stage(trip + kLoraStages - 1);
        float y[2][2][8];
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < kY; ++i) {
                    const uint32_t w[4] = {yq[half][h][i].x, yq[half][h][i].y, yq[half][h][i].z, yq[half][h][i].w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if constexpr (BF16) y[half][h][2 * e] = __uint_as_float(w[e] << 16), y[half][h][2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
                        else y[half][h][4 * i + e] = __uint_as_float(w[e]);
                    }
                }
        fetch(trip + 1);
        if (!active) continue;
        const uint32_t from = smem_u32(smem) + (trip % kLoraStages) * S::kStage + g * S::kPitch + 8 * cq;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            float acc[4][4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][e] = 0.0f;
#pragma unroll
            for (int s = 0; s < RS; ++s) {
                if (16 * s >= p.rank) break;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint2 b = lds64(from + (32 * half + 8 * i) * S::kPitch + 32 * s);
#pragma unroll
                    for (int part = 0; part < kParts; ++part) mma_bf16(acc[i], ta[part][s], b.x, b.y);
                }
            }
            const int n = n_begin + 64 * trip + 32 * half + 8 * cq;
            if (n < n_end) lora_finish<BF16>(p, row, have, n, y[half], acc);
        }
    }
    cp_async_wait<0>();
}

}  // namespace qift
