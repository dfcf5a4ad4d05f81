// Norms of queries and keys for each head and the rotation by their positions, in one pass.
//
//     y = x / sqrt(mean(x^2) + eps) * w          (where a weight is given; over the D dimensions of a head)
//     (y_a, y_b) <- (y_a cos - y_b sin, y_b cos + y_a sin),  angle = position * inv_freq[i] for pair i
//
// Pairs are (i, i + rot / 2) or (2i, 2i + 1) of the first rot dimensions.  A thread holds eight pairs: two 16-byte pieces of a
// bf16 head (four of an fp32 one) that are rotated with one another, so nothing is exchanged but the sum of squares.  A warp takes
// the heads of one row, as many at once as D / 16 threads each allow; it works the row's sines and cosines out once, rot / 2 of them
// over its lanes.  Angles: the product in fp64 (position up to 2^31 times
// an fp32 frequency), its whole turns taken off there (at 2^31 radians its roundings are some 1e-7 of a turn, at 10^6 nothing), then sincospif of what is
// left, rounded to fp32: at most pi 2^-24 of an angle, beside values that are rounded to fp32 themselves (fp32 rows: error 7.6e-8
// against 64 bits, 6.3e-8 where sines and cosines come from fp64).
//
// Bound by HBM for many rows, every element in and out once: 18000 rows of 32 + 8 heads in bf16 with norms take 58 us (5.7 TB/s; 111 at
// first).  A lane asks for the next heads' pieces before it works on these; a trip is heads of the queries or of the keys, so that
// nothing is chosen per lane; fp32 pairs are worked on two at a time; sines and weights stand in shared memory in the lanes' order,
// since in registers they cost spills.  (Pieces on their way through shared memory, four trips ahead, were slower: 81.)  By latency for
// single tokens.  fp32 rows by L1 and shared memory: 1237 of 32 + 32 heads, neighbours, 18.3 us (3.9 TB/s) at 77 % of L1, 32 % of issue; a lane's
// sixteen values are four 16-byte pieces 64 bytes from the next lane's, so that an access takes several passes.
#pragma once

#include "common.cuh"
#include "kv4_paged.cuh"

namespace qift {

constexpr int kRopeThreads = 256, kRopeWarps = kRopeThreads / 32;
constexpr int kRopeMaxD = 512;

struct RopeParams {
    const void* q;
    const void* k;
    void* q_out;
    void* k_out;
    long long q_stride, k_stride, qo_stride, ko_stride;   // elements from row to row
    const void* q_weight;           // [D] of the rows' type, or null: no norm
    const void* k_weight;
    const float* inv_freq;          // [rot / 2]
    const int32_t* position;        // [total]
    int total, Hq, H, D, rot;
    int parts;                      // warps that share a row's heads
    float eps;
};

// Eight consecutive elements: as they are (one 16-byte access, or two), as four fp32 pairs, and back.
template <bool BF16>
struct RopePiece {
    uint4 w[BF16 ? 1 : 2];
    __device__ __forceinline__ void load(const char* from) {
        w[0] = reinterpret_cast<const uint4*>(from)[0];
        if constexpr (!BF16) w[1] = reinterpret_cast<const uint4*>(from)[1];
    }
    __device__ __forceinline__ void values(uint64_t (&v)[4]) const {
        if constexpr (BF16) {
            const uint32_t u[4] = {w[0].x, w[0].y, w[0].z, w[0].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = pair_of(__uint_as_float(u[i] << 16), __uint_as_float(u[i] & 0xffff0000u));
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                v[2 * i] = pair_of(__uint_as_float(w[i].x), __uint_as_float(w[i].y));
                v[2 * i + 1] = pair_of(__uint_as_float(w[i].z), __uint_as_float(w[i].w));
            }
        }
    }
};
template <bool BF16>
__device__ __forceinline__ void rope_store(char* to, const uint64_t (&v)[4]) {
    float f[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) pair_to(v[i], f[2 * i], f[2 * i + 1]);
    if constexpr (BF16) {
        uint32_t u[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(u[i]) : "f"(f[2 * i + 1]), "f"(f[2 * i]));
        *reinterpret_cast<uint4*>(to) = make_uint4(u[0], u[1], u[2], u[3]);
    } else {
        float4* dst = reinterpret_cast<float4*>(to);
        dst[0] = make_float4(f[0], f[1], f[2], f[3]), dst[1] = make_float4(f[4], f[5], f[6], f[7]);
    }
}

// LANES: threads of a head, a power of two >= D / 16 (those beyond D / 16 have nothing to do).
template <bool BF16, int LANES, bool NORM, bool NEAR>
__global__ void __launch_bounds__(kRopeThreads, 4)
qk_norm_rope_kernel(const __grid_constant__ RopeParams p) {
    constexpr int GROUPS = 32 / LANES;
    // What a lane needs of its row and of the weights, lane after lane so that reads are free of bank conflicts.
    __shared__ float4 turns[kRopeWarps][4][LANES];        // of pairs 8c + 2i, + 1 of the warp's row: two cosines, two sines
    __shared__ float4 weights[2][NORM ? 4 : 1][LANES];    // of queries, of keys: four values of a lane's first, second piece
    pdl_launch_dependents();
    pdl_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int c = lane % LANES, group = lane / LANES;
    constexpr int SIZE = BF16 ? 2 : 4;
    const bool on = 16 * c < p.D;
    // the two pieces of the lane: pieces of the rotated part that are pairs of one another, or two of the rest
    const int pairs = p.rot / 2;
    const bool turned = 16 * c < p.rot;
    const int a = turned && !NEAR ? 8 * c : 16 * c, b = turned && !NEAR ? pairs + 8 * c : 16 * c + 8;
    const float inv_d = 1.0f / p.D;
    if constexpr (NORM) {
        for (int i = threadIdx.x; i < 2 * 4 * LANES; i += kRopeThreads) {
            const int k = i / (4 * LANES), j = i / LANES % 4, l = i % LANES;
            const int at = (j & 2 ? (16 * l < p.rot && !NEAR ? pairs + 8 * l : 16 * l + 8) : (16 * l < p.rot && !NEAR ? 8 * l : 16 * l)) + 4 * (j & 1);
            const void* w = k ? p.k_weight : p.q_weight;
            float v[4] = {1.0f, 1.0f, 1.0f, 1.0f};
            if (w && 16 * l < p.D) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    v[e] = BF16 ? __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t*>(w)[at + e]) << 16) : static_cast<const float*>(w)[at + e];
            }
            weights[k][j][l] = make_float4(v[0], v[1], v[2], v[3]);
        }
        __syncthreads();
    }
    // a trip is GROUPS heads of the queries or of the keys, never of both
    const int q_trips = (p.Hq + GROUPS - 1) / GROUPS, trips = q_trips + (p.H + GROUPS - 1) / GROUPS;
    const long long tasks = static_cast<long long>(p.total) * p.parts, step = static_cast<long long>(gridDim.x) * kRopeWarps;
    long long task = blockIdx.x * static_cast<long long>(kRopeWarps) + warp;
    int position = task < tasks ? p.position[task / p.parts] : -1;
    for (; task < tasks; task += step) {
        const int row = static_cast<int>(task / p.parts), part = static_cast<int>(task - static_cast<long long>(row) * p.parts);
        const int here = position;
        if (task + step < tasks) position = p.position[(task + step) / p.parts];   // asked for a row ahead
        if (here < 0) continue;                // the row belongs to nobody
        const char* const q_row = static_cast<const char*>(p.q) + row * p.q_stride * SIZE;
        const char* const k_row = static_cast<const char*>(p.k) + row * p.k_stride * SIZE;
        char* const qo_row = static_cast<char*>(p.q_out) + row * p.qo_stride * SIZE;
        char* const ko_row = static_cast<char*>(p.k_out) + row * p.ko_stride * SIZE;
        RopePiece<BF16> next[2] = {};
        auto fetch = [&](int trip) {           // the lane's pieces of its head of a trip
            const bool is_q = trip < q_trips;
            const int h = (is_q ? trip : trip - q_trips) * GROUPS + group;
            if (on && trip < trips && h < (is_q ? p.Hq : p.H)) {
                const char* head = (is_q ? q_row : k_row) + h * (p.D * SIZE);
                next[0].load(head + a * SIZE), next[1].load(head + b * SIZE);
            }
        };
        fetch(part);
        __syncwarp();
        for (int i = lane; i < pairs; i += 32) {
            double turn = static_cast<double>(here) * static_cast<double>(p.inv_freq[i]) * 0.15915494309189533577;
            turn -= rint(turn);
            float s, co;
            sincospif(2.0f * static_cast<float>(turn), &s, &co);
            float* to = &turns[warp][(i >> 1) & 3][i >> 3].x + (i & 1);
            to[0] = co, to[2] = s;
        }
        __syncwarp();
        for (int trip = part; trip < trips; trip += p.parts) {
            const bool is_q = trip < q_trips;  // the same for the whole warp
            const int h = (is_q ? trip : trip - q_trips) * GROUPS + group;
            uint64_t x[2][4];                  // (of a lane without a head, whatever the last trip left)
            next[0].values(x[0]), next[1].values(x[1]);
            fetch(trip + p.parts);             // the next heads are on their way while these are worked on
            if constexpr (NORM) {
                if (is_q ? p.q_weight : p.k_weight) {
                    uint64_t squares = 0;
#pragma unroll
                    for (int i = 0; i < 4; ++i) squares = pair_fma(x[1][i], x[1][i], pair_fma(x[0][i], x[0][i], squares));
                    float even, odd;
                    pair_to(squares, even, odd);
                    float sum = on ? even + odd : 0.0f;
#pragma unroll
                    for (int o = LANES / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                    const float r = 1.0f / sqrtf(sum * inv_d + p.eps);
                    const uint64_t rr = pair_of(r, r);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float4 v = weights[is_q ? 0 : 1][j][c];
                        uint64_t* to = &x[j >> 1][2 * (j & 1)];
                        to[0] = pair_mul(pair_mul(to[0], rr), pair_of(v.x, v.y));
                        to[1] = pair_mul(pair_mul(to[1], rr), pair_of(v.z, v.w));
                    }
                }
            }
            if (turned) {
                uint64_t cs[4], sn[4];         // cosines, sines of the lane's eight pairs, two by two: read again for every trip, there are no registers to keep them in
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float4 t = turns[warp][i][c];
                    cs[i] = pair_of(t.x, t.y), sn[i] = pair_of(t.z, t.w);
                }
                if constexpr (NEAR) {
#pragma unroll
                    for (int j = 0; j < 2; ++j)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            float u, v, c0, c1, s0, s1;
                            pair_to(x[j][i], u, v), pair_to(cs[2 * j + (i >> 1)], c0, c1), pair_to(sn[2 * j + (i >> 1)], s0, s1);
                            const float co = i & 1 ? c1 : c0, si = i & 1 ? s1 : s0;
                            x[j][i] = pair_of(u * co - v * si, v * co + u * si);
                        }
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint64_t u = x[0][i], v = x[1][i];
                        const uint64_t minus = pair_mul(v, sn[i]) ^ 0x8000000080000000ull;
                        x[0][i] = pair_fma(u, cs[i], minus), x[1][i] = pair_fma(v, cs[i], pair_mul(u, sn[i]));
                    }
                }
            }
            if (on && h < (is_q ? p.Hq : p.H)) {
                char* head = (is_q ? qo_row : ko_row) + h * (p.D * SIZE);
                rope_store<BF16>(head + a * SIZE, x[0]), rope_store<BF16>(head + b * SIZE, x[1]);
            }
        }
    }
}

}  // namespace qift
