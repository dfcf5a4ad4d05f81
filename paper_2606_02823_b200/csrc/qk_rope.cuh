// Norms of queries and keys for each head and the rotation by their positions, in one pass.
//
//     y = x / sqrt(mean(x^2) + eps) * w          (where a weight is given; over the D dimensions of a head)
//     (y_a, y_b) <- (y_a cos - y_b sin, y_b cos + y_a sin),  angle = position * inv_freq[i] for pair i
//
// Pairs are (i, i + rot / 2) or (2i, 2i + 1) of the first rot dimensions.  A thread holds eight pairs: two 16-byte pieces of a
// bf16 head (four of an fp32 one) that are rotated with one another, so nothing is exchanged but the sum of squares.  A warp takes
// the heads of one row, as many at once as D / 16 threads each allow; it works the row's sines and cosines out once, rot / 2 of them
// over its lanes, and keeps each lane's eight in registers over all heads.  Angles: the product in fp64 (position up to 2^31 times
// an fp32 frequency), its whole turns taken off there, then sincospif of what is left -- far positions lose nothing.
// Bound by HBM for many rows (every element in and out once); by latency for single tokens, whose rows are split over several warps.
#pragma once

#include "common.cuh"

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
    int total, Hq, H, D, rot, near; // near: neighbouring dimensions are pairs
    int parts;                      // warps that share a row's heads
    float eps;
};

// Eight consecutive elements as fp32 and back (one 16-byte access, or two).
template <bool BF16>
__device__ __forceinline__ void rope_load(const void* base, long long at, float (&v)[8]) {
    if constexpr (BF16) {
        const uint4 w = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(base) + at);
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) v[2 * i] = __uint_as_float(u[i] << 16), v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    } else {
        const float4* src = reinterpret_cast<const float4*>(static_cast<const float*>(base) + at);
        const float4 a = src[0], b = src[1];
        v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    }
}
template <bool BF16>
__device__ __forceinline__ void rope_store(void* base, long long at, const float (&v)[8]) {
    if constexpr (BF16) {
        uint32_t u[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] = f32_to_bf16_bits(v[2 * i]) | static_cast<uint32_t>(f32_to_bf16_bits(v[2 * i + 1])) << 16;
        *reinterpret_cast<uint4*>(static_cast<uint16_t*>(base) + at) = make_uint4(u[0], u[1], u[2], u[3]);
    } else {
        float4* dst = reinterpret_cast<float4*>(static_cast<float*>(base) + at);
        dst[0] = make_float4(v[0], v[1], v[2], v[3]), dst[1] = make_float4(v[4], v[5], v[6], v[7]);
    }
}

// LANES: threads of a head, a power of two >= D / 16 (those beyond D / 16 have nothing to do).
template <bool BF16, int LANES>
__global__ void __launch_bounds__(kRopeThreads)
qk_norm_rope_kernel(const RopeParams p) {
    __shared__ float2 turns[kRopeWarps][kRopeMaxD / 2];   // cosine, sine of the warp's row
    pdl_launch_dependents();
    pdl_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int c = lane % LANES, group = lane / LANES, groups = 32 / LANES;
    const bool on = 16 * c < p.D;
    // the two pieces of the lane: pieces of the rotated part that are pairs of one another, or two of the rest
    const int pairs = p.rot / 2, heads = p.Hq + p.H;
    const bool turned = 16 * c < p.rot;
    const int a = turned && !p.near ? 8 * c : 16 * c, b = turned && !p.near ? pairs + 8 * c : 16 * c + 8;
    float wq[2][8], wk[2][8];
#pragma unroll
    for (int i = 0; i < 8; ++i) wq[0][i] = wq[1][i] = wk[0][i] = wk[1][i] = 1.0f;
    if (on && p.q_weight) rope_load<BF16>(p.q_weight, a, wq[0]), rope_load<BF16>(p.q_weight, b, wq[1]);
    if (on && p.k_weight) rope_load<BF16>(p.k_weight, a, wk[0]), rope_load<BF16>(p.k_weight, b, wk[1]);
    const float inv_d = 1.0f / p.D;
    const long long tasks = static_cast<long long>(p.total) * p.parts, step = static_cast<long long>(gridDim.x) * kRopeWarps;
    for (long long task = blockIdx.x * static_cast<long long>(kRopeWarps) + warp; task < tasks; task += step) {
        const int row = static_cast<int>(task / p.parts), part = static_cast<int>(task - static_cast<long long>(row) * p.parts);
        const int position = p.position[row];
        if (position < 0) continue;            // the row belongs to nobody
        __syncwarp();
        for (int i = lane; i < pairs; i += 32) {
            double turn = static_cast<double>(position) * static_cast<double>(p.inv_freq[i]) * 0.15915494309189533577;
            turn -= rint(turn);
            float s, co;
            sincospif(2.0f * static_cast<float>(turn), &s, &co);
            turns[warp][i] = make_float2(co, s);
        }
        __syncwarp();
        float cs[8], sn[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float2 t = turned ? turns[warp][8 * c + i] : make_float2(1.0f, 0.0f);   // (not used where nothing turns)
            cs[i] = t.x, sn[i] = t.y;
        }
        for (int h0 = part * groups; h0 < heads; h0 += p.parts * groups) {
            const int h = h0 + group;
            const bool is_q = h < p.Hq, here = on && h < heads;
            float x[2][8] = {};
            if (here) {
                const void* src = is_q ? p.q : p.k;
                const long long at = row * (is_q ? p.q_stride : p.k_stride) + static_cast<long long>(is_q ? h : h - p.Hq) * p.D;
                rope_load<BF16>(src, at + a, x[0]), rope_load<BF16>(src, at + b, x[1]);
            }
            if (p.q_weight || p.k_weight) {     // the same for all lanes
                float sum = 0.0f;
#pragma unroll
                for (int i = 0; i < 8; ++i) sum += x[0][i] * x[0][i] + x[1][i] * x[1][i];
#pragma unroll
                for (int o = LANES / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                const float r = (is_q ? p.q_weight : p.k_weight) ? 1.0f / sqrtf(sum * inv_d + p.eps) : 1.0f;
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[j][i] *= r * (is_q ? wq[j][i] : wk[j][i]);
            }
            if (!here) continue;
            if (turned && p.near) {
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float u = x[j][2 * i], v = x[j][2 * i + 1], co = cs[4 * j + i], si = sn[4 * j + i];
                        x[j][2 * i] = u * co - v * si, x[j][2 * i + 1] = v * co + u * si;
                    }
            } else if (turned) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float u = x[0][i], v = x[1][i];
                    x[0][i] = u * cs[i] - v * sn[i], x[1][i] = v * cs[i] + u * sn[i];
                }
            }
            void* dst = is_q ? p.q_out : p.k_out;
            const long long to = row * (is_q ? p.qo_stride : p.ko_stride) + static_cast<long long>(is_q ? h : h - p.Hq) * p.D;
            rope_store<BF16>(dst, to + a, x[0]), rope_store<BF16>(dst, to + b, x[1]);
        }
    }
}

}  // namespace qift
