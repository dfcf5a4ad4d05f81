// The gated products of up to sixteen token rows: a stream of packed weights.
//
// Bound by HBM: 2 N K bits / 8 bytes of codes (4096 -> 14336 in two bits: 29.4 MB, 4.6 us at the copy rate) against next to nothing
// else.  One call has few 128-row items, so the unit here is small: 16 channels of both matrices, 128 words deep (2 x 8 KB, two bulk
// copies), and a CTA's share of a call is about what its shared memory holds -- nearly all of it is asked for before the CTA
// does anything else, the wait for the preceding kernel included.
//
//   warp 16     producer: fills a ring of units
//   warps 0-15  one (matrix, 16-word slice) of a unit each: packed words become operands with one logic operation each
//               (mma_tile_step) against activations that stand in shared memory for the whole kernel
// The CTA itself turns q_a into the operands' order (even planes times four, or table order) and sums each token's values, so there is no
// launch before this one and no workspace.  After a tile's last chunk the eight slices' sums of each matrix meet in shared memory (two
// buffers by turns, one barrier a tile): an integer per output, since the place values divide each warp's sum exactly.
#pragma once

#include "common.cuh"
#include "decode.cuh"
#include "gated.cuh"
#include "grouped.cuh"
#include "kv4_tree_tc.cuh"

namespace qift {

constexpr int kGsWarps = 16, kGsConsumers = 32 * kGsWarps, kGsThreads = kGsConsumers + 32;
constexpr int kGsMaxM = 16;
constexpr int kGsSmem = 226 * 1024;

__host__ __device__ constexpr int gs_unit_bytes(int lv) { return 2 * kChunkWords * tile_word_bytes(lv); }
// activations, two reduction buffers, sums and scales of the tokens, and a flag
__host__ __device__ inline size_t gs_fixed_bytes(int M, int K, int lv) {
    return static_cast<size_t>(M) * packed_pitch(K, lv) * codes_per_word(lv) + 2 * static_cast<size_t>(kGsWarps) * M * 64 + 256;
}
__host__ __device__ inline int gs_stages(int M, int K, int lv) {
    const size_t fixed = gs_fixed_bytes(M, K, lv);
    return fixed >= kGsSmem ? 0 : static_cast<int>((kGsSmem - fixed) / (gs_unit_bytes(lv) + 16));
}

// A warp's sum of level * q over its slices, up to the correction by sum q (gs_result).
template <int LV, int NACC>
__device__ __forceinline__ int gs_partial(const int (&v)[NACC]) {
    if constexpr (LV == QIFT_LEVELS_POT) return v[0];           // table lookup: the operands were the levels
    else if constexpr (LV == QIFT_LEVELS_INT4 || LV == QIFT_LEVELS_INT3) return level_sum<LV, true, NACC>(v, 0);
    else return (v[0] >> acc_shift<LV, true>(0)) + (v[1] >> acc_shift<LV, true>(1));
}
template <int LV>
__device__ __forceinline__ int gs_result(int S, int sum_q) {
    if constexpr (LV == QIFT_LEVELS_MNZ) return 2 * S - 3 * sum_q;
    if constexpr (LV == QIFT_LEVELS_SYM) return S - 2 * sum_q;
    if constexpr (LV == QIFT_LEVELS_INT4) return S - 8 * sum_q;
    return S;
}

template <int LV, int NT>
__global__ void __launch_bounds__(kGsThreads, 1)
gated_stream_kernel(const __grid_constant__ GatedParams p, int stages) {
    constexpr int PER = codes_per_word(LV), NPL = PER / 4;
    constexpr int NACC = LV == QIFT_LEVELS_POT ? 1 : DecodeTraits<LV>::NACC;
    constexpr int WB = tile_word_bytes(LV), HALF = kChunkWords * WB, UNIT = 2 * HALF;
    constexpr int SLICE = 16 * PER;                             // activation bytes of a slice and token
    extern __shared__ __align__(128) unsigned char smem[];
    const int M = p.M, pitch = packed_pitch(p.K, LV), slices = pitch / 16;
    const int tiles = (p.N + 15) / 16, chunks = (pitch + kChunkWords - 1) / kChunkWords;
    unsigned char* ring = smem;
    unsigned char* act = ring + static_cast<size_t>(stages) * UNIT;               // [slice][token][SLICE], pieces permuted (swizzled_group)
    int* red = reinterpret_cast<int*>(act + static_cast<size_t>(M) * slices * SLICE);   // [2][warp][token][row]
    uint64_t* full = reinterpret_cast<uint64_t*>(red + 2 * kGsWarps * M * 16);
    uint64_t* empty = full + stages;
    int* sum_q = reinterpret_cast<int*>(empty + stages);                          // [16]
    volatile int* fail = sum_q + kGsMaxM;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

    pdl_launch_dependents();
    if (tid == 0) {
        for (int s = 0; s < stages; ++s) mbar_init(&full[s], 1), mbar_init(&empty[s], kGsWarps);
        mbar_fence_init();
        *fail = 0;
    }
    if (tid < kGsMaxM) sum_q[tid] = 0;
    __syncthreads();

    if (warp == kGsWarps) {
        // ---------------------------------------------------------------- producer: the weights depend on no kernel before this one
        int s = 0, k = 0;
        uint32_t ph = 0;
        for (int t = blockIdx.x; t < tiles; t += gridDim.x) {
            const size_t tile = static_cast<size_t>(t) * pitch * WB;
            for (int c = 0; c < chunks; ++c, ++k) {
                if (k >= stages && !mbar_wait_near(&empty[s], ph, 80)) {
                    *fail = 1;
                    return;
                }
                if (elect_one()) {
                    const uint32_t bytes = min(kChunkWords, pitch - c * kChunkWords) * WB;
                    mbar_expect_tx(&full[s], 2 * bytes);
#pragma unroll
                    for (int i = 0; i < 2; ++i)
                        bulk_g2s(ring + s * UNIT + i * HALF, reinterpret_cast<const unsigned char*>(p.w[i].packed) + tile + static_cast<size_t>(c) * HALF,
                                 bytes, &full[s]);
                }
                __syncwarp();
                if (++s == stages) s = 0, ph ^= (k >= stages);
            }
        }
        return;
    }

    // -------------------------------------------------------------------- consumers: first the activations
    pdl_wait();
    {
        const int pieces = slices * (SLICE / 16), all = M * pieces;
        for (int i0 = 0; i0 < all; i0 += kGsConsumers) {         // eight neighbouring threads are always at the same token
            const int i = i0 + tid, m = i / pieces, q = i - m * pieces;
            int sum = 0;
            if (i < all) {
                uint4 v = make_uint4(0, 0, 0, 0);
                const int8_t* src = p.q_a + static_cast<size_t>(m) * p.K + 16 * q;
                if (PER == 16 || p.K % 16 == 0) {
                    if (16 * q < p.K) v = *reinterpret_cast<const uint4*>(src);
                } else {                                        // rows of eight-byte alignment
                    if (16 * q < p.K) *reinterpret_cast<uint2*>(&v.x) = *reinterpret_cast<const uint2*>(src);
                    if (16 * q + 8 < p.K) *reinterpret_cast<uint2*>(&v.z) = *reinterpret_cast<const uint2*>(src + 8);
                }
                const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) sum = __dp4a(static_cast<int>(u[j]), 0x01010101, sum);
                if constexpr (LV == QIFT_LEVELS_POT) v = pot_lut_order(v);
                else if constexpr (LV == QIFT_LEVELS_INT4) v.x = (v.x << 4) & 0xf0f0f0f0u, v.z = (v.z << 4) & 0xf0f0f0f0u;
                else v.x = (v.x << 2) & 0xfcfcfcfcu, v.z = (v.z << 2) & 0xfcfcfcfcu;   // |q| <= 8: the products fit a byte
                const int sl = q / (SLICE / 16), piece = q - sl * (SLICE / 16);
                *reinterpret_cast<uint4*>(act + (static_cast<size_t>(sl) * M + m) * SLICE + 16 * swizzled_group(piece, m, PER == 16)) = v;
            }
#pragma unroll
            for (int o = 4; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            if ((lane & 7) == 0 && i < all) atomicAdd(&sum_q[m], sum);
        }
    }
    const int e_row = tid & 15, e_m = tid >> 4;                  // this thread's output of a tile
    const float e_sa = e_m < M ? p.s_a[e_m] : 0.0f;
    asm volatile("bar.sync 1, %0;" ::"n"(kGsConsumers) : "memory");
    const int e_sq = e_m < M ? sum_q[e_m] : 0;

    const int g = lane >> 2, cq = lane & 3, mat = warp >> 3, slice = warp & 7;
    int tok[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) tok[nt] = min(nt * 8 + g, M - 1);   // columns beyond M repeat the last token, nobody reads them
    bool ok = true;
    int s = 0;
    uint32_t ph = 0, turn = 0;
    for (int t = blockIdx.x; t < tiles; t += gridDim.x, turn ^= 1) {
        const int n = t * 16 + e_row;
        const bool on = e_m < M && n < p.N;
        float sg = 0.0f, su = 0.0f;
        if (on) sg = __ldg(p.w[0].s_n + n), su = __ldg(p.w[1].s_n + n);
        int acc[NT][NACC][4] = {};
        for (int c = 0; c < chunks; ++c) {
            // a wait that has run out once is not tried again; the warp goes on to the barriers that the others wait at
            if (ok && !mbar_wait_near(&full[s], ph, 81)) ok = false, *fail = 1;
            const int at = c * (kChunkWords / 16) + slice;       // the slice among the row's
            if (ok && at < slices) {
                const uint32_t w = smem_u32(ring + s * UNIT + mat * HALF) + slice * (16 * WB) + lane * 16;
                const uint32_t q = smem_u32(act) + static_cast<uint32_t>(at) * M * SLICE;
                uint32_t qb[NT][4 * NPL];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < NPL; ++i) {
                        const uint4 v = lds128(q + tok[nt] * SLICE + 16 * swizzled_group(NPL * cq + i, tok[nt], PER == 16));
                        qb[nt][4 * i] = v.x, qb[nt][4 * i + 1] = v.y, qb[nt][4 * i + 2] = v.z, qb[nt][4 * i + 3] = v.w;
                    }
                const uint4 wa = lds128(w), wb = lds128(w + 512);
                if constexpr (LV == QIFT_LEVELS_INT3) mma_tile_step_int3<NT>(acc, wa, wb, lds128(w + 1024), qb);
                else if constexpr (LV == QIFT_LEVELS_POT) mma_tile_step_pot_lut<NT>(acc, wa, wb, qb);
                else mma_tile_step<LV, NT, true>(acc, wa, wb, qb);
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&empty[s]);
            if (++s == stages) s = 0, ph ^= 1;
        }
        int* mine = red + (turn * kGsWarps + warp) * M * 16;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int m = nt * 8 + 2 * cq + (i & 1);
                int v[NACC];
#pragma unroll
                for (int a = 0; a < NACC; ++a) v[a] = acc[nt][a][i];
                if (m < M) mine[m * 16 + g + ((i & 2) ? 8 : 0)] = gs_partial<LV, NACC>(v);
            }
        asm volatile("bar.sync 1, %0;" ::"n"(kGsConsumers) : "memory");
        if (on && !*fail) {
            const int* from = red + turn * kGsWarps * M * 16 + e_m * 16 + e_row;
            int S[2] = {};
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int w = 0; w < 8; ++w) S[i] += from[(8 * i + w) * M * 16];
            gated_store(p, static_cast<size_t>(e_m) * p.N + n, gs_result<LV>(S[0], e_sq), gs_result<LV>(S[1], e_sq), e_sa, sg, su);
        }
    }
}

}  // namespace qift
