// The gated products of up to sixteen token rows: a stream of packed weights.
//
// Bound by HBM: 2 N K bits / 8 bytes of codes (4096 -> 14336 in two bits: 29.4 MB, 4.6 us at the copy rate) against next to nothing
// else.  One call has few rows of tiles (896 of 16 channels there), so hand-overs between warps are what has to be avoided: a pair of warps
// takes a tile, one the gate's rows, one the other matrix's, each with a ring of its own that it fills by bulk copies itself, 64
// words deep (4 KB) a slot.  A CTA's share of a call is about what its shared memory holds: two slots a warp are asked for before anything else
// happens, the wait for the preceding kernel included, the rest behind the activations.  Packed words become operands with one logic operation each
// (mma_tile_step) against activations that stand in shared memory for the whole kernel; at the end of a tile one warp of the pair hands its
// sums to the other (64-thread barrier, two buffers by turns), which writes h.
//
// 4096 -> 14336, 1 row and 8: two bits 9.4 us and 10.2, PoT 12.0 and 12.8, three bits 12.3 and 12.8, INT4 11.8 and 12.8.  From nine rows on there
// are two tiles of tokens, and this kernel is left with calls of fewer channels and PoT (16 rows: PoT 14.5; 4096 -> 9472: two bits 11.0,
// three bits 13.3, PoT 11.4; 4096 -> 4736: INT4 11.0).  The first bytes arrive some 3 us after the launch, which longer calls make up for
// (8192 -> 28672, 4 rows: 23.4 us, 5.0 TB/s).  PoT: the table lookup (7 rows, under the profiler: ALU 49 %, issue 40 %; two bits 26 and 30).
//
// The CTA itself turns q_a into the operands' order (even planes times four, or table order) and sums each token's values, so there is no
// launch before this one and no workspace.
#pragma once

#include "common.cuh"
#include "decode.cuh"
#include "gated.cuh"
#include "grouped.cuh"
#include "kv4_tree_tc.cuh"

namespace qift {

constexpr int kGsPairs = 8, kGsThreads = 64 * kGsPairs;
constexpr int kGsMaxM = 16;
constexpr int kGsWords = 64, kGsMaxSlots = 8;               // packed words per row of a slot; slots of a warp
constexpr int kGsEarly = 2;          // slots that are asked for before the activations (8 rows, 4096 -> 14336: all three 11.2 us, two 10.6, one 10.4; 1 row: 10.0, 9.6, 9.6)
constexpr int kGsSmem = 226 * 1024;

__host__ __device__ constexpr int gs_slot_bytes(int lv) { return kGsWords * tile_word_bytes(lv); }
__host__ __device__ constexpr int gs_exchange_bytes(int M) { return 2 * 32 * (M > 8 ? 8 : 4) * 4; }   // of a pair: two buffers
// activations, and the tokens' sums and a flag; then, per pair, the exchange, two rings and their barriers
__host__ __device__ inline size_t gs_fixed_bytes(int M, int K, int lv) {
    return static_cast<size_t>(M) * packed_pitch(K, lv) * codes_per_word(lv) + 128;
}
__host__ __device__ inline size_t gs_pair_bytes(int M, int lv, int slots) {
    return gs_exchange_bytes(M) + 2 * static_cast<size_t>(slots) * (gs_slot_bytes(lv) + 8);
}

// A warp's sum of level * q, up to the correction by sum q (gs_result).
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

template <int LV, int NT, bool PROBE = false>
__global__ void __launch_bounds__(kGsThreads, 1)
gated_stream_kernel(const __grid_constant__ GatedParams p, int pairs, int slots) {
    constexpr int PER = codes_per_word(LV), NPL = PER / 4;
    constexpr int NACC = LV == QIFT_LEVELS_POT ? 1 : DecodeTraits<LV>::NACC;
    constexpr int WB = tile_word_bytes(LV), SLOT = gs_slot_bytes(LV);
    constexpr int SLICE = 16 * PER;                             // activation bytes of a slice and token
    constexpr int KS = NT == 1 && LV != QIFT_LEVELS_INT3 ? 2 : 1;   // accumulators by turns: shorter chains of products
    extern __shared__ __align__(128) unsigned char smem[];
    const int M = p.M, pitch = packed_pitch(p.K, LV), slices = pitch / 16;
    const int tiles = (p.N + 15) / 16, chunks = (pitch + kGsWords - 1) / kGsWords;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int pair = warp >> 1, mat = warp & 1;
    unsigned char* ring = smem + static_cast<size_t>(warp) * slots * SLOT;
    unsigned char* act = smem + static_cast<size_t>(2 * pairs) * slots * SLOT;    // [slice][token][SLICE], pieces permuted (swizzled_group)
    int* exchange = reinterpret_cast<int*>(act + static_cast<size_t>(M) * slices * SLICE) + pair * (gs_exchange_bytes(M) / 4);
    uint64_t* full = reinterpret_cast<uint64_t*>(act + static_cast<size_t>(M) * slices * SLICE + pairs * gs_exchange_bytes(M)) + warp * slots;
    int* sum_q = reinterpret_cast<int*>(full - warp * slots + 2 * pairs * slots);  // [16]
    volatile int* fail = sum_q + kGsMaxM;
    uint64_t* never = reinterpret_cast<uint64_t*>(sum_q + kGsMaxM + 2);            // (self-test)

    pdl_launch_dependents();
    // this warp's copies run over its tiles, chunk by chunk
    int f_tile = blockIdx.x + pair * gridDim.x, f_chunk = 0;
    const int step = pairs * gridDim.x;
    const unsigned char* base = reinterpret_cast<const unsigned char*>(p.w[mat].packed);
    auto fetch = [&](int slot) {                                // one thread: the next chunk -> slot
        if (f_tile < tiles) {
            const uint32_t bytes = min(kGsWords, pitch - f_chunk * kGsWords) * WB;
            mbar_expect_tx(&full[slot], bytes);
            bulk_g2s(ring + slot * SLOT, base + static_cast<size_t>(f_tile) * pitch * WB + static_cast<size_t>(f_chunk) * SLOT, bytes, &full[slot]);
        }
    };
    auto advance = [&]() {
        if (++f_chunk == chunks) f_chunk = 0, f_tile += step;
    };
    if (pair < pairs) {
        if (elect_one()) {
            for (int s = 0; s < slots; ++s) mbar_init(&full[s], 1);
            if (PROBE && warp == 0) mbar_init(never, 1);
            mbar_fence_init();
        }
        __syncwarp();
        for (int s = 0; s < min(slots, kGsEarly); ++s, advance())   // the weights depend on no kernel before this one
            if (elect_one()) fetch(s);
    }
    if (tid <= kGsMaxM) sum_q[tid] = 0;                         // and the flag behind them
    __syncthreads();
    pdl_wait();

    // -------------------------------------------------------------------- the activations
    {
        // Asked for four pieces a thread at a time, and before the rest of the weights: behind those they arrived 2 us later.  Eight neighbouring
        // threads are always at the same token.
        constexpr int BATCH = 4;
        const int pieces = slices * (SLICE / 16), all = M * pieces;
        for (int i0 = 0; i0 < all; i0 += BATCH * kGsThreads) {
            uint4 v[BATCH];
#pragma unroll
            for (int b = 0; b < BATCH; ++b) {
                const int i = i0 + b * kGsThreads + tid, m = i / pieces, q = i - m * pieces;
                v[b] = make_uint4(0, 0, 0, 0);
                if (i < all) {
                    const int8_t* src = p.q_a + static_cast<size_t>(m) * p.K + 16 * q;
                    if (PER == 16 || p.K % 16 == 0) {
                        if (16 * q < p.K) v[b] = *reinterpret_cast<const uint4*>(src);
                    } else {                                    // rows of eight-byte alignment
                        if (16 * q < p.K) *reinterpret_cast<uint2*>(&v[b].x) = *reinterpret_cast<const uint2*>(src);
                        if (16 * q + 8 < p.K) *reinterpret_cast<uint2*>(&v[b].z) = *reinterpret_cast<const uint2*>(src + 8);
                    }
                }
            }
            if (i0 + BATCH * kGsThreads >= all && pair < pairs) {   // the last of them are on their way
                for (int s = min(slots, kGsEarly); s < slots; ++s, advance())
                    if (elect_one()) fetch(s);
            }
#pragma unroll
            for (int b = 0; b < BATCH; ++b) {
                const int i = i0 + b * kGsThreads + tid, m = i / pieces, q = i - m * pieces;
                const uint32_t u[4] = {v[b].x, v[b].y, v[b].z, v[b].w};
                int sum = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) sum = __dp4a(static_cast<int>(u[j]), 0x01010101, sum);
                if constexpr (LV == QIFT_LEVELS_POT) v[b] = pot_lut_order(v[b]);
                else if constexpr (LV == QIFT_LEVELS_INT4) v[b].x = (v[b].x << 4) & 0xf0f0f0f0u, v[b].z = (v[b].z << 4) & 0xf0f0f0f0u;
                else v[b].x = (v[b].x << 2) & 0xfcfcfcfcu, v[b].z = (v[b].z << 2) & 0xfcfcfcfcu;   // |q| <= 8: the products fit a byte
                if (i < all) {
                    const int sl = q / (SLICE / 16), piece = q - sl * (SLICE / 16);
                    *reinterpret_cast<uint4*>(act + (static_cast<size_t>(sl) * M + m) * SLICE + 16 * swizzled_group(piece, m, PER == 16)) = v[b];
                }
                if constexpr (LV != QIFT_LEVELS_POT && LV != QIFT_LEVELS_INT3) {
                    if (i0 + b * kGsThreads >= all) break;      // the same for all threads
#pragma unroll
                    for (int o = 4; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                    if ((lane & 7) == 0 && i < all) atomicAdd(&sum_q[m], sum);
                }
            }
        }
    }
    __syncthreads();
    if (pair >= pairs) return;

    // -------------------------------------------------------------------- a tile's rows of one matrix
    const int g = lane >> 2, cq = lane & 3;
    uint32_t q_at[NT][NPL];                                     // the lane's pieces of a slice; columns beyond M repeat the last token, nobody reads them
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int tok = min(nt * 8 + g, M - 1);
#pragma unroll
        for (int i = 0; i < NPL; ++i) q_at[nt][i] = smem_u32(act) + tok * SLICE + 16 * swizzled_group(NPL * cq + i, tok, PER == 16);
    }
    float sa[NT][2];
    int sq[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int m = min(nt * 8 + 2 * cq + j, M - 1);
            sa[nt][j] = p.s_a[m], sq[nt][j] = sum_q[m];
        }
    const GateFunction function(p.act);
    GatedWait<PROBE> wait(p.probe, never, warp);
    bool ok = true;
    int s = 0;
    uint32_t ph = 0, turn = 0;
    for (int t = blockIdx.x + pair * gridDim.x; t < tiles; t += step, turn ^= 1) {
        float sg[2] = {}, su[2] = {};
        if (mat == 0) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int n = t * 16 + g + 8 * j;
                if (n < p.N) sg[j] = __ldg(p.w[0].s_n + n), su[j] = __ldg(p.w[1].s_n + n);
            }
        }
        int acc[KS][NT][NACC][4] = {};
        for (int c = 0; c < chunks; ++c) {
            // a wait that has run out once is not tried again; the warp goes on to the barriers that its partner waits at
            if (ok) ok = __all_sync(0xffffffffu, wait(&full[s], ph, 81));
            const uint32_t w0 = smem_u32(ring + s * SLOT) + lane * 16;
            auto slice = [&](int sl, auto ks) {
                const uint32_t w = w0 + sl * (16 * WB), q = static_cast<uint32_t>((c * (kGsWords / 16) + sl) * M * SLICE);
                uint32_t qb[NT][4 * NPL];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < NPL; ++i) {
                        const uint4 v = lds128(q_at[nt][i] + q);
                        qb[nt][4 * i] = v.x, qb[nt][4 * i + 1] = v.y, qb[nt][4 * i + 2] = v.z, qb[nt][4 * i + 3] = v.w;
                    }
                const uint4 wa = lds128(w), wb = lds128(w + 512);
                constexpr int k = decltype(ks)::value;
                if constexpr (LV == QIFT_LEVELS_INT3) mma_tile_step_int3<NT>(acc[k], wa, wb, lds128(w + 1024), qb);
                else if constexpr (LV == QIFT_LEVELS_POT) mma_tile_step_pot_lut<NT>(acc[k], wa, wb, qb);
                else mma_tile_step<LV, NT, true>(acc[k], wa, wb, qb);
            };
            const int here = min(kGsWords / 16, slices - c * (kGsWords / 16));
            if (here == kGsWords / 16) {
#pragma unroll
                for (int sl = 0; sl < kGsWords / 16; sl += 2) {
                    slice(sl, std::integral_constant<int, 0>{});
                    slice(sl + 1, std::integral_constant<int, KS - 1>{});
                }
            } else {
                for (int sl = 0; sl < here; ++sl) slice(sl, std::integral_constant<int, 0>{});
            }
            __syncwarp();                                       // every lane has read the slot before it is filled again
            if (ok && elect_one()) fetch(s);
            advance();
            if (ok && ++s == slots) s = 0, ph ^= 1;
        }
        int sum[NT][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                int v[NACC];
#pragma unroll
                for (int a = 0; a < NACC; ++a) v[a] = KS == 2 ? acc[0][nt][a][i] + acc[KS - 1][nt][a][i] : acc[0][nt][a][i];
                sum[nt][i] = gs_result<LV>(gs_partial<LV, NACC>(v), sq[nt][i & 1]);
            }
        int* buffer = exchange + turn * 32 * NT * 4 + lane;
        if (mat == 1) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 4; ++i) buffer[(nt * 4 + i) * 32] = sum[nt][i];
        }
        if (!ok) *fail = 1;
        asm volatile("bar.sync %0, 64;" ::"r"(1 + pair) : "memory");
        if (mat == 0 && !*fail) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int m = nt * 8 + 2 * cq + (i & 1), n = t * 16 + g + 8 * (i >> 1);
                    const int up = buffer[(nt * 4 + i) * 32];
                    const float h = gated_value(sum[nt][i], up, sa[nt][i & 1], sg[i >> 1], su[i >> 1], function);
                    if (m < M && n < p.N) {
                        const size_t at = static_cast<size_t>(m) * p.N + n;
                        if (p.h_bf16) static_cast<uint16_t*>(p.H)[at] = f32_to_bf16_bits(h);
                        else static_cast<float*>(p.H)[at] = h;
                        if (p.w[0].acc_debug) p.w[0].acc_debug[at] = sum[nt][i];
                        if (p.w[1].acc_debug) p.w[1].acc_debug[at] = up;
                    }
                }
        }
    }
    // given up: what has been asked for still arrives before the warp ends (slots behind the one that failed, their next fill)
    for (int i = 0; !ok && i < slots; ++i) mbar_wait(&full[(s + i) % slots], s + i < slots ? ph : ph ^ 1, 81, 1000000ull);
}

}  // namespace qift
