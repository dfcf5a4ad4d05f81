// The gated products of some tens to some hundreds of token rows on the tcgen05 tensor cores, with the packed codes as the operand in
// tensor memory (as in decode_tc.cuh: they never exist as int8 in shared memory).
//
// An item is 128 channels of both matrices times one block of up to 128 token rows (N of the instruction, any multiple of 16: 48 rows
// cost what 48 cost).  The two matrices are two independent streams over one sequence of activation blocks:
//
//   warp 0        activations: per 128-byte k-block the q_a rows of the token block, one tensor copy into a swizzled stage
//   warps 1, 2    issue the products of the gate's, of the other matrix's operands: D[matrix][128 channels x tokens]
//   warps 3-10    while the products run, the token sums of the staged activations (an eighth of the rows each); then the epilogue, two
//                 warps per tensor-memory lane quarter on alternate 16-token pieces: both accumulators, h, stores of 32 channels
//   warps 11-18   expanders, one per matrix and lane quarter: packed words of their 32 channels by cp.async (kGtSlots slices ahead,
//                 across items), one to four logic operations per operand word, tcgen05.st into the matrix's four k-blocks of operands
// Activations come as they are (no prescaling, no launch before this one): the operand bytes are the codes themselves, unsigned, and the
// affine level map is undone with the token sums; the power-of-two set's bytes are its levels by table lookup, in k order.
// Token blocks of one channel tile are neighbours in the item list, so that its codes come from L2 for all but the first.
//
// Bound by the tensor cores from about 64 rows on (a 128 x N x 32 product takes N / 2 cycles, a thread issues one every 50), by the
// codes' way into an SM below (256 KB an item at about 76 GB/s).
#pragma once

#include "common.cuh"
#include "decode_tc.cuh"
#include "gated.cuh"
#include "prefill.cuh"

namespace qift {

constexpr int kGtRows = 128;                 // channels of an item
constexpr int kGtTokens = 128;               // token rows of an item, at most
constexpr int kGtThreads = 32 * 19;
constexpr int kGtEpiWarps = 8;
constexpr int kGtRing = 4;                   // k-blocks of operands in tensor memory, per matrix
constexpr int kGtOperands = 256;             // first operand column
constexpr int kGtSmem = 226 * 1024;

__host__ __device__ constexpr int gt_slot_bytes(int lv) { return 32 * (lv == QIFT_LEVELS_INT3 ? 96 : 64); }   // 32 rows of a slice
__host__ __device__ constexpr int gt_slots(int lv) { return lv == QIFT_LEVELS_INT3 ? 4 : 7; }                  // slices ahead, per expander
__host__ __device__ inline int gt_stages(int lv, int ntok) {
    const int left = (kGtSmem - 2048 - 8 * gt_slots(lv) * gt_slot_bytes(lv)) / (ntok * 128);
    return left < 10 ? left : 10;
}

struct GatedTcParams {
    GatedParams g;
    int ntok, blocks;        // token rows of a block (a multiple of 16), blocks
    int stages;
};

// Operand bytes of one k-block (128 codes) of a channel, in k order.  hi: the words of the third bits (INT3).
template <int LV>
__device__ __forceinline__ void gt_operands(const uint32_t* w, const uint32_t* hi, uint32_t (&o)[32]) {
    if constexpr (LV == QIFT_LEVELS_INT4) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            o[2 * i] = (w[i] & 0x0f0f0f0fu) ^ 0x08080808u;
            o[2 * i + 1] = ((w[i] >> 4) & 0x0f0f0f0fu) ^ 0x08080808u;
        }
    } else if constexpr (LV == QIFT_LEVELS_POT) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            uint32_t a[4];
            pot_lut_operands(w[i], a);       // codes {0,8,1,9}, {4,12,5,13}, {2,10,3,11}, {6,14,7,15} of the word
            o[4 * i] = __byte_perm(a[0], a[2], 0x6420), o[4 * i + 2] = __byte_perm(a[0], a[2], 0x7531);
            o[4 * i + 1] = __byte_perm(a[1], a[3], 0x6420), o[4 * i + 3] = __byte_perm(a[1], a[3], 0x7531);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const uint32_t c = (w[i] >> (2 * t)) & 0x03030303u;
                if constexpr (LV == QIFT_LEVELS_INT3) {      // the third bit, turned over, to its place: (code ^ 4) = level + 4
                    const int at = int3_high_shift(i, t);
                    const uint32_t b = at >= 2 ? hi[i >> 1] >> (at - 2) : hi[i >> 1] << (2 - at);
                    o[4 * i + t] = c | ((b & 0x04040404u) ^ 0x04040404u);
                } else {
                    o[4 * i + t] = c;
                }
            }
    }
}
template <int LV>
__device__ __forceinline__ int gt_result(int d, int sum_q) {
    if constexpr (LV == QIFT_LEVELS_POT) return d;
    if constexpr (LV == QIFT_LEVELS_MNZ) return 2 * d - 3 * sum_q;
    if constexpr (LV == QIFT_LEVELS_SYM) return d - 2 * sum_q;
    if constexpr (LV == QIFT_LEVELS_INT3) return d - 4 * sum_q;
    return d - 8 * sum_q;
}

template <int LV>
__global__ void __launch_bounds__(kGtThreads, 1)
gated_tc_kernel(const __grid_constant__ CUtensorMap map, const GatedTcParams tp) {
    constexpr int PER = codes_per_word(LV), KPS = PER == 16 ? 2 : 1;   // k-blocks of a 16-word slice
    constexpr int WB = tile_word_bytes(LV), SLOTS = gt_slots(LV), SLOT = gt_slot_bytes(LV);
    const GatedParams& p = tp.g;
    const int ntok = tp.ntok, stages = tp.stages;
    const uint32_t act_bytes = ntok * 128;
    // D = s32, A = u8 (the power-of-two set: s8), B = s8, both K-major, M = 128
    const uint32_t idesc = (2u << 4) | ((LV == QIFT_LEVELS_POT ? 1u : 0u) << 7) | (1u << 10) | (static_cast<uint32_t>(ntok >> 3) << 17) |
                           (static_cast<uint32_t>(kGtRows >> 4) << 24);
    const int sets = ntok <= 32 ? 4 : ntok <= 64 ? 2 : 1;              // accumulators of a matrix, by turns: 2 * sets * ntok <= 256

    extern __shared__ unsigned char smem_raw[];
    unsigned char* act = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    unsigned char* words = act + stages * act_bytes;
    uint64_t* act_full = reinterpret_cast<uint64_t*>(words + 8 * SLOTS * SLOT);
    uint64_t* act_empty = act_full + stages;
    uint64_t* a_full = act_empty + stages;           // [matrix][kGtRing]
    uint64_t* a_empty = a_full + 2 * kGtRing;
    uint64_t* d_full = a_empty + 2 * kGtRing;
    uint64_t* d_empty = d_full + 1;
    int* sum_q = reinterpret_cast<int*>(d_empty + 1);                 // [kGtTokens]
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(sum_q + kGtTokens);
    volatile int* fail = reinterpret_cast<volatile int*>(tmem_slot + 1);

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int pitch = packed_pitch(p.K, LV), slices = pitch / 16, kblocks = slices * KPS;
    const int items = ((p.N + kGtRows - 1) / kGtRows) * tp.blocks;

    pdl_launch_dependents();
    if (tid == 0) {
        for (int s = 0; s < stages; ++s) mbar_init(&act_full[s], 1), mbar_init(&act_empty[s], 2 + kGtEpiWarps);
        for (int s = 0; s < 2 * kGtRing; ++s) mbar_init(&a_full[s], 4), mbar_init(&a_empty[s], 1);
        mbar_init(d_full, 2), mbar_init(d_empty, kGtEpiWarps);
        *fail = 0;
        mbar_fence_init();
        tma_prefetch_desc(&map);
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;

    if (warp == 0) {
        // ------------------------------------------------------------------ activations
        pdl_wait();
        if (lane == 0) {
            int s = 0;
            uint32_t ph = 1;                                           // the first round finds the stages empty
            bool ok = true;
            for (int item = blockIdx.x; item < items && ok; item += gridDim.x) {
                const int m0 = (item % tp.blocks) * ntok;
                for (int kb = 0; kb < kblocks; ++kb) {
                    if (!mbar_wait(&act_empty[s], ph, 82)) {
                        *fail = 1, ok = false;
                        break;
                    }
                    mbar_expect_tx(&act_full[s], act_bytes);
                    tma_load_2d(act + s * act_bytes, &map, kb * 128, m0, &act_full[s]);
                    if (++s == stages) s = 0, ph ^= 1;
                }
            }
        }
    } else if (warp <= 2) {
        // ------------------------------------------------------------------ products of one matrix
        if (lane == 0) {
            const int mat = warp - 1;
            const uint64_t desc0 = make_kmajor_sw128_desc(smem_u32(act));
            const uint32_t d = tmem + mat * sets * ntok, a = tmem + kGtOperands + mat * kGtRing * 32;
            int s = 0, slot = 0, count = 0;
            uint32_t ph = 0, slot_ph = 0;
            bool ok = true;
            for (int item = blockIdx.x; item < items && ok; item += gridDim.x, ++count) {
                if (count > 0 && !mbar_wait(d_empty, (count - 1) & 1, 83)) {
                    *fail = 1;
                    break;
                }
                tc_fence_after();
                for (int kb = 0; kb < kblocks; ++kb) {
                    if (!mbar_wait(&act_full[s], ph, 84) || !mbar_wait(&a_full[mat * kGtRing + slot], slot_ph, 85)) {
                        *fail = 1, ok = false;
                        break;
                    }
                    tc_fence_after();
                    const uint64_t b = desc0 + s * (act_bytes >> 4);
#pragma unroll
                    for (int k4 = 0; k4 < 4; ++k4)
                        tc_mma_i8_ts(d + (k4 & (sets - 1)) * ntok, a + slot * 32 + 8 * k4, b + 2 * k4, idesc, kb > 0 || k4 >= sets);
                    tc_commit(&a_empty[mat * kGtRing + slot]);
                    tc_commit(&act_empty[s]);
                    if (++s == stages) s = 0, ph ^= 1;
                    if (++slot == kGtRing) slot = 0, slot_ph ^= 1;
                }
                if (ok) tc_commit(d_full);
            }
        }
    } else if (warp <= 2 + kGtEpiWarps) {
        // ------------------------------------------------------------------ token sums, epilogue
        const int e = warp - 3, quarter = warp & 3, eg = e >> 2;       // two warps of each lane quarter
        const int per_warp = ntok / kGtEpiWarps;                       // rows whose sums this warp takes: 2 .. 16
        pdl_wait();
        bool ok = true;       // a wait that has run out is not tried again; the warp keeps coming to the barriers of the eight
        int s = 0, count = 0;
        uint32_t ph = 0;
        for (int item = blockIdx.x; item < items; item += gridDim.x, ++count) {
            const int m0 = (item % tp.blocks) * ntok, n0 = (item / tp.blocks) * kGtRows;
            const int rows = min(ntok, p.M - m0);
            if constexpr (LV != QIFT_LEVELS_POT) {
                int sum[4] = {};
                for (int kb = 0; kb < kblocks; ++kb) {
                    if (ok && !mbar_wait(&act_full[s], ph, 86)) ok = false, *fail = 1;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int r = 4 * j + (lane >> 3);             // eight lanes read a row's 128 bytes, in whatever order they stand
                        if (ok && r < per_warp) {
                            const uint4 v = lds128(smem_u32(act) + s * act_bytes + (e * per_warp + r) * 128 + (lane & 7) * 16);
                            sum[j] = __dp4a(static_cast<int>(v.x), 0x01010101, __dp4a(static_cast<int>(v.y), 0x01010101, sum[j]));
                            sum[j] = __dp4a(static_cast<int>(v.z), 0x01010101, __dp4a(static_cast<int>(v.w), 0x01010101, sum[j]));
                        }
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&act_empty[s]);
                    if (++s == stages) s = 0, ph ^= 1;
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
#pragma unroll
                    for (int o = 4; o > 0; o >>= 1) sum[j] += __shfl_xor_sync(0xffffffffu, sum[j], o);
                    if ((lane & 7) == 0 && 4 * j + (lane >> 3) < per_warp) sum_q[e * per_warp + 4 * j + (lane >> 3)] = sum[j];
                }
                asm volatile("bar.sync 1, %0;" ::"n"(32 * kGtEpiWarps) : "memory");
            } else {
                for (int kb = 0; kb < kblocks; ++kb) {
                    if (ok && !mbar_wait(&act_full[s], ph, 86)) ok = false, *fail = 1;
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&act_empty[s]);
                    if (++s == stages) s = 0, ph ^= 1;
                }
            }
            if (ok && !mbar_wait(d_full, count & 1, 87)) ok = false, *fail = 1;
            if (ok) {
                tc_fence_after();
                const int n = n0 + quarter * 32 + lane;
                float sg = 0.0f, su = 0.0f;
                if (n < p.N) sg = __ldg(p.w[0].s_n + n), su = __ldg(p.w[1].s_n + n);
                const uint32_t lanes = tmem + (static_cast<uint32_t>(quarter * 32) << 16);
                for (int c = 16 * eg; c < rows; c += 32) {
                    int v[2][16];
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        uint32_t x[16];
                        tc_ld16(lanes + i * sets * ntok + c, x);
                        tc_wait_ld();
#pragma unroll
                        for (int j = 0; j < 16; ++j) v[i][j] = static_cast<int>(x[j]);
                        for (int k = 1; k < sets; ++k) {
                            tc_ld16(lanes + (i * sets + k) * ntok + c, x);
                            tc_wait_ld();
#pragma unroll
                            for (int j = 0; j < 16; ++j) v[i][j] += static_cast<int>(x[j]);
                        }
                    }
                    if (n < p.N) {
#pragma unroll
                        for (int j = 0; j < 16; ++j) {
                            if (c + j < rows) {
                                const int m = m0 + c + j, sq = LV == QIFT_LEVELS_POT ? 0 : sum_q[c + j];
                                gated_store(p, static_cast<size_t>(m) * p.N + n, gt_result<LV>(v[0][j], sq), gt_result<LV>(v[1][j], sq),
                                            __ldg(p.s_a + m), sg, su);
                            }
                        }
                    }
                }
                tc_fence_before();
            }
            if constexpr (LV != QIFT_LEVELS_POT)
                asm volatile("bar.sync 1, %0;" ::"n"(32 * kGtEpiWarps) : "memory");   // the sums have been read
            __syncwarp();
            if (lane == 0) mbar_arrive(d_empty);
        }
    } else {
        // ------------------------------------------------------------------ expanders
        const int e = warp - 11, q = warp & 3, mat = e >> 2;           // q: the lane quarter this warp's tcgen05.st can reach
        const uint32_t ring = smem_u32(words + e * SLOTS * SLOT);
        const unsigned char* base = reinterpret_cast<const unsigned char*>(p.w[mat].packed);
        const size_t rb_bytes = static_cast<size_t>(pitch) * WB;
        const int row_blocks = (p.N + 15) / 16;
        int f_item = blockIdx.x, f_slice = 0;
        auto fetch = [&](int slot) {                                   // the next slice -> ring slot; always commits a group
            if (f_item < items) {
                const int rb0 = (f_item / tp.blocks) * 8 + 2 * q;
                const unsigned char* src = base + rb0 * rb_bytes + static_cast<size_t>(f_slice) * (16 * WB) + lane * 16;
#pragma unroll
                for (int h = 0; h < 4; ++h)                            // row h * 8 + lane / 4: 16-byte pieces exclusive-ored by (row >> 1) & 3
                    if (rb0 + (h >> 1) < row_blocks)
                        cp_async16(ring + slot * SLOT + (h * 8 + (lane >> 2)) * 64 + (((lane & 3) ^ ((lane >> 3) & 3)) << 4),
                                   src + (h >> 1) * rb_bytes + (h & 1) * 512);
                if constexpr (LV == QIFT_LEVELS_INT3) {
#pragma unroll
                    for (int h = 0; h < 2; ++h)                        // third bits of eight rows and the eight behind them: as they stand
                        if (rb0 + h < row_blocks) cp_async16(ring + slot * SLOT + 2048 + h * 512 + lane * 16, src + h * rb_bytes + 1024);
                }
                if (++f_slice == slices) f_slice = 0, f_item += gridDim.x;
            }
            cp_async_commit();
        };
        for (int s = 0; s < SLOTS; ++s) fetch(s);
        int slot = 0, a_slot = 0;
        uint32_t a_ph = 1;
        bool ok = true;
        for (int item = blockIdx.x; item < items && ok; item += gridDim.x) {
            const bool row_valid = (item / tp.blocks) * 8 + 2 * q + (lane >> 4) < row_blocks;
            for (int sl = 0; sl < slices && ok; ++sl) {
                cp_async_wait<SLOTS - 1>();
                __syncwarp();
                uint32_t w[16], hi[8];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint4 v = make_uint4(0, 0, 0, 0);
                    if (row_valid) v = lds128(ring + slot * SLOT + lane * 64 + ((i ^ ((lane >> 1) & 3)) << 4));
                    w[4 * i] = v.x, w[4 * i + 1] = v.y, w[4 * i + 2] = v.z, w[4 * i + 3] = v.w;
                    if constexpr (LV == QIFT_LEVELS_INT3) {
                        uint2 u = make_uint2(0, 0);
                        if (row_valid) u = lds64(ring + slot * SLOT + 2048 + (lane >> 4) * 512 + ((lane & 7) * 4 + i) * 16 + ((lane >> 3) & 1) * 8);
                        hi[2 * i] = u.x, hi[2 * i + 1] = u.y;
                    }
                }
                __syncwarp();                                          // every lane has read the slot before it is filled again
                fetch(slot);
                if (++slot == SLOTS) slot = 0;
#pragma unroll
                for (int j = 0; j < KPS; ++j) {
                    if (!mbar_wait(&a_empty[mat * kGtRing + a_slot], a_ph, 88)) {
                        *fail = 1, ok = false;
                        break;
                    }
                    tc_fence_after();
                    uint32_t o[32];
                    gt_operands<LV>(w + (PER == 16 ? 8 * j : 0), hi + 4 * j, o);
                    tc_st32(tmem + (static_cast<uint32_t>(q * 32) << 16) + kGtOperands + (mat * kGtRing + a_slot) * 32, o);
                    tc_wait_st();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&a_full[mat * kGtRing + a_slot]);
                    if (++a_slot == kGtRing) a_slot = 0, a_ph ^= 1;
                }
            }
        }
        cp_async_wait<0>();
    }

    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    }
}

}  // namespace qift
