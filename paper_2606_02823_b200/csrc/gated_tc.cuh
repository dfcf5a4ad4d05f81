// The gated products of some tens to some hundreds of token rows on the tcgen05 tensor cores, with the packed codes as the operand in
// tensor memory (as in decode_tc.cuh: they never exist as int8 in shared memory).
//
// An item is 128 channels of both matrices times one block of up to 128 token rows (N of the instruction, any multiple of 16: 48 rows
// cost what 48 cost).  The two matrices are two independent streams over one sequence of activation blocks:
//
//   warp 0        fills a ring of steps (256 codes deep) with tensor copies: the packed words of both matrices (three dimensions: a row's 64
//                 bytes of a slice, swizzled; rows; blocks of sixteen rows) and the q_a rows of the token block, two 128-byte k-blocks
//   warps 1, 2    issue the products D[matrix][128 channels x tokens] of a matrix each, eight a step (here and above one elected thread of a
//                 warp does it all: with a vote of the lanes after each wait 48 rows took 14.2 us)
//   warps 4-19    expanders, two per matrix and lane quarter, for the even and the odd steps: the packed words of their 32 channels, one to
//                 four operations per operand word, tcgen05.st into their slot of the matrix's operands; then the epilogue, four per
//                 lane quarter on 8-token pieces by turns: both accumulators, h, stores of 32 channels
//
// Activations come as they are, and there is no launch before this one: the operand bytes are the levels themselves times a power of two, made
// by moving a code to the top of its byte -- (code << 6) ^ 0xa0 = 32 (2 code - 3) as a signed byte, (code << 6) ^ 0x80 = 64 (code - 2), the
// four- and three-bit codes 16 and 32 times themselves -- or, for the power-of-two set, by table lookup.  No correction by token sums (which
// took as long as the products) and no place values; an arithmetic shift takes the factor off.
// Token blocks of one channel tile are neighbours in the item list, so that its codes come from L2 for all but the first.
//
// Bounds: a 128 x N x 32 product takes N / 2 cycles of the tensor cores, 16 at least; operands enter tensor memory at 128 bytes a cycle
// (1 MB an item of K = 4096: 4.3 us); their logic is 56 operations per k-block and warp.  What sets the pace is handing over: with logic,
// tensor memory stores and seven of eight products left out, 48 rows, 4096 -> 14336, still took 13.5 of 15.6 us (launches one after the
// other).  So a step passes
// through as few barriers as there are roles: an expander waits twice for its 256 codes of every second step, and its partner's
// step is expanded meanwhile (each step shared between both: 8 to 15 % longer over 8192 codes; a hand-over per 128 codes: 15 to 25 %).  A
// thread that a whole warp has elected issues a product in 16 cycles; one that a comparison of lanes has picked takes 60 (the compiler
// cannot know it is alone, and tries every lane's operands), which alone set the pace at first: 23 us for 48 rows.  Waits carry no time
// hint (with one they are a loop around a sleep) and are bounded by their trips.  4096 -> 14336 in two bits: 9 rows 11.0 us, 48 rows
// 12.8, 128 rows 17.8, 512 rows 57.5.
#pragma once

#include "common.cuh"
#include "decode_tc.cuh"
#include "gated.cuh"
#include "kv4_tree_tc.cuh"
#include "prefill.cuh"

namespace qift {

constexpr int kGtRows = 128;                 // channels of an item
constexpr int kGtTokens = 128;               // token rows of an item, at most
constexpr int kGtExpanders = 16, kGtExpander0 = 4;                   // warps, the first of them
constexpr int kGtThreads = 32 * (kGtExpander0 + kGtExpanders);
constexpr int kGtRing = 2;                   // steps of operands in tensor memory, per matrix
constexpr int kGtOperands = 256;             // first operand column
constexpr int kGtSmem = 226 * 1024;
constexpr int kGtMaxK = 1 << 21;              // K < this: operands up to 128 times activations up to 8 add up within 32 bits

__host__ __device__ constexpr int gt_slices(int lv) { return lv == QIFT_LEVELS_INT4 ? 2 : 1; }            // 16-word slices of a step
__host__ __device__ constexpr int gt_slice_rows(int lv) { return lv == QIFT_LEVELS_INT3 ? 24 : 16; }      // 64-byte rows of a slice and row block
__host__ __device__ constexpr int gt_word_bytes(int lv) { return 8 * 64 * gt_slices(lv) * gt_slice_rows(lv); }   // of a step and matrix
__host__ __device__ inline int gt_stages(int lv, int ntok) {
    const int n = (kGtSmem - 3 * 1024) / (2 * gt_word_bytes(lv) + ntok * 256);
    return n < 8 ? n : 8;
}

struct GatedTcParams {
    GatedParams g;
    int ntok, blocks;        // token rows of a block (a multiple of 16), blocks
    int stages;              // steps in shared memory
};
struct alignas(64) GatedTcMaps {
    CUtensorMap act;         // q_a [M, K], box = 128 bytes x ntok rows
    CUtensorMap words[2];    // [row blocks][rows of a block's slices][64 bytes], box = 8 x a step's rows x 64
};

// Operand bytes of one k-block (128 codes) of a channel, in k order: level * 2^gt_shift.  hi: the words of the third bits (INT3).
template <int LV>
__host__ __device__ constexpr int gt_shift() {
    return LV == QIFT_LEVELS_MNZ || LV == QIFT_LEVELS_INT3 ? 5 : LV == QIFT_LEVELS_SYM ? 6 : LV == QIFT_LEVELS_INT4 ? 4 : 0;
}
// (a & b) ^ c with all three in registers: one instruction (with two immediates it would be two, and the operands' logic is what the
// expanders' time goes into).
__device__ __forceinline__ uint32_t and_xor(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t d;
    asm("lop3.b32 %0, %1, %2, %3, 0x6a;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}
// (a & b) | (c & ~b)
__device__ __forceinline__ uint32_t select_bits(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t d;
    asm("lop3.b32 %0, %1, %2, %3, 0xe2;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}
__device__ __forceinline__ uint32_t in_register(uint32_t v) {
    asm volatile("" : "+r"(v));
    return v;
}
template <int LV>
__device__ __forceinline__ void gt_operands(const uint32_t* w, const uint32_t* hi, uint32_t (&o)[32]) {
    if constexpr (LV == QIFT_LEVELS_INT4) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            o[2 * i] = (w[i] << 4) & 0xf0f0f0f0u;
            o[2 * i + 1] = w[i] & 0xf0f0f0f0u;
        }
    } else if constexpr (LV == QIFT_LEVELS_POT) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            uint32_t a[4];
            pot_lut_operands(w[i], a);       // codes {0,8,1,9}, {4,12,5,13}, {2,10,3,11}, {6,14,7,15} of the word
            o[4 * i] = __byte_perm(a[0], a[2], 0x6420), o[4 * i + 2] = __byte_perm(a[0], a[2], 0x7531);
            o[4 * i + 1] = __byte_perm(a[1], a[3], 0x6420), o[4 * i + 3] = __byte_perm(a[1], a[3], 0x7531);
        }
    } else if constexpr (LV == QIFT_LEVELS_INT3) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const uint32_t c = t < 3 ? w[i] << (5 - 2 * t) : w[i] >> 1, b = hi[i >> 1] << (7 - int3_high_shift(i, t));
                o[4 * i + t] = select_bits(b, 0x80808080u, c) & 0xe0e0e0e0u;
            }
    } else {
        const uint32_t keep = in_register(0xc0c0c0c0u), turn = in_register(LV == QIFT_LEVELS_MNZ ? 0xa0a0a0a0u : 0x80808080u);
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int t = 0; t < 4; ++t) o[4 * i + t] = and_xor(w[i] << (6 - 2 * t), keep, turn);
    }
}
__device__ __forceinline__ void gt_ld8(uint32_t taddr, uint32_t (&v)[8]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7])
                 : "r"(taddr)
                 : "memory");
}
__device__ __forceinline__ void tma_load_3d(void* dst, const CUtensorMap* map, int x, int y, int z, uint64_t* bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(smem_u32(dst)),
                 "l"(map), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z)
                 : "memory");
}
template <int LV, bool PROBE = false>
__global__ void __launch_bounds__(kGtThreads, 1)
gated_tc_kernel(const __grid_constant__ GatedTcMaps maps, const __grid_constant__ GatedTcParams tp) {
    constexpr int SPS = gt_slices(LV), SROWS = gt_slice_rows(LV), RB = 64 * SPS * SROWS;   // bytes of a row block in a step
    constexpr uint32_t WORDS = gt_word_bytes(LV);
    const GatedParams& p = tp.g;
    const int ntok = tp.ntok, stages = tp.stages;
    const uint32_t act_bytes = ntok * 128, stage_bytes = 2 * WORDS + 2 * act_bytes;        // a stage: both matrices' words, two k-blocks
    // D = s32, A = B = s8, both K-major, M = 128
    const uint32_t idesc = (2u << 4) | (1u << 7) | (1u << 10) | (static_cast<uint32_t>(ntok >> 3) << 17) |
                           (static_cast<uint32_t>(kGtRows >> 4) << 24);

    extern __shared__ unsigned char smem_raw[];
    unsigned char* staged = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint64_t* full = reinterpret_cast<uint64_t*>(staged + stages * stage_bytes);
    uint64_t* empty = full + stages;
    uint64_t* a_full = empty + stages;               // [matrix][kGtRing]
    uint64_t* a_empty = a_full + 2 * kGtRing;
    uint64_t* d_full = a_empty + 2 * kGtRing;
    uint64_t* d_empty = d_full + 1;
    uint64_t* never = d_empty + 1;                                    // (self-test)
    float* scale = reinterpret_cast<float*>(never + 1);               // [kGtTokens] of the tokens
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(scale + kGtTokens);

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int steps = (packed_pitch(p.K, LV) / 16 + SPS - 1) / SPS;
    const int items = ((p.N + kGtRows - 1) / kGtRows) * tp.blocks;
    // CTAs begin at different steps (the sums are integers, their order is free): all of them read the same activations, and a line
    // that a hundred of them ask for at once takes as long as a hundred lines
    const int first_step = blockIdx.x % steps;

    pdl_launch_dependents();
    if (warp == 0 && lane == 0) {
        for (int s = 0; s < stages; ++s) mbar_init(&full[s], 1), mbar_init(&empty[s], 2 + kGtExpanders / 2);
        for (int s = 0; s < 2 * kGtRing; ++s) mbar_init(&a_full[s], 4), mbar_init(&a_empty[s], 1);
        mbar_init(d_full, 2), mbar_init(d_empty, kGtExpanders);
        if constexpr (PROBE) mbar_init(never, 1);
        mbar_fence_init();
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    GatedWait<PROBE> wait(p.probe, never, warp);

    if (warp == 0) {
        // ------------------------------------------------------------------ words and activations
        auto words = [&](int s, int rb, int step) {
            mbar_expect_tx(&full[s], stage_bytes);
            tma_load_3d(staged + s * stage_bytes, &maps.words[0], 0, step * (SPS * SROWS), rb, &full[s]);
            tma_load_3d(staged + s * stage_bytes + WORDS, &maps.words[1], 0, step * (SPS * SROWS), rb, &full[s]);
        };
        auto activations = [&](int s, int m0, int step) {
            unsigned char* to = staged + s * stage_bytes + 2 * WORDS;
            tma_load_2d(to, &maps.act, step * 256, m0, &full[s]);
            tma_load_2d(to + act_bytes, &maps.act, step * 256 + 128, m0, &full[s]);
        };
        // the words depend on no kernel before this one: the first stages' are asked for before the wait for it
        const int early = min(stages, steps);
        if (elect_one()) {
            for (int i = 0, step = first_step; i < early; ++i, step = step + 1 == steps ? 0 : step + 1) words(i, (blockIdx.x / tp.blocks) * 8, step);
            pdl_wait();
            int s = 0, k = 0;
            uint32_t ph = 1;                                           // the first round finds the stages empty
            bool ok = true;
            for (int item = blockIdx.x; item < items && ok; item += gridDim.x) {
                const int rb = (item / tp.blocks) * 8, m0 = (item % tp.blocks) * ntok;
                for (int i = 0, step = first_step; i < steps; ++i, ++k) {
                    if (!(ok = wait(&empty[s], ph, 82))) break;
                    if (k >= early) words(s, rb, step);
                    activations(s, m0, step);
                    if (++s == stages) s = 0, ph ^= 1;
                    if (++step == steps) step = 0;
                }
            }
            // what has been asked for arrives before the CTA ends, also where those who should wait for it have given up (and given up itself, this
            // thread may have asked for words alone, whose stages never fill: a millisecond each)
            const int asked = max(k, early);
            for (int i = 0; i < min(asked, stages); ++i) mbar_wait(&full[i], ((asked - 1 - i) / stages) & 1, 82, ok ? kWaitLimitNs : 1000000ull);
        }
        __syncwarp();
    } else if (warp <= 2) {
        // ------------------------------------------------------------------ products of a matrix
        const int mat = warp - 1;
        const uint64_t desc0 = make_kmajor_sw128_desc(smem_u32(staged) + 2 * WORDS);
        const uint32_t d = tmem + mat * ntok, a = tmem + kGtOperands + mat * kGtRing * 64;
        if (elect_one()) {
            int s = 0, count = 0;
            uint32_t ph = 0, turn = 0, turn_ph = 0;                    // turn: the step's slot of operands, the parity of its running number
            uint32_t issued = 0;                                       // steps
            bool ok = true;
            for (int item = blockIdx.x; item < items && ok; item += gridDim.x, ++count) {
                if (count > 0) ok = wait(d_empty, (count - 1) & 1, 83);
                for (int i = 0; i < steps; ++i) {
                    if (ok) ok = wait(&full[s], ph, 84);
                    if (ok) ok = wait(&a_full[mat * kGtRing + turn], turn_ph, 85);
                    if (!ok) break;
                    tc_fence_after();
                    const uint64_t b = desc0 + s * (stage_bytes >> 4);
                    const uint32_t at = a + turn * 64;
#pragma unroll
                    for (int k = 0; k < 8; ++k) tc_mma_i8_ts(d, at + 8 * k, b + (k >> 2) * (act_bytes >> 4) + 2 * (k & 3), idesc, i | k);
                    tc_commit(&a_empty[mat * kGtRing + turn]);
                    tc_commit(&empty[s]);
                    if (i + 1 == steps) tc_commit(d_full);
                    ++issued;
                    if (++s == stages) s = 0, ph ^= 1;
                    if ((turn ^= 1) == 0) turn_ph ^= 1;
                }
            }
            // products under way end before the CTA does, also where nobody waits for their sums any more
            if (issued) mbar_wait_near(&a_empty[mat * kGtRing + ((issued - 1) & 1)], ((issued - 1) >> 1) & 1, 86);
        }
        __syncwarp();
    } else if (warp >= kGtExpander0) {
        // ------------------------------------------------------------------ operands, then the epilogue
        const int quarter = warp & 3;                                  // the lanes of tensor memory that this warp can reach
        const int e = warp - kGtExpander0, mat = (e >> 2) & 1, odd = e >> 3;    // its matrix; the even or the odd steps
        // its words of a k-block: two 16-byte pieces of a row (INT4: all four of a slice); pieces are exclusive-ored by (row >> 1) & 3
        constexpr int PIECES = SPS == 2 ? 4 : 2;
        const uint32_t rows64 = smem_u32(staged) + mat * WORDS + (2 * quarter + (lane >> 4)) * RB;
        const uint32_t get = rows64 + (lane & 15) * 64;
        const uint32_t put = tmem + (static_cast<uint32_t>(quarter * 32) << 16) + kGtOperands + (mat * kGtRing + odd) * 64;
        const uint32_t get_hi = rows64 + 1024 + (lane & 7) * 64 + ((lane >> 3) & 1) * 8;   // INT3: rows 16 .. 23: {third bits of row r, of row r + 8}
        uint32_t at[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) at[j] = (j ^ ((lane >> 1) & 3)) << 4;
        uint64_t* const mine_empty = &a_empty[mat * kGtRing + odd];
        uint64_t* const mine_full = &a_full[mat * kGtRing + odd];
        const GateFunction act(p.act);
        pdl_wait();
        // A wait that has run out is not tried again: the warp keeps coming to the barriers of the sixteen and hands nothing over any more.  Without its
        // operands the products of the item never end, so that no warp stores any of it, and without its word that the sums have been read
        // there is no next item.
        bool ok = true;
        int s = 0, count = 0;
        uint32_t ph = 0, turn = 0, a_ph = 1;                           // turn: the running step's parity
        for (int item = blockIdx.x; item < items; item += gridDim.x, ++count) {
            const int m0 = (item % tp.blocks) * ntok, n0 = (item / tp.blocks) * kGtRows;
            const int rows = min(ntok, p.M - m0), n = n0 + quarter * 32 + lane;
            float sg = 0.0f, su = 0.0f;                                // asked for long before they are needed
            if (n < p.N) sg = __ldg(p.w[0].s_n + n), su = __ldg(p.w[1].s_n + n);
            const int r = 32 * e + lane;
            if (r < ntok) scale[r] = r < rows ? p.s_a[m0 + r] : 0.0f;
            for (int i = 0; i < steps; ++i, turn ^= 1) {
                if (ok && turn == odd) {
                    ok = wait(&full[s], ph, 87);
                    uint32_t w[2][4 * PIECES], hi[2][4] = {};
                    const uint32_t from = get + s * stage_bytes;
#pragma unroll
                    for (int half = 0; half < 2; ++half)
#pragma unroll
                        for (int j = 0; j < PIECES; ++j) {
                            const uint32_t piece = at[SPS == 2 ? j : 2 * half + j];
                            const uint4 v = lds128(from + (SPS == 2 ? half * 1024 : 0) + piece);
                            w[half][4 * j] = v.x, w[half][4 * j + 1] = v.y, w[half][4 * j + 2] = v.z, w[half][4 * j + 3] = v.w;
                            if constexpr (LV == QIFT_LEVELS_INT3) {
                                const uint2 u = lds64(get_hi + s * stage_bytes + piece);
                                hi[half][2 * j] = u.x, hi[half][2 * j + 1] = u.y;
                            }
                        }
                    ok = __all_sync(0xffffffffu, ok);
                    if (ok && lane == 0) mbar_arrive(&empty[s]);
                    uint32_t o[32];
                    gt_operands<LV>(w[0], hi[0], o);
                    if (ok) ok = wait(mine_empty, a_ph, 88);
                    tc_fence_after();                                  // (operands without a slot spoil sums that nobody will be given)
                    tc_st32(put, o);
                    gt_operands<LV>(w[1], hi[1], o);
                    tc_st32(put + 32, o);
                    tc_wait_st();
                    tc_fence_before();
                    ok = __all_sync(0xffffffffu, ok);
                    if (ok && lane == 0) mbar_arrive(mine_full);
                    a_ph ^= 1;
                }
                if (++s == stages) s = 0, ph ^= 1;
            }
            asm volatile("bar.sync 1, %0;" ::"n"(32 * kGtExpanders) : "memory");      // the scales are there
            if (ok) ok = __all_sync(0xffffffffu, wait(d_full, count & 1, 89));
            if (ok) {
                tc_fence_after();
                const uint32_t lanes = tmem + (static_cast<uint32_t>(quarter * 32) << 16);
                // a loop of eight tokens a trip, not more: code that runs once has to be fetched first, which took longer than running it
#pragma unroll 1
                for (int c = 8 * (e >> 2); c < rows; c += 8 * (kGtExpanders / 4)) {
                    int v[2][8];
                    {
                        uint32_t x[8], y[8];
                        gt_ld8(lanes + c, x);
                        gt_ld8(lanes + ntok + c, y);
                        tc_wait_ld();
#pragma unroll
                        for (int j = 0; j < 8; ++j) v[0][j] = static_cast<int>(x[j]), v[1][j] = static_cast<int>(y[j]);
                    }
                    float h[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        v[0][j] >>= gt_shift<LV>(), v[1][j] >>= gt_shift<LV>();
                        h[j] = gated_value(v[0][j], v[1][j], scale[c + j], sg, su, act);
                    }
                    if (n < p.N) {
                        const size_t at = static_cast<size_t>(m0 + c) * p.N + n;
                        if (p.h_bf16) {
                            uint16_t* to = static_cast<uint16_t*>(p.H) + at;
#pragma unroll
                            for (int j = 0; j < 8; ++j, to += p.N)
                                if (c + j < rows) *to = f32_to_bf16_bits(h[j]);
                        } else {
                            float* to = static_cast<float*>(p.H) + at;
#pragma unroll
                            for (int j = 0; j < 8; ++j, to += p.N)
                                if (c + j < rows) *to = h[j];
                        }
#pragma unroll
                        for (int i = 0; i < 2; ++i)
                            if (p.w[i].acc_debug) {
#pragma unroll
                                for (int j = 0; j < 8; ++j)
                                    if (c + j < rows) p.w[i].acc_debug[at + static_cast<size_t>(j) * p.N] = v[i][j];
                            }
                    }
                }
                tc_fence_before();
            }
            asm volatile("bar.sync 1, %0;" ::"n"(32 * kGtExpanders) : "memory");       // and have been read
            if (ok && lane == 0) mbar_arrive(d_empty);
        }
    }

    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    }
}

}  // namespace qift
