// The gated half of a feed-forward block: two products of one quantized activation, the activation function and the product of both,
//
//     h[m,n] = act(g) u,   g = s_gate[n] s_a[m] sum_k level(gate[n,k]) q_a[m,k],   u likewise with the other weights,
//
// so that neither product is written: only h leaves the kernel.  The sums are exact (INT32), scaled as in the linear calls (two
// rounded multiplies), everything after that is fp32, rounded once where h is bf16.
//
// The kernels, by rows (which of them a call takes, and both sides measured: beside the host's rules):
//   * gated_stream_kernel: up to 16 rows, bound by the stream of codes;
//   * gated_tc_kernel: up to 1024 rows, the codes as the tcgen05 operand in tensor memory;
//   * gemm_i8_pair_kernel, gated: beyond, or on levels that an earlier call has decoded: int8 levels, a tile on two SMs;
//   * gated_generic_kernel, here: one warp per channel, dp4a, any M and K: rows that a tensor copy cannot take (K not a multiple of 16,
//     more than 16 rows) and sums past what the others hold.  48 rows, 4096 -> 14336: 452 us, where the tcgen05 kernel takes 12.8.
#pragma once

#include "common.cuh"
#include "decode.cuh"
#include "kv4_tree.cuh"

namespace qift {

// act(g): g sigmoid(z) with z = g (SiLU) or z = 2 sqrt(2 / pi) (g + 0.044715 g^3) (GELU in its tanh form: (1 + tanh t) / 2 = sigmoid(2t)), as
// z = g (a + b g^2) for both: no branch per output.  With e = exp(-|z|), which does not overflow, the values are g / (1 + e) and g e / (1 + e):
// those of far negative gates fade out with e, down to 2^-149.  The denominator lies in 1 .. 2, so that the quotient may be a product with
// its reciprocal, within 2 units in the last place (a quotient that minds the range of its denominator: 512 rows, 4096 -> 14336, 58.6 us against 57.8).
struct GateFunction {
    float a, b;
    __host__ __device__ explicit GateFunction(int act) : a(act == QIFT_ACT_SILU ? 1.0f : 1.5957691216057308f), b(act == QIFT_ACT_SILU ? 0.0f : 0.0713548162726f) {}
    __device__ __forceinline__ float operator()(float g) const {
        const float z = g * fmaf(b, fminf(g * g, 1e30f), a);
        const float e = expf(-fabsf(z));
        float r;
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + e));     // within one unit in the last place
        return (z < 0.0f ? g * e : g) * r;
    }
};
__device__ __forceinline__ float gated_value(int acc_g, int acc_u, float s_a, float s_gate, float s_up, GateFunction act) {
    return act(scale_epilogue(acc_g, s_a, s_gate)) * scale_epilogue(acc_u, s_a, s_up);
}

struct GatedMatrix {
    const uint32_t* packed;
    const float* s_n;       // [N]
    int32_t* acc_debug;     // [M][N] or null
};
struct GatedProbe {         // self-test alone (qift_selftest_gated_wait): a warp whose waits, after the first few, are for what nobody signals
    int warp, waits;
    uint32_t trips;         // bound of every wait
};
struct GatedParams {
    GatedMatrix w[2];       // gate, up
    const int8_t* q_a;      // [M][K]
    const float* s_a;       // [M]
    void* H;                // [M][N]
    int M, N, K, h_bf16, act;
    GatedProbe probe;
};

// The bounded waits of a thread.  Lanes have to agree on whether a wait has run out before an instruction of the whole warp depends on it.
template <bool PROBE>
struct GatedWait {
    const GatedProbe& probe;
    uint64_t* never;        // PROBE: a barrier that nobody arrives at
    int left;
    __device__ __forceinline__ GatedWait(const GatedProbe& p, uint64_t* nobody, int warp)
        : probe(p), never(nobody), left(warp == p.warp ? p.waits : 0x7fffffff) {}
    __device__ __forceinline__ bool operator()(uint64_t* bar, uint32_t parity, unsigned int site) {
        if constexpr (PROBE) {
            const bool held = left-- <= 0;
            return mbar_wait_near(held ? never : bar, held ? 0u : parity, site, probe.trips);
        } else {
            return mbar_wait_near(bar, parity, site);
        }
    }
};

__device__ __forceinline__ void gated_store(const GatedParams& p, size_t at, int acc_g, int acc_u, float s_a, float s_gate, float s_up) {
    if (p.w[0].acc_debug) p.w[0].acc_debug[at] = acc_g;
    if (p.w[1].acc_debug) p.w[1].acc_debug[at] = acc_u;
    const float h = gated_value(acc_g, acc_u, s_a, s_gate, s_up, GateFunction(p.act));
    if (p.h_bf16) static_cast<uint16_t*>(p.H)[at] = f32_to_bf16_bits(h);
    else static_cast<float*>(p.H)[at] = h;
}

constexpr int kGatedTokens = 4;   // token rows of a warp at a time

template <int LV>
__global__ void __launch_bounds__(kGenericWarps * 32)
gated_generic_kernel(const GatedParams p) {
    constexpr int PER = codes_per_word(LV);
    constexpr int NPL = PER / 4;
    constexpr int BITS = 32 / PER;
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31;
    const int n = blockIdx.x * kGenericWarps + (threadIdx.x >> 5);
    if (n >= p.N) return;
    const int words = p.K / PER;
    const int pitch = round_up16(words);
    const uint32_t* q32 = reinterpret_cast<const uint32_t*>(p.q_a);
    const size_t qpitch = p.K / 4;
    for (long long m0 = blockIdx.y * kGatedTokens; m0 < p.M; m0 += gridDim.y * kGatedTokens) {
        int S[2][kGatedTokens] = {}, Sb[2][kGatedTokens] = {}, Sq[kGatedTokens] = {};
        for (int j = lane; j < words; j += 32) {
            uint32_t w[2], wh[2] = {0, 0};
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                if constexpr (LV == QIFT_LEVELS_INT3) {
                    w[i] = p.w[i].packed[int3_low_address(n, j, pitch)];
                    wh[i] = p.w[i].packed[int3_high_address(n, j, pitch)];
                } else {
                    w[i] = p.w[i].packed[packed_word_address(n, j, pitch)];
                }
            }
#pragma unroll
            for (int t = 0; t < NPL; ++t) {
                uint32_t a[2], hb[2] = {0, 0};
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    if constexpr (LV == QIFT_LEVELS_INT4) {
                        a[i] = ((w[i] >> (BITS * t)) & 0x0f0f0f0fu) ^ 0x08080808u;
                    } else {
                        a[i] = (w[i] >> (BITS * t)) & 0x03030303u;
                        hb[i] = LV == QIFT_LEVELS_INT3 ? (wh[i] >> int3_high_shift(j, t)) & 0x01010101u : (a[i] >> 1) & 0x01010101u;
                    }
                }
#pragma unroll
                for (int mm = 0; mm < kGatedTokens; ++mm) {
                    if (m0 + mm < p.M) {
                        const uint32_t qv = q32[(m0 + mm) * qpitch + static_cast<size_t>(j) * NPL + t];
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            S[i][mm] = dp4a_us(a[i], qv, S[i][mm]);
                            if constexpr (LV == QIFT_LEVELS_POT || LV == QIFT_LEVELS_INT3) Sb[i][mm] = dp4a_us(hb[i], qv, Sb[i][mm]);
                        }
                        Sq[mm] = dp4a_us(0x01010101u, qv, Sq[mm]);
                    }
                }
            }
        }
#pragma unroll
        for (int mm = 0; mm < kGatedTokens; ++mm) {
            int acc[2];
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) Sq[mm] += __shfl_xor_sync(0xffffffffu, Sq[mm], o);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) {
                    S[i][mm] += __shfl_xor_sync(0xffffffffu, S[i][mm], o);
                    Sb[i][mm] += __shfl_xor_sync(0xffffffffu, Sb[i][mm], o);
                }
                acc[i] = combine_generic<LV>(S[i][mm], Sb[i][mm], Sq[mm]);
            }
            const long long m = m0 + mm;
            if (lane == 0 && m < p.M)
                gated_store(p, static_cast<size_t>(m) * p.N + n, acc[0], acc[1], p.s_a[m], p.w[0].s_n[n], p.w[1].s_n[n]);
        }
    }
}

}  // namespace qift
