// Low-rank adapters of many requests beside a shared projection: out[m] = y[m] + scaling_a * B_a (A_a x[m]).
#pragma once

#include "common.cuh"

namespace qift {

struct LoraParams {
    const void* x;            // [M][K], rows x_stride elements apart
    const uint16_t* A;        // bf16 [adapters][rank][K]
    const uint16_t* B;        // bf16 [adapters][N][rank]
    const float* scaling;     // [adapters]
    const int32_t* row_start; // [R + 1]
    const int32_t* adapter;   // [R]
    const void* y;            // [M][N] or nullptr (zeros)
    void* out;                // [M][N]
    float* t;                 // workspace: fp32 [M][rank]
    int M, N, K, rank, adapters, R;
};

__device__ __forceinline__ float bf16_bits_to_f32(uint16_t b) { return __uint_as_float(static_cast<uint32_t>(b) << 16); }
template <bool BF16>
__device__ __forceinline__ float lora_load(const void* p, size_t i) {
    if constexpr (BF16) return bf16_bits_to_f32(static_cast<const uint16_t*>(p)[i]);
    else return static_cast<const float*>(p)[i];
}

// The request of a row and its adapter (-1: none, -2: the row belongs to no request).
__device__ __forceinline__ int lora_adapter_of(const LoraParams& p, int m) {
    for (int r = 0; r < p.R; ++r)
        if (m >= p.row_start[r] && m < p.row_start[r + 1]) return p.adapter[r] >= 0 && p.adapter[r] < p.adapters ? p.adapter[r] : -1;
    return -2;
}

template <bool BF16>
__global__ void __launch_bounds__(256)
lora_down_kernel(const LoraParams p) {
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31, m = blockIdx.x;
    const int a = lora_adapter_of(p, m);
    if (a < 0) return;
    for (int j = threadIdx.x >> 5; j < p.rank; j += 8) {
        float s = 0.0f;
        for (int k = lane; k < p.K; k += 32)
            s = fmaf(lora_load<BF16>(p.x, static_cast<size_t>(m) * p.K + k), bf16_bits_to_f32(p.A[(static_cast<size_t>(a) * p.rank + j) * p.K + k]), s);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        if (lane == 0) p.t[static_cast<size_t>(m) * p.rank + j] = s * p.scaling[a];
    }
}

template <bool BF16>
__global__ void __launch_bounds__(256)
lora_up_kernel(const LoraParams p) {
    pdl_launch_dependents();
    pdl_wait();
    const int m = blockIdx.x;
    const int a = lora_adapter_of(p, m);
    if (a == -2) return;
    for (int n = threadIdx.x; n < p.N; n += 256) {
        const size_t at = static_cast<size_t>(m) * p.N + n;
        float s = 0.0f;
        if (a >= 0)
            for (int j = 0; j < p.rank; ++j)
                s = fmaf(p.t[static_cast<size_t>(m) * p.rank + j], bf16_bits_to_f32(p.B[(static_cast<size_t>(a) * p.N + n) * p.rank + j]), s);
        if (p.y) s += lora_load<BF16>(p.y, at);
        if constexpr (BF16) static_cast<uint16_t*>(p.out)[at] = f32_to_bf16_bits(s);
        else static_cast<float*>(p.out)[at] = s;
    }
}

}  // namespace qift
