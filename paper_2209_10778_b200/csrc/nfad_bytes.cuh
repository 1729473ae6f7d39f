// nfad_bytes.cuh -- rows in 8-bit integers: q = rint(x (127 / amax)), scale = amax / 127, amax the row's largest magnitude.
//
// One read from memory, one byte written per element: the row stays in registers, or is swept twice, the second time from L1.  A row whose amax
// is below 2^-120 counts as zero (127 / amax would leave fp32's range): scale 0, q 0.  A row that holds an infinity or a
// NaN has scale NaN and q 0, so that everything computed from it is NaN.
#pragma once

#include "nfad_hw.cuh"
#include "nfad_norm.cuh"

namespace nfad {

struct QuantizeArgs {
    const void* x;
    signed char* q;
    float* scale;
    size_t rows;
    uint32_t cols;
    int vec;
};

// the factor that takes a row to its integers, and the row's scale
__device__ __forceinline__ float quantize_factor(float amax, float* scale)
{
    const bool finite = amax <= 3.40282347e+38f;                      // false for NaN too
    *scale = finite ? (amax < 7.5231638e-37f ? 0.0f : __fdiv_rn(amax, 127.0f)) : __int_as_float(0x7fffffff);
    return finite && amax >= 7.5231638e-37f ? __fdiv_rn(127.0f, amax) : 0.0f;
}
// amax (127 / amax) may round to 127 + 2^-17 at most: the integer is in [-127, 127].  A factor of 0 stands for a row of zeros, whatever x.
__device__ __forceinline__ int quantize1(float x, float factor) { return factor == 0.0f ? 0 : __float2int_rn(__fmul_rn(x, factor)); }

// fmaxf drops a NaN; this keeps it
__device__ __forceinline__ float larger(float a, float b) { return hw::max_nan(a, b); }

template <class S> __device__ __forceinline__ uint32_t quantize4(const float* v, float f)
{
    return uint32_t(quantize1(v[0], f) & 0xff) | uint32_t(quantize1(v[1], f) & 0xff) << 8 | uint32_t(quantize1(v[2], f) & 0xff) << 16 |
           uint32_t(quantize1(v[3], f) & 0xff) << 24;
}

template <class S> __global__ void __launch_bounds__(kBlock) quantize_kernel(const __grid_constant__ QuantizeArgs a)
{
    constexpr int V = S::kVec;
    __shared__ float part[2][kBlock / 32];
    // in this order: the next kernel may start only when everything in front of this one is complete, so that it may read what
    // neither of the two writes (the weights) before this one has ended
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    int turn = 0;
    for (size_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
        const typename S::elem* x = static_cast<const typename S::elem*>(a.x) + row * a.cols;
        signed char* q = a.q + row * a.cols;
        const uint32_t packets = a.vec ? a.cols / V : 0;
        float m = 0.0f;
        for (uint32_t p = threadIdx.x; p < packets; p += kBlock) {
            float v[V];
            S::unpack(reinterpret_cast<const uint4*>(x)[p], v);
#pragma unroll
            for (int e = 0; e < V; ++e) m = larger(m, fabsf(v[e]));
        }
        for (uint32_t c = packets * V + threadIdx.x; c < a.cols; c += kBlock) m = larger(m, fabsf(S::load1(x + c)));
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) m = larger(m, __shfl_xor_sync(0xffffffffu, m, o));
        if ((threadIdx.x & 31) == 0) part[turn][threadIdx.x >> 5] = m;
        __syncthreads();
        m = part[turn][0];
#pragma unroll
        for (int w = 1; w < kBlock / 32; ++w) m = larger(m, part[turn][w]);
        float scale;
        const float f = quantize_factor(m, &scale);
        if (threadIdx.x == 0) a.scale[row] = scale;
        for (uint32_t p = threadIdx.x; p < packets; p += kBlock) {
            float v[V];
            S::unpack(reinterpret_cast<const uint4*>(x)[p], v);
            if constexpr (V == 8) reinterpret_cast<uint2*>(q)[p] = make_uint2(quantize4<S>(v, f), quantize4<S>(v + 4, f));
            else reinterpret_cast<uint32_t*>(q)[p] = quantize4<S>(v, f);
        }
        for (uint32_t c = packets * V + threadIdx.x; c < a.cols; c += kBlock) q[c] = (signed char)quantize1(S::load1(x + c), f);
    }
}

// Aligned rows of up to 4 packets a thread, by a warp each (kWarp) or by a CTA: in registers, read once.
template <class S, int kI, bool kWarp> __global__ void __launch_bounds__(kBlock) quantize_held_kernel(const __grid_constant__ QuantizeArgs a)
{
    constexpr int V = S::kVec;
    __shared__ float part[kBlock / 32];
    asm volatile("griddepcontrol.wait;" ::: "memory");               // the order: see above
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const uint32_t lane = kWarp ? threadIdx.x & 31 : threadIdx.x, width = kWarp ? 32 : blockDim.x, packets = a.cols / V;
    const size_t row = kWarp ? size_t(blockIdx.x) * (kBlock / 32) + (threadIdx.x >> 5) : blockIdx.x;
    if (row >= a.rows) return;                                       // a whole warp, or a whole CTA
    const uint4* x = static_cast<const uint4*>(a.x) + row * packets;
    uint4 raw[kI];
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < kI; ++i) {
        const uint32_t p = lane + i * width;
        raw[i] = p < packets ? load_packet(x + p) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < kI; ++i) {
        float v[V];
        S::unpack(raw[i], v);
#pragma unroll
        for (int e = 0; e < V; ++e) m = larger(m, fabsf(v[e]));
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = larger(m, __shfl_xor_sync(0xffffffffu, m, o));
    if (!kWarp && blockDim.x > 32) {
        if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = m;
        __syncthreads();
        m = part[0];
        for (uint32_t w = 1; w < blockDim.x / 32; ++w) m = larger(m, part[w]);
    }
    float scale;
    const float f = quantize_factor(m, &scale);
    if (lane == 0) a.scale[row] = scale;
#pragma unroll
    for (int i = 0; i < kI; ++i) {
        const uint32_t p = lane + i * width;
        if (p >= packets) continue;
        float v[V];
        S::unpack(raw[i], v);
        if constexpr (V == 8) reinterpret_cast<uint2*>(a.q + row * a.cols)[p] = make_uint2(quantize4<S>(v, f), quantize4<S>(v + 4, f));
        else reinterpret_cast<uint32_t*>(a.q + row * a.cols)[p] = quantize4<S>(v, f);
    }
}

template <class S> cudaError_t launch_quantize(const void* x, signed char* q, float* scale, size_t rows, uint32_t cols, cudaStream_t st)
{
    QuantizeArgs a = {x, q, scale, rows, cols, 0};
    // rows of x begin on 16-byte boundaries and rows of q on a packet's integers
    a.vec = cols % S::kVec == 0 && (reinterpret_cast<uintptr_t>(x) & 15u) == 0 && (reinterpret_cast<uintptr_t>(q) & (S::kVec - 1)) == 0;
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute attr[1];
    const uint32_t packets = cols / S::kVec;
    if (a.vec && packets >= 1 && packets <= 128) {                    // [65536, 512] bf16: 19 us, 86 by a CTA each
        norm_launch_config(&cfg, attr, (rows + kBlock / 32 - 1) / (kBlock / 32), kBlock, st);
        if (packets <= 32) return cudaLaunchKernelEx(&cfg, quantize_held_kernel<S, 1, true>, a);
        if (packets <= 64) return cudaLaunchKernelEx(&cfg, quantize_held_kernel<S, 2, true>, a);
        return cudaLaunchKernelEx(&cfg, quantize_held_kernel<S, 4, true>, a);
    }
    if (a.vec && packets >= 1 && packets <= 4 * kBlock) {
        norm_launch_config(&cfg, attr, rows, packets <= 512 ? (packets + 63) / 64 * 32 : kBlock, st);
        if (packets <= 512) return cudaLaunchKernelEx(&cfg, quantize_held_kernel<S, 2, false>, a);
        return cudaLaunchKernelEx(&cfg, quantize_held_kernel<S, 4, false>, a);
    }
    norm_launch_config(&cfg, attr, rows, kBlock, st);
    return cudaLaunchKernelEx(&cfg, quantize_kernel<S>, a);
}

}  // namespace nfad
