// nfad_blocks.cuh -- values to 8-bit floating point (four exponent bits, three of the significand, largest 448) with a scale for each block of 128:
// scale = amax / 448, q = 448 x / amax rounded to nearest even, amax the block's largest magnitude.
//
// Activations: blocks of 128 along a row.  A block is 16 bytes to a thread (half a warp for 16-bit values, a warp for fp32), read once, with its
// largest magnitude found by shuffles; no block waits for another.  Weights: blocks of 128 x 128, a CTA each, held in registers.
// Bound by memory: 3 bytes an element of 16-bit tensors.
//
// 16-bit values often lie exactly between two of the 8-bit ones (a largest magnitude that is a multiple of 7 makes such quotients common), and
// x (448 / amax) in fp32 misses such a border by its roundings, to either side.  The quotient of two 16-bit significands is either on a border
// (a multiple of half a step: five bits) or away from it by 2^-16 of itself at least, while the fp32 product errs by less than 2^-22: so
// rounding it to 18 bits first puts it back on the border, and the result is the nearest 8-bit value to the exact quotient, ties to even.
// (fp32 values are not rounded twice: theirs is the nearest to the fp32 product.)
//
// A block with amax below 2^-110 counts as zero (448 / amax would leave fp32's range): scale 0, q 0.  One with an infinity or a NaN has scale
// NaN and q 0, so that everything computed from it is NaN.
#pragma once

#include <type_traits>

#include "nfad_bytes.cuh"

namespace nfad {

constexpr int kBlockSide = 128;
template <class S> struct IsBF16 { static constexpr bool value = false; };
template <> struct IsBF16<StoreBF16> { static constexpr bool value = true; };
constexpr float kLargestE4M3 = 448.0f;

struct BlockArgs {
    const void* x;
    unsigned char* q;
    float* scale;
    size_t rows;                         // of all matrices
    uint32_t cols, groups;               // groups: blocks along a row
    uint32_t matrix_rows;                // blocks of 128 x 128: of one matrix
    int vec;
};

// The factor that takes a block to its bytes (0: a block of zeros, whatever it holds), and its scale.  kSnap: an estimate of the reciprocal
// (2^-23) does, see above.
template <bool kSnap> __device__ __forceinline__ float block_factor(float amax, float* scale)
{
    const bool finite = amax <= 3.40282347e+38f;                      // false for NaN too
    const bool some = amax >= 7.7037198e-34f;                         // 2^-110
    *scale = finite ? (some ? __fdiv_rn(amax, kLargestE4M3) : 0.0f) : __int_as_float(0x7fffffff);
    return finite && some ? (kSnap ? (kLargestE4M3 * 0.0009765625f) * hw::rcp_approx(amax * 0.0009765625f)      // neither end of the range leaves fp32
                                    : __fdiv_rn(kLargestE4M3, amax)) : 0.0f;
}

// four values to four bytes; kSnap: through 18 bits, see above
template <bool kSnap> __device__ __forceinline__ uint32_t block_bytes(const float* x, float factor)
{
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        v[e] = __fmul_rn(x[e], factor);
        if (kSnap) v[e] = __uint_as_float((__float_as_uint(v[e]) + 32u) & ~63u);
    }
    unsigned short lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(v[1]), "f"(v[0]));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(v[3]), "f"(v[2]));
    return uint32_t(lo) | uint32_t(hi) << 16;
}
template <class S> struct Snap { static constexpr bool value = S::kVec == 8; };

// a packet's largest magnitude (NaN if it holds one); 16-bit values two at a time
template <class S> __device__ __forceinline__ float packet_largest(const uint4& p)
{
    if constexpr (S::kVec == 4) {
        float v[4];
        S::unpack(p, v);
        return larger(larger(fabsf(v[0]), fabsf(v[1])), larger(fabsf(v[2]), fabsf(v[3])));
    } else {
        using E2 = typename std::conditional<IsBF16<S>::value, __nv_bfloat162, __half2>::type;
        auto two = [](uint32_t w) { w &= 0x7fff7fffu; return *reinterpret_cast<const E2*>(&w); };
        const E2 m = __hmax2_nan(__hmax2_nan(two(p.x), two(p.y)), __hmax2_nan(two(p.z), two(p.w)));
        return larger(S::load1(&m.x), S::load1(&m.y));
    }
}

// V values from element c of a row on (zeros behind its end); returns their largest magnitude.  vec: rows begin on 16-byte boundaries
template <class S> __device__ __forceinline__ float block_load(const BlockArgs& a, bool vec, size_t row, uint32_t c, float (&v)[S::kVec])
{
    constexpr int V = S::kVec;
    const typename S::elem* x = static_cast<const typename S::elem*>(a.x) + row * a.cols + c;
    float m = 0.0f;
    if (vec) {
        const uint4 p = c < a.cols ? load_packet(reinterpret_cast<const uint4*>(x)) : make_uint4(0, 0, 0, 0);
        S::unpack(p, v);
        m = packet_largest<S>(p);
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e) {
            v[e] = c + e < a.cols ? S::load1(x + e) : 0.0f;
            m = larger(m, fabsf(v[e]));
        }
    }
    return m;
}
template <class S> __device__ __forceinline__ void block_store(const BlockArgs& a, bool vec, size_t row, uint32_t c, const float (&v)[S::kVec], float factor)
{
    constexpr int V = S::kVec;
    unsigned char* q = a.q + row * a.cols + c;
    uint32_t w[V / 4] = {};
    if (factor != 0.0f)
#pragma unroll
        for (int i = 0; i < V / 4; ++i) w[i] = block_bytes<Snap<S>::value>(v + i * 4, factor);
    if (vec) {
        if (c >= a.cols) return;
        if constexpr (V == 8) *reinterpret_cast<uint2*>(q) = make_uint2(w[0], w[1]);
        else *reinterpret_cast<uint32_t*>(q) = w[0];
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (c + e < a.cols) q[e] = (unsigned char)(w[e >> 2] >> 8 * (e & 3));
    }
}

// Rows on 16-byte boundaries: a group of kBlockSide / V threads has one block of each of kGroupRows rows, so that nothing is divided to find its
// place, and one division makes the scales of all of them, a lane each.
constexpr int kGroupRows = 4;
template <class S> __global__ void __launch_bounds__(kBlock) quantize_row_groups_kernel(const __grid_constant__ BlockArgs a)
{
    constexpr int V = S::kVec, T = kBlockSide / V, U = kGroupRows;
    asm volatile("griddepcontrol.wait;" ::: "memory");               // the order: see quantize_groups_kernel
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const uint32_t lane = threadIdx.x % T, group = (blockIdx.x * blockDim.x + threadIdx.x) / T, c = group * kBlockSide + lane * V;
    const bool on = c < a.cols;                                       // else a thread behind the row's end, there for the shuffles
    for (size_t row0 = size_t(blockIdx.y) * U; row0 < a.rows; row0 += size_t(gridDim.y) * U) {
        const uint4* x = reinterpret_cast<const uint4*>(static_cast<const typename S::elem*>(a.x) + row0 * a.cols + c);
        const size_t pitch = a.cols / V;
        uint4 raw[U];
        float m[U];
#pragma unroll
        for (int u = 0; u < U; ++u) raw[u] = on && row0 + u < a.rows ? load_packet(x + u * pitch) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int u = 0; u < U; ++u) m[u] = packet_largest<S>(raw[u]);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int o = T / 2; o > 0; o >>= 1) m[u] = larger(m[u], __shfl_xor_sync(0xffffffffu, m[u], o));
        float mine = m[0];
#pragma unroll
        for (int u = 1; u < U; ++u) mine = lane == u ? m[u] : mine;
        float scale;
        const float f = block_factor<Snap<S>::value>(mine, &scale);
        if (lane < U && group < a.groups && row0 + lane < a.rows) a.scale[size_t(group) * a.rows + row0 + lane] = scale;
        unsigned char* q = a.q + row0 * a.cols + c;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float factor = __shfl_sync(0xffffffffu, f, u, T);
            if (!on || row0 + u >= a.rows) continue;
            float v[V];
            S::unpack(raw[u], v);
            uint32_t w[V / 4] = {};
            if (factor != 0.0f)
#pragma unroll
                for (int i = 0; i < V / 4; ++i) w[i] = block_bytes<Snap<S>::value>(v + i * 4, factor);
            if constexpr (V == 8) *reinterpret_cast<uint2*>(q + size_t(u) * a.cols) = make_uint2(w[0], w[1]);
            else *reinterpret_cast<uint32_t*>(q + size_t(u) * a.cols) = w[0];
        }
    }
}

// Rows off the 16-byte boundaries: groups of kBlockSide / V threads, a block of a row each, element by element; scale [groups, rows].
template <class S> __global__ void __launch_bounds__(kBlock) quantize_groups_kernel(const __grid_constant__ BlockArgs a)
{
    constexpr int V = S::kVec, T = kBlockSide / V, U = 2;
    // in this order: the next kernel may start only when everything in front of this one is complete, so that it may read what
    // neither of the two writes (the weights) before this one has ended
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const uint32_t lane = threadIdx.x % T, per = kBlock / T * U;
    const size_t total = a.rows * a.groups;
    for (size_t i0 = size_t(blockIdx.x) * per; i0 < total; i0 += size_t(gridDim.x) * per) {
        float v[U][V], m[U];
        size_t row[U];
        uint32_t c[U], group[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const size_t i = i0 + u * (kBlock / T) + threadIdx.x / T;
            row[u] = total >> 32 ? i / a.groups : uint32_t(i) / a.groups;
            group[u] = uint32_t(i - row[u] * a.groups);
            c[u] = i < total ? group[u] * kBlockSide + lane * V : a.cols;
            if (i >= total) row[u] = 0;
            m[u] = block_load<S>(a, false, row[u], c[u], v[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int o = T / 2; o > 0; o >>= 1) m[u] = larger(m[u], __shfl_xor_sync(0xffffffffu, m[u], o));
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float scale;
            const float f = block_factor<Snap<S>::value>(m[u], &scale);
            if (lane == 0 && c[u] < a.cols) a.scale[size_t(group[u]) * a.rows + row[u]] = scale;
            block_store<S>(a, false, row[u], c[u], v[u], f);
        }
    }
}

// A CTA to a block of 128 x 128; scale [matrices, blocks of rows, groups].
template <class S> __global__ void __launch_bounds__(kBlock) quantize_blocks_kernel(const __grid_constant__ BlockArgs a)
{
    constexpr int V = S::kVec, T = kBlockSide / V, kRows = kBlock / T, kTurns = kBlockSide / kRows;
    __shared__ float part[kBlock / 32];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const uint32_t row_blocks = (a.matrix_rows + kBlockSide - 1) / kBlockSide;
    const size_t matrix = blockIdx.x / (size_t(row_blocks) * a.groups), in_matrix = blockIdx.x - matrix * row_blocks * a.groups;
    const uint32_t block = uint32_t(in_matrix / a.groups), group = uint32_t(in_matrix - size_t(block) * a.groups);
    const uint32_t c = group * kBlockSide + threadIdx.x % T * V, r0 = block * kBlockSide + threadIdx.x / T;
    float v[kTurns][V], m = 0.0f;
#pragma unroll
    for (int i = 0; i < kTurns; ++i) {
        const uint32_t r = r0 + i * kRows;
        if (r < a.matrix_rows) m = larger(m, block_load<S>(a, a.vec, matrix * a.matrix_rows + r, c, v[i]));
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = larger(m, __shfl_xor_sync(0xffffffffu, m, o));
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = m;
    __syncthreads();
    m = part[0];
#pragma unroll
    for (int w = 1; w < kBlock / 32; ++w) m = larger(m, part[w]);
    float scale;
    const float f = block_factor<Snap<S>::value>(m, &scale);
    if (threadIdx.x == 0) a.scale[blockIdx.x] = scale;
#pragma unroll
    for (int i = 0; i < kTurns; ++i) {
        const uint32_t r = r0 + i * kRows;
        if (r < a.matrix_rows) block_store<S>(a, a.vec, matrix * a.matrix_rows + r, c, v[i], f);
    }
}

template <class S> BlockArgs block_args(const void* x, unsigned char* q, float* scale, size_t rows, uint32_t matrix_rows, uint32_t cols)
{
    BlockArgs a = {x, q, scale, rows, cols, (cols + kBlockSide - 1) / kBlockSide, matrix_rows, 0};
    // rows of x begin on 16-byte boundaries and rows of q on a packet's bytes
    a.vec = cols % S::kVec == 0 && (reinterpret_cast<uintptr_t>(x) & 15u) == 0 && (reinterpret_cast<uintptr_t>(q) & (S::kVec - 1)) == 0;
    return a;
}

template <class S> cudaError_t launch_quantize_groups(const void* x, unsigned char* q, float* scale, size_t rows, uint32_t cols, cudaStream_t st)
{
    const BlockArgs a = block_args<S>(x, q, scale, rows, 0, cols);
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute attr[1];
    if (a.vec) {
        const uint32_t threads = (a.groups * (kBlockSide / S::kVec) + 31) / 32 * 32, block = threads < kBlock ? threads : kBlock;
        const size_t runs = (rows + kGroupRows - 1) / kGroupRows;
        norm_launch_config(&cfg, attr, (threads + block - 1) / block, block, st);
        cfg.gridDim.y = unsigned(runs < 65535 ? runs : 65535);
        return cudaLaunchKernelEx(&cfg, quantize_row_groups_kernel<S>, a);
    }
    constexpr size_t per = kBlock / (kBlockSide / S::kVec) * 2;
    const size_t grid = (rows * a.groups + per - 1) / per;
    norm_launch_config(&cfg, attr, grid < 0x7fffffff ? grid : 0x7fffffff, kBlock, st);
    return cudaLaunchKernelEx(&cfg, quantize_groups_kernel<S>, a);
}

template <class S> cudaError_t launch_quantize_blocks(const void* x, unsigned char* q, float* scale, size_t matrices, uint32_t rows, uint32_t cols, cudaStream_t st)
{
    const BlockArgs a = block_args<S>(x, q, scale, matrices * rows, rows, cols);
    const size_t grid = matrices * ((rows + kBlockSide - 1) / kBlockSide) * a.groups;
    if (grid >= (size_t(1) << 31)) return cudaErrorInvalidValue;     // beyond what any device's memory holds
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute attr[1];
    norm_launch_config(&cfg, attr, grid, kBlock, st);
    return cudaLaunchKernelEx(&cfg, quantize_blocks_kernel<S>, a);
}

}  // namespace nfad
