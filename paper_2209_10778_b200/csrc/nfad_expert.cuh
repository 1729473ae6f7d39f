// nfad_expert.cuh -- Eq. 4 on rows grouped by expert: gz = grad_out f', and each expert's bias gradient, in one pass.
//
// A thread owns one column packet of a chunk of consecutive rows, as in the bias-fused backward.  An expert's rows may begin
// and end anywhere in a chunk: at each border the thread hands its column sums over, straight to the result when the
// expert's rows all lie in the chunk, else to the chunk's slot 0 (the expert that the chunk begins in) or 1 (the one it
// ends in); a second kernel adds the slots of an expert in row order.  The sums are of the unrounded products (exact in
// fp32 for 16-bit factors), in fp32 and in a fixed order.  Three tensors of traffic bound it.
#pragma once

#include "nfad_bias.cuh"

namespace nfad {

struct ExpertActArgs {
    const void *g, *d;                   // d null: f' = 1
    void* gz;                            // may be null when d is null
    float *grad_bias, *partial;          // grad_bias null: not wanted; partial [chunks][2][cols]
    const int* offsets;
    size_t rows;
    uint32_t cols, row_packets, chunk_rows, chunks, experts;
};

__device__ __forceinline__ size_t expert_offset(const ExpertActArgs& a, uint32_t e)
{
    const int v = __ldg(a.offsets + e);
    return v < 0 ? 0 : size_t(v) < a.rows ? size_t(v) : a.rows;
}

// The expert that `row` belongs to (experts when none) and where its run of rows ends (always past `row`).
__device__ __forceinline__ uint32_t expert_of(const ExpertActArgs& a, size_t row, size_t* end)
{
    if (row < expert_offset(a, 0)) {
        *end = expert_offset(a, 0);
        return a.experts;
    }
    uint32_t lo = 0, hi = a.experts + 1;
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) / 2;
        if (expert_offset(a, mid) <= row) lo = mid;
        else hi = mid;
    }
    *end = lo < a.experts ? expert_offset(a, lo + 1) : a.rows;
    if (*end <= row) *end = row + 1;
    return lo;
}

__device__ __forceinline__ float* expert_target(const ExpertActArgs& a, size_t chunk, size_t r0, size_t r1, uint32_t e)
{
    const size_t g0 = expert_offset(a, e), g1 = expert_offset(a, e + 1);
    if (g0 >= r0 && g1 <= r1) return a.grad_bias + size_t(e) * a.cols;
    return a.partial + (chunk * 2 + (g0 <= r0 ? 0 : 1)) * a.cols;
}

// kVec: whole 16-byte packets; else one column a thread
template <class S, bool kVec>
__global__ void __launch_bounds__(kBiasMaxBlock) expert_act_kernel(const __grid_constant__ ExpertActArgs a)
{
    constexpr int V = kVec ? S::kVec : 1, U = kBiasRows;
    using E = typename S::elem;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const uint32_t cp = blockIdx.x * blockDim.x + threadIdx.x;
    if (cp >= a.row_packets) return;
    const size_t r0 = size_t(blockIdx.y) * a.chunk_rows, r1 = r0 + a.chunk_rows < a.rows ? r0 + a.chunk_rows : a.rows;
    auto load = [&](const void* base, size_t row, float (&v)[V]) {
        if constexpr (kVec) S::unpack(load_packet(static_cast<const uint4*>(base) + row * a.row_packets + cp), v);
        else v[0] = S::load1(static_cast<const E*>(base) + row * a.cols + cp);
    };
    auto store = [&](size_t row, const float (&v)[V]) {
        if constexpr (kVec) store_packet<true>(static_cast<uint4*>(a.gz) + row * a.row_packets + cp, S::pack(v));
        else S::store1(static_cast<E*>(a.gz) + row * a.cols + cp, v[0]);
    };
    for (size_t row = r0; row < r1;) {
        size_t end;
        const uint32_t e = expert_of(a, row, &end);
        if (end > r1) end = r1;
        float acc[V];
#pragma unroll
        for (int i = 0; i < V; ++i) acc[i] = 0.0f;
        if (e >= a.experts) {                                        // nobody's rows
            if (a.gz)
                for (; row < end; ++row) store(row, acc);
            row = end;
            continue;
        }
        for (; row < end; row += U) {
            float g[U][V], d[U][V];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (row + u < end) {
                    load(a.g, row + u, g[u]);
                    if (a.d) load(a.d, row + u, d[u]);
                }
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (row + u < end) {
                    if (a.d)
#pragma unroll
                        for (int i = 0; i < V; ++i) g[u][i] = __fmul_rn(g[u][i], d[u][i]);
                    if (a.gz) store(row + u, g[u]);
#pragma unroll
                    for (int i = 0; i < V; ++i) acc[i] = __fadd_rn(acc[i], g[u][i]);
                }
        }
        row = end;
        if (a.grad_bias) {
            float* dst = expert_target(a, blockIdx.y, r0, r1, e) + size_t(cp) * V;
#pragma unroll
            for (int i = 0; i < V; ++i) dst[i] = acc[i];
        }
    }
}

// The experts whose rows lie in several chunks, and those without rows.
static __global__ void __launch_bounds__(32 * kBiasGroups) expert_reduce_kernel(const __grid_constant__ ExpertActArgs a)
{
    __shared__ float smem[kBiasGroups][32];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int lane = threadIdx.x & 31, group = threadIdx.x >> 5;
    const size_t col = size_t(blockIdx.x) * 32 + lane;
    const uint32_t e = blockIdx.y;
    const size_t g0 = expert_offset(a, e), g1 = expert_offset(a, e + 1);
    float* out = a.grad_bias + size_t(e) * a.cols;
    if (g1 <= g0) {
        if (group == 0 && col < a.cols) out[col] = 0.0f;
        return;
    }
    const size_t c0 = g0 / a.chunk_rows, c1 = (g1 - 1) / a.chunk_rows + 1;
    if (c1 - c0 == 1) return;                                        // written by its chunk
    const size_t per = (c1 - c0 + kBiasGroups - 1) / kBiasGroups;
    const size_t k0 = c0 + group * per, k1 = k0 + per < c1 ? k0 + per : c1;
    float s = 0.0f;
    if (col < a.cols)
        for (size_t k = k0; k < k1; ++k) s = __fadd_rn(s, a.partial[(k * 2 + (g0 <= k * a.chunk_rows ? 0 : 1)) * a.cols + col]);
    smem[group][lane] = s;
    __syncthreads();
    if (group == 0 && col < a.cols) {
        float t = smem[0][lane];
#pragma unroll
        for (int j = 1; j < kBiasGroups; ++j) t = __fadd_rn(t, smem[j][lane]);
        out[col] = t;
    }
}

inline size_t expert_act_scratch_bytes(size_t rows, size_t cols, int sms)
{
    if (rows == 0 || cols == 0) return 0;
    return size_t(bias_plan<8>(rows, cols, sms).chunks) * 2 * cols * sizeof(float);
}

template <class S> cudaError_t launch_expert_act(const ExpertActArgs& in, cudaStream_t st)
{
    ExpertActArgs a = in;
    DeviceInfo di;
    cudaError_t e = device_info(&di);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute attr[1];
    const BiasPlan p = bias_plan<8>(a.rows ? a.rows : 1, a.cols, di.sm_count);
    a.chunk_rows = p.chunk_rows;
    a.chunks = p.chunks;
    if (a.rows) {
        const bool vec = a.cols % 8 == 0 && aligned16(a.g) && aligned16(a.d) && aligned16(a.gz);
        a.row_packets = vec ? a.cols / 8 : a.cols;
        const unsigned block = bias_block(a.row_packets);
        bias_launch_config(&cfg, attr, (a.row_packets + block - 1) / block, block, st, true);
        cfg.gridDim.y = p.chunks;
        e = vec ? cudaLaunchKernelEx(&cfg, expert_act_kernel<S, true>, a) : cudaLaunchKernelEx(&cfg, expert_act_kernel<S, false>, a);
        if (e != cudaSuccess) return e;
    }
    if (!a.grad_bias) return cudaSuccess;
    bias_launch_config(&cfg, attr, (a.cols + 31) / 32, 32 * kBiasGroups, st, true);
    cfg.gridDim.y = a.experts;
    return cudaLaunchKernelEx(&cfg, expert_reduce_kernel, a);
}

}  // namespace nfad
