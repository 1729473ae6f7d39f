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

// kVec: whole 16-byte packets; else one column a thread.  The rows go by fours, whatever experts they belong to, so that the
// loads of a group are all in flight before the first is used and an expert's border costs a thread one look at the offsets.
template <class S, bool kVec> struct ExpertPacket { uint4 v; };
template <class S> struct ExpertPacket<S, false> { typename S::elem v; };

template <class S, bool kVec>
__global__ void __launch_bounds__(kBiasMaxBlock, 4) expert_act_kernel(const __grid_constant__ ExpertActArgs a)
{
    constexpr int V = kVec ? S::kVec : 1, U = kBiasRows;
    using E = typename S::elem;
    using Packet = ExpertPacket<S, kVec>;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const uint32_t cp = blockIdx.x * blockDim.x + threadIdx.x;
    if (cp >= a.row_packets) return;
    const size_t r0 = size_t(blockIdx.y) * a.chunk_rows, r1 = r0 + a.chunk_rows < a.rows ? r0 + a.chunk_rows : a.rows;
    if (r0 >= r1) return;
    auto load = [&](const void* base, size_t row) {
        Packet p;
        if constexpr (kVec) p.v = load_packet(static_cast<const uint4*>(base) + row * a.row_packets + cp);
        else p.v = static_cast<const E*>(base)[row * a.cols + cp];
        return p;
    };
    auto widen = [&](const Packet& p, float (&v)[V]) {
        if constexpr (kVec) S::unpack(p.v, v);
        else v[0] = S::load1(&p.v);
    };
    float acc[V];
#pragma unroll
    for (int i = 0; i < V; ++i) acc[i] = 0.0f;
    uint32_t e = a.experts;
    size_t end = r0;                                                  // of the run of rows that `row` is in
    auto hand_over = [&]() {
        if (a.grad_bias && e < a.experts) {
            float* dst = expert_target(a, blockIdx.y, r0, r1, e) + size_t(cp) * V;
#pragma unroll
            for (int i = 0; i < V; ++i) dst[i] = acc[i];
        }
#pragma unroll
        for (int i = 0; i < V; ++i) acc[i] = 0.0f;
    };
    for (size_t row = r0; row < r1; row += U) {
        Packet g[U], d[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (row + u < r1) {
                g[u] = load(a.g, row + u);
                if (a.d) d[u] = load(a.d, row + u);
            }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (row + u >= r1) break;
            if (row + u == end) {
                if (row + u > r0) hand_over();
                e = expert_of(a, row + u, &end);
            }
            float v[V];
            if (e < a.experts) {
                widen(g[u], v);
                if (a.d) {
                    float f[V];
                    widen(d[u], f);
#pragma unroll
                    for (int i = 0; i < V; ++i) v[i] = __fmul_rn(v[i], f[i]);
                }
#pragma unroll
                for (int i = 0; i < V; ++i) acc[i] = __fadd_rn(acc[i], v[i]);
            } else {                                                 // nobody's row, whatever it holds
#pragma unroll
                for (int i = 0; i < V; ++i) v[i] = 0.0f;
            }
            if (a.gz) {
                if constexpr (kVec) store_packet<true>(static_cast<uint4*>(a.gz) + (row + u) * a.row_packets + cp, S::pack(v));
                else S::store1(static_cast<E*>(a.gz) + (row + u) * a.cols + cp, v[0]);
            }
        }
    }
    hand_over();
}

// The experts whose rows lie in several chunks, and those without rows.  32 columns times kExpertGroups runs of consecutive
// chunks to a CTA: small, as an expert has few chunks when there are many experts (32 runs: 14 us for 61 experts of 1416).
constexpr int kExpertGroups = 8;
static __global__ void __launch_bounds__(32 * kExpertGroups) expert_reduce_kernel(const __grid_constant__ ExpertActArgs a)
{
    __shared__ float smem[kExpertGroups][32];
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
    const size_t per = (c1 - c0 + kExpertGroups - 1) / kExpertGroups;
    const size_t k0 = c0 + group * per, k1 = k0 + per < c1 ? k0 + per : c1;
    float s = 0.0f;
    if (col < a.cols)
        for (size_t k = k0; k < k1; k += 8) {
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j)
                v[j] = k + j < k1 ? a.partial[((k + j) * 2 + (g0 <= (k + j) * a.chunk_rows ? 0 : 1)) * a.cols + col] : 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (k + j < k1) s = __fadd_rn(s, v[j]);
        }
    smem[group][lane] = s;
    __syncthreads();
    if (group == 0 && col < a.cols) {
        float t = smem[0][lane];
#pragma unroll
        for (int j = 1; j < kExpertGroups; ++j) t = __fadd_rn(t, smem[j][lane]);
        out[col] = t;
    }
}

// Rows of a chunk, by shape and device alone: as many CTAs of 256 threads as are resident at a time (four to an SM), twice over, and
// no fewer than eight rows to a chunk.
inline uint32_t expert_chunk_rows(size_t rows, size_t cols, int sms)
{
    const size_t strips = (cols / 8 + kBiasMaxBlock - 1) / kBiasMaxBlock + (cols < 8);
    const size_t chunks = (size_t(sms) * 8 + strips - 1) / strips;
    size_t n = (rows + chunks - 1) / chunks;
    n = (n + kBiasRows - 1) / kBiasRows * kBiasRows;
    return uint32_t(n < 8 ? 8 : n);
}

inline size_t expert_act_scratch_bytes(size_t rows, size_t cols, int sms)
{
    if (rows == 0 || cols == 0) return 0;
    const size_t n = expert_chunk_rows(rows, cols, sms);
    return (rows + n - 1) / n * 2 * cols * sizeof(float);
}

template <class S> cudaError_t launch_expert_act(const ExpertActArgs& in, cudaStream_t st)
{
    ExpertActArgs a = in;
    DeviceInfo di;
    cudaError_t e = device_info(&di);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute attr[1];
    a.chunk_rows = expert_chunk_rows(a.rows, a.cols, di.sm_count);
    a.chunks = uint32_t((a.rows + a.chunk_rows - 1) / a.chunk_rows);
    if (a.rows) {
        const bool vec = a.cols % 8 == 0 && aligned16(a.g) && aligned16(a.d) && aligned16(a.gz);
        a.row_packets = vec ? a.cols / 8 : a.cols;
        const unsigned block = bias_block(a.row_packets);
        bias_launch_config(&cfg, attr, (a.row_packets + block - 1) / block, block, st, true);
        cfg.gridDim.y = a.chunks;
        e = vec ? cudaLaunchKernelEx(&cfg, expert_act_kernel<S, true>, a) : cudaLaunchKernelEx(&cfg, expert_act_kernel<S, false>, a);
        if (e != cudaSuccess) return e;
    }
    if (!a.grad_bias) return cudaSuccess;
    bias_launch_config(&cfg, attr, (a.cols + 31) / 32, 32 * kExpertGroups, st, true);
    cfg.gridDim.y = a.experts;
    return cudaLaunchKernelEx(&cfg, expert_reduce_kernel, a);
}

}  // namespace nfad
