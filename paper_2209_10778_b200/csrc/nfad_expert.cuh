// nfad_expert.cuh -- Eq. 4 on rows grouped by expert: gz = grad_out f', and each expert's bias gradient, in one pass.
//
// A thread owns one column packet of a chunk of consecutive rows, as in the bias-fused backward.  An expert's rows may begin
// and end anywhere in a chunk: at each border the thread hands its column sums over, straight to the result when the
// expert's rows all lie in the chunk, else to the chunk's slot 0 (an expert whose rows begin before the chunk) or 1 (one whose rows
// begin in it and go on); a second kernel adds the slots of an expert in row order.  The sums are of the unrounded products (exact in
// fp32 for 16-bit factors), in fp32 and in a fixed order.  Three tensors of traffic bound it.
#pragma once

#include "nfad_bias.cuh"
#include "nfad_product_args.h"

namespace nfad {

struct ExpertActArgs {
    const void *g, *d;                   // d null: f' = 1
    void* gz;                            // may be null when d is null
    float *grad_bias, *partial;          // grad_bias null: not wanted; partial [chunks][2][cols]
    int* begin;                          // [experts + 1] where each expert's rows begin, for the second kernel
    const int* offsets;
    size_t rows;
    uint32_t cols, row_packets, chunk_rows, chunks, experts;
};

// Offsets mean what they mean to the products: they are held to [0, rows], and an expert begins no earlier than the largest offset before
// it.  So a row belongs to the expert in front of the first offset above it, whose rows end at that offset.
__device__ __forceinline__ int expert_offset(const ExpertActArgs& a, uint32_t e) { return min(max(__ldg(a.offsets + e), 0), int(a.rows)); }

struct ExpertRun {
    uint32_t next;                       // the first offset above the run's rows: they are expert next - 1's (0 or experts + 1: nobody's)
    int end;                             // behind its last row
    bool here;                           // its first row is in this chunk
};

// The run that holds `row`, found by a warp together, 32 kWide offsets at a time; no offset before `from` is above it.  here: it begins at `row`.
template <int kWide> __device__ __forceinline__ ExpertRun expert_run(const ExpertActArgs& a, int row, uint32_t from)
{
    const int lane = threadIdx.x & 31;
    uint32_t at_row = 0;
    for (uint32_t i0 = from; i0 <= a.experts; i0 += 32 * kWide) {
        int v[kWide];
#pragma unroll
        for (int j = 0; j < kWide; ++j) v[j] = i0 + j * 32 + lane <= a.experts ? expert_offset(a, i0 + j * 32 + lane) : -1;
#pragma unroll
        for (int j = 0; j < kWide; ++j) {
            const uint32_t above = __ballot_sync(0xffffffffu, v[j] > row);
            at_row |= __ballot_sync(0xffffffffu, v[j] == row) & (above - 1 & ~above);       // those in front of the first above
            if (above) {
                const int first = __ffs(above) - 1;
                return {i0 + j * 32 + first, __shfl_sync(0xffffffffu, v[j], first), at_row != 0};
            }
        }
    }
    return {a.experts + 1, int(a.rows), at_row != 0};
}

// By one warp: where each expert's rows begin.
__device__ __forceinline__ void expert_begins(const ExpertActArgs& a)
{
    const uint32_t lane = threadIdx.x & 31;
    int last = 0;
    for (uint32_t i0 = 0; i0 <= a.experts; i0 += 32) {
        int v = i0 + lane <= a.experts ? max(expert_offset(a, i0 + lane), last) : last;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int w = __shfl_up_sync(0xffffffffu, v, o);
            if (lane >= o) v = max(v, w);
        }
        if (i0 + lane <= a.experts) a.begin[i0 + lane] = v;
        last = __shfl_sync(0xffffffffu, v, 31);
    }
}

// kVec: whole 16-byte packets; else one column a thread.  The rows go by fours, whatever experts they belong to, so that the
// loads of a group are all in flight before the first is used and an expert's border costs a warp one look at the offsets.
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
    if ((cp & ~31u) >= a.row_packets) return;                         // whole warps only: a warp looks at the offsets together
    const bool on = cp < a.row_packets;
    const int r0 = int(blockIdx.y * a.chunk_rows), r1 = int(min(size_t(r0) + a.chunk_rows, a.rows));      // rows are below 2^31
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
    ExpertRun run = {0, r0, false};                                   // of the row at hand
    // straight to the result when all of the expert's rows are in the chunk; else to slot 0 (they begin before it) or 1
    auto hand_over = [&]() {
        const uint32_t e = run.next - 1;
        if (a.grad_bias && on && e < a.experts) {
            float* dst = (run.here && run.end <= r1 ? a.grad_bias + size_t(e) * a.cols : a.partial + (size_t(blockIdx.y) * 2 + run.here) * a.cols) + size_t(cp) * V;
#pragma unroll
            for (int i = 0; i < V; ++i) dst[i] = acc[i];
        }
#pragma unroll
        for (int i = 0; i < V; ++i) acc[i] = 0.0f;
    };
    for (int row = r0; row < r1; row += U) {
        Packet g[U], d[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (on && row + u < r1) {
                g[u] = load(a.g, row + u);
                if (a.d) d[u] = load(a.d, row + u);
            }
        if (row == r0) run = expert_run<4>(a, row, 0);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (row + u >= r1) break;
            if (row + u == run.end) {
                hand_over();
                run = expert_run<1>(a, row + u, run.next);
                run.here = true;                                     // the offset that ended the run before is this row
            }
            float v[V];
            if (run.next - 1 < a.experts) {
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
            if (a.gz && on) {
                if constexpr (kVec) store_packet<true>(static_cast<uint4*>(a.gz) + size_t(row + u) * a.row_packets + cp, S::pack(v));
                else S::store1(static_cast<E*>(a.gz) + size_t(row + u) * a.cols + cp, v[0]);
            }
        }
    }
    hand_over();
    if (a.grad_bias && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x < 32) expert_begins(a);
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
    const size_t g0 = a.rows ? a.begin[e] : 0, g1 = a.rows ? a.begin[e + 1] : 0;
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
                v[j] = k + j < k1 ? a.partial[((k + j) * 2 + (g0 < (k + j) * a.chunk_rows ? 0 : 1)) * a.cols + col] : 0.0f;
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
    return (rows + n - 1) / n * 2 * cols * sizeof(float) + (kMaxExperts + 1) * sizeof(int);
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
    a.begin = reinterpret_cast<int*>(a.partial + size_t(a.chunks) * 2 * a.cols);
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
