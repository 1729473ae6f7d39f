// nfad_norm.cuh -- the norms before and after a block, fused with the block's gate and the residual scale.
//
//   a = N_post(u) g_post + b_post            u: the block's output
//   s = alpha r + gate a                     r: the residual stream; s: its new value, stored rounded once
//   h = N_pre(s) g_pre + b_pre               of the unrounded s: the next block's input
//
// N is nothing, x rho with rho = (mean x^2 + eps)^-1/2 (RMS), or (x - mu) rho with rho = (var + eps)^-1/2 (LAYER).
// Unfused this is four passes (norm, gate, residual sum, norm) of 2 to 3 tensors each; here each row is read once,
// held in registers across its two reductions, and s and h are written once: two tensors in, two out, which bounds it
// by HBM traffic.  All arithmetic is fp32; the variance is taken about the mean in a second sweep over the registers.
//
// Backward, from dh and the stream's own gradient ds', the stored s, u and the four row statistics (^: normalised):
//   d = dh g_pre;  ds = ds' + rho_s (d - mean d [LAYER] - s^ mean(d s^));      grad_r = alpha ds
//   da = gate ds;  e = da g_post;  grad_u = rho_u (e - mean e [LAYER] - u^ mean(e u^))
//   grad g_pre = sum dh s^, grad b_pre = sum dh, grad g_post = sum da u^, grad b_post = sum da over all rows;
//   grad gate = sum ds a over the rows that a gate row governs.  All in fp32 and in a fixed order.
// A CTA owns a run of consecutive rows and a thread the same columns of each, so the five column sums stay in
// registers; each CTA writes its sums once and a second kernel adds the CTAs' in a fixed order.  The next row's packets
// are in flight during the current row's two reductions.  Four tensors in, two out.
#pragma once

#include "nfad_hw.cuh"
#include "nfad_internal.h"
#include "nfad_norm_args.h"
#include "nfad_stream.cuh"
#include "nfad_tcgen.cuh"

namespace nfad {

// ---------------------------------------------------------------- sums over a row

// N sums over the threads of a row: the lanes of a warp (kWarp) or the whole CTA.  `turn` alternates between two buffers,
// so that one barrier per call is enough: a buffer is written again only after every thread has passed the next call's.
template <int N, bool kWarp> struct RowSum {
    float (*buf)[N][32];
    int turn;
    __device__ __forceinline__ void operator()(float (&v)[N])
    {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
        if (kWarp || blockDim.x == 32) return;
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = (blockDim.x + 31) >> 5;
        float (*b)[32] = buf[turn];
        turn ^= 1;
        if (lane == 0)
#pragma unroll
            for (int k = 0; k < N; ++k) b[k][warp] = v[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = (lane & 15) < warps ? b[k][lane & 15] : 0.0f;       // both halves of the warp alike
        if (warps > 16) {
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] += (lane & 15) + 16 < warps ? b[k][(lane & 15) + 16] : 0.0f;
        }
#pragma unroll
        for (int o = 8; o > 0; o >>= 1)
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
    }
};

// ---------------------------------------------------------------- forward

// parameters are read by every row: plain cached loads
template <class S> __device__ __forceinline__ void load_parameter(const void* base, size_t row, uint32_t packets, uint32_t p, float (&v)[S::kVec])
{
    S::unpack(__ldg(static_cast<const uint4*>(base) + row * packets + p), v);
}

// Rows that do not start on 16-byte boundaries: a thread's packet of V elements is V / kUnit pieces of kUnit elements, the pieces of
// neighbouring threads side by side.
template <class S, int kUnit> struct RowColumns {
    static constexpr int V = S::kVec, kPieces = V / kUnit;
    using E = typename S::elem;
    uint32_t lane, width, cols;
    __device__ __forceinline__ uint32_t column(int i, int piece) const { return ((i * kPieces + piece) * width + lane) * kUnit; }
    // one bit for each element that is inside the row (rows hold whole pieces)
    __device__ __forceinline__ uint32_t mask(int i) const
    {
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < kPieces; ++j)
            if (column(i, j) < cols) m |= ((1u << kUnit) - 1) << (j * kUnit);
        return m;
    }
    // outside the row: zeros
    __device__ __forceinline__ uint4 load(const void* base, size_t row, int i) const
    {
        uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
            const E* at = static_cast<const E*>(base) + row * cols + column(i, j);
            if (column(i, j) < cols) {
                if constexpr (kUnit * sizeof(E) == 2) w[j >> 1] |= uint32_t(*reinterpret_cast<const unsigned short*>(at)) << (16 * (j & 1));
                else w[j] = *reinterpret_cast<const unsigned*>(at);
            }
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    __device__ __forceinline__ void store(void* base, size_t row, int i, const uint4& v) const
    {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
            E* at = static_cast<E*>(base) + row * cols + column(i, j);
            if (column(i, j) < cols) {
                if constexpr (kUnit * sizeof(E) == 2) *reinterpret_cast<unsigned short*>(at) = (unsigned short)(w[j >> 1] >> (16 * (j & 1)));
                else *reinterpret_cast<unsigned*>(at) = w[j];
            }
        }
    }
};

// 1 / sqrt(x): the hardware's approximation y and one Newton step, y + y (1 - x y^2) / 2, within one unit in the last place; 0 for a
// sum of squares that has overflowed (its row's normalised values are 0 then; the step alone would make NaN of it).  The intrinsic that
// rounds exactly takes a tenth longer on short rows ([65536, 128] bf16 20.6 us for 18.8, [14808, 100] 6.2 for 5.6).
__device__ __forceinline__ float reciprocal_root(float x)
{
    const float y = rsqrtf(x), root = fmaf(0.5f * y, fmaf(-x * y, y, 1.0f), y);
    return x > 3.40282347e+38f ? 0.0f : root;
}

// which gate row governs a row; divisions of 64 bits cost as much as a row's arithmetic, and are rarely needed
__device__ __forceinline__ size_t gate_row_of(size_t row, size_t rows_per_gate)
{
    if (row < rows_per_gate) return 0;
    if ((row | rows_per_gate) >> 32) return row / rows_per_gate;
    return uint32_t(row) / uint32_t(rows_per_gate);
}

// Means and reciprocal deviations of kR rows whose threads hold kI packets each; packets past the row hold zeros.
template <int V, int kUnit, int kR, int kI, bool kWarp, bool kMean>
__device__ __forceinline__ void row_statistics(const float (&v)[kR][kI][V], const uint32_t (&on)[kI], int kind, float inv_cols, float eps,
                                               RowSum<kR, kWarp>& sum, float (&mean)[kR], float (&rstd)[kR])
{
    float t[kR];
    if (kMean && kind == kNormLayer) {
#pragma unroll
        for (int k = 0; k < kR; ++k) {
            t[k] = 0.0f;
#pragma unroll
            for (int i = 0; i < kI; ++i)
#pragma unroll
                for (int e = 0; e < V; ++e) t[k] += v[k][i][e];
        }
        sum(t);
#pragma unroll
        for (int k = 0; k < kR; ++k) mean[k] = t[k] * inv_cols;
    }
#pragma unroll
    for (int k = 0; k < kR; ++k) {
        t[k] = 0.0f;
#pragma unroll
        for (int i = 0; i < kI; ++i)
            if (!kMean || on[i])
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    float c = kMean ? v[k][i][e] - mean[k] : v[k][i][e];
                    if (kMean && kUnit < V && !(on[i] >> e & 1)) c = 0.0f;
                    t[k] = fmaf(c, c, t[k]);
                }
    }
    sum(t);
#pragma unroll
    for (int k = 0; k < kR; ++k) rstd[k] = reciprocal_root(fmaf(t[k], inv_cols, eps));
}

// kR consecutive rows per CTA, or per warp (kWarp), kI packets of each per thread; cols a multiple of the packet, every pointer on a
// 16-byte boundary.  kMean: one of the norms is LAYER.  For 16-bit storage instructions are what is short (49 per element at
// first, 4.1 TB/s on [16384, 4096] bf16 against 6.0 for fp32 storage, where they are half as many per byte): so rows share
// each parameter's load and widening and each barrier, threads are few with much work each, and no 64-bit division is left.
// (A ring of bulk copies kept ahead of CTAs that stay, as backward has it, came to 92 us where this takes 87.)
template <class S, int kI, int kR, bool kWarp, bool kMean>
__global__ void __launch_bounds__(kWarp ? 128 : kI == 1 ? 512 : 256) norm_forward_kernel(const __grid_constant__ NormForwardArgs a)
{
    constexpr int V = S::kVec;
    __shared__ float buf[2][kR][32];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const uint32_t lane = kWarp ? threadIdx.x & 31 : threadIdx.x, width = kWarp ? 32 : blockDim.x;
    const size_t per_cta = kWarp ? blockDim.x >> 5 : 1;
    RowSum<kR, kWarp> sum{buf, 0};
    for (size_t turn = blockIdx.x * per_cta + (kWarp ? threadIdx.x >> 5 : 0); turn * kR < a.rows; turn += gridDim.x * per_cta) {
        const size_t row = turn * kR;
        uint4 ru[kR][kI], rr[kR][kI];
        uint32_t on[kI];
        bool there[kR];
#pragma unroll
        for (int k = 0; k < kR; ++k) there[k] = k == 0 || row + k < a.rows;
#pragma unroll
        for (int i = 0; i < kI; ++i) {
            const uint32_t p = lane + i * width;
            on[i] = p < a.packets;
#pragma unroll
            for (int k = 0; k < kR; ++k) {
                ru[k][i] = rr[k][i] = make_uint4(0, 0, 0, 0);
                if (on[i] && there[k]) {
                    ru[k][i] = load_packet(static_cast<const uint4*>(a.u) + (row + k) * a.packets + p);
                    if (a.r) rr[k][i] = load_packet(static_cast<const uint4*>(a.r) + (row + k) * a.packets + p);
                }
            }
        }
        float v[kR][kI][V], mean[kR], rstd[kR], mean2[kR], rstd2[kR];
#pragma unroll
        for (int k = 0; k < kR; ++k) {
            mean[k] = rstd[k] = mean2[k] = rstd2[k] = 0.0f;
#pragma unroll
            for (int i = 0; i < kI; ++i) S::unpack(ru[k][i], v[k][i]);
        }
        if (a.post != kNormNone) row_statistics<V, V, kR, kI, kWarp, kMean>(v, on, a.post, a.inv_cols, a.eps, sum, mean, rstd);
        size_t gate_row[kR];
#pragma unroll
        for (int k = 0; k < kR; ++k) gate_row[k] = a.gate ? gate_row_of(row + k, a.rows_per_gate) : 0;
#pragma unroll
        for (int i = 0; i < kI; ++i) {
            const uint32_t p = lane + i * width;
            if (!on[i]) continue;
            float w[V];
            if (a.post != kNormNone) {
#pragma unroll
                for (int k = 0; k < kR; ++k)
#pragma unroll
                    for (int e = 0; e < V; ++e) v[k][i][e] = kMean ? (v[k][i][e] - mean[k]) * rstd[k] : v[k][i][e] * rstd[k];
                if (a.post_gain) {
                    load_parameter<S>(a.post_gain, 0, a.packets, p, w);
#pragma unroll
                    for (int k = 0; k < kR; ++k)
#pragma unroll
                        for (int e = 0; e < V; ++e) v[k][i][e] *= w[e];
                }
                if (a.post_bias) {
                    load_parameter<S>(a.post_bias, 0, a.packets, p, w);
#pragma unroll
                    for (int k = 0; k < kR; ++k)
#pragma unroll
                        for (int e = 0; e < V; ++e) v[k][i][e] += w[e];
                }
            }
            if (a.gate) {
#pragma unroll
                for (int k = 0; k < kR; ++k) {
                    if (k > 0 && !there[k]) continue;
                    if (k == 0 || gate_row[k] != gate_row[0]) load_parameter<S>(a.gate, gate_row[k], a.packets, p, w);
#pragma unroll
                    for (int e = 0; e < V; ++e) v[k][i][e] *= w[e];
                }
            }
#pragma unroll
            for (int k = 0; k < kR; ++k) {
                if (a.r) {
                    S::unpack(rr[k][i], w);
#pragma unroll
                    for (int e = 0; e < V; ++e) v[k][i][e] = fmaf(a.alpha, w[e], v[k][i][e]);
                }
                if (a.s && there[k]) store_packet<true>(static_cast<uint4*>(a.s) + (row + k) * a.packets + p, S::pack(v[k][i]));
            }
        }
        if (a.pre != kNormNone) {
            row_statistics<V, V, kR, kI, kWarp, kMean>(v, on, a.pre, a.inv_cols, a.eps, sum, mean2, rstd2);
#pragma unroll
            for (int i = 0; i < kI; ++i) {
                const uint32_t p = lane + i * width;
                if (!on[i]) continue;
                float w[V];
#pragma unroll
                for (int k = 0; k < kR; ++k)
#pragma unroll
                    for (int e = 0; e < V; ++e) v[k][i][e] = kMean ? (v[k][i][e] - mean2[k]) * rstd2[k] : v[k][i][e] * rstd2[k];
                if (a.pre_gain) {
                    load_parameter<S>(a.pre_gain, 0, a.packets, p, w);
#pragma unroll
                    for (int k = 0; k < kR; ++k)
#pragma unroll
                        for (int e = 0; e < V; ++e) v[k][i][e] *= w[e];
                }
                if (a.pre_bias) {
                    load_parameter<S>(a.pre_bias, 0, a.packets, p, w);
#pragma unroll
                    for (int k = 0; k < kR; ++k)
#pragma unroll
                        for (int e = 0; e < V; ++e) v[k][i][e] += w[e];
                }
#pragma unroll
                for (int k = 0; k < kR; ++k)
                    if (there[k]) store_packet<true>(static_cast<uint4*>(a.h) + (row + k) * a.packets + p, S::pack(v[k][i]));
            }
        }
        if (a.stats && lane == 0)
#pragma unroll
            for (int k = 0; k < kR; ++k)
                if (there[k]) a.stats[row + k] = make_float4(mean[k], rstd[k], mean2[k], rstd2[k]);
    }
}

// The same for rows off the 16-byte boundaries: packets of pieces, and a bit for each element that is inside the row.
template <class S, int kUnit, int kI, int kR, bool kWarp, bool kMean>
__global__ void __launch_bounds__(kWarp ? 128 : 256, kWarp ? 8 : kI == 4 ? 3 : 2) norm_forward_odd_kernel(const __grid_constant__ NormForwardArgs a)
{
    constexpr int V = S::kVec;
    __shared__ float buf[2][kR][32];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const uint32_t lane = kWarp ? threadIdx.x & 31 : threadIdx.x, width = kWarp ? 32 : blockDim.x;
    const size_t per_cta = kWarp ? blockDim.x >> 5 : 1;
    RowSum<kR, kWarp> sum{buf, 0};
    const RowColumns<S, kUnit> at{lane, width, a.cols};
    uint32_t on[kI];
#pragma unroll
    for (int i = 0; i < kI; ++i) on[i] = at.mask(i);
    auto parameter = [&](const void* base, size_t row, int i, float (&w)[V]) { S::unpack(at.load(base, row, i), w); };
    for (size_t turn = blockIdx.x * per_cta + (kWarp ? threadIdx.x >> 5 : 0); turn * kR < a.rows; turn += gridDim.x * per_cta) {
        const size_t row = turn * kR;
        uint4 ru[kR][kI], rr[kR][kI];
        bool there[kR];
#pragma unroll
        for (int k = 0; k < kR; ++k) there[k] = k == 0 || row + k < a.rows;
#pragma unroll
        for (int i = 0; i < kI; ++i)
#pragma unroll
            for (int k = 0; k < kR; ++k) {
                ru[k][i] = rr[k][i] = make_uint4(0, 0, 0, 0);
                if (there[k]) {
                    ru[k][i] = at.load(a.u, row + k, i);
                    if (a.r) rr[k][i] = at.load(a.r, row + k, i);
                }
            }
        float v[kR][kI][V], mean[kR], rstd[kR], mean2[kR], rstd2[kR];
#pragma unroll
        for (int k = 0; k < kR; ++k) {
            mean[k] = rstd[k] = mean2[k] = rstd2[k] = 0.0f;
#pragma unroll
            for (int i = 0; i < kI; ++i) S::unpack(ru[k][i], v[k][i]);
        }
        if (a.post != kNormNone) row_statistics<V, kUnit, kR, kI, kWarp, kMean>(v, on, a.post, a.inv_cols, a.eps, sum, mean, rstd);
        size_t gate_row[kR];
#pragma unroll
        for (int k = 0; k < kR; ++k) gate_row[k] = a.gate ? gate_row_of(row + k, a.rows_per_gate) : 0;
#pragma unroll
        for (int i = 0; i < kI; ++i) {
            if (!on[i]) continue;
            float w[V];
            if (a.post != kNormNone) {
#pragma unroll
                for (int k = 0; k < kR; ++k)
#pragma unroll
                    for (int e = 0; e < V; ++e) v[k][i][e] = kMean ? (v[k][i][e] - mean[k]) * rstd[k] : v[k][i][e] * rstd[k];
                if (a.post_gain) {
                    parameter(a.post_gain, 0, i, w);
#pragma unroll
                    for (int k = 0; k < kR; ++k)
#pragma unroll
                        for (int e = 0; e < V; ++e) v[k][i][e] *= w[e];
                }
                if (a.post_bias) {
                    parameter(a.post_bias, 0, i, w);
#pragma unroll
                    for (int k = 0; k < kR; ++k)
#pragma unroll
                        for (int e = 0; e < V; ++e) v[k][i][e] += w[e];
                }
            }
            if (a.gate) {
#pragma unroll
                for (int k = 0; k < kR; ++k) {
                    if (k > 0 && !there[k]) continue;
                    if (k == 0 || gate_row[k] != gate_row[0]) parameter(a.gate, gate_row[k], i, w);
#pragma unroll
                    for (int e = 0; e < V; ++e) v[k][i][e] *= w[e];
                }
            }
#pragma unroll
            for (int k = 0; k < kR; ++k) {
                if (a.r) {
                    S::unpack(rr[k][i], w);
#pragma unroll
                    for (int e = 0; e < V; ++e) v[k][i][e] = fmaf(a.alpha, w[e], v[k][i][e]);
                }
                if (kMean && kUnit < V)                              // columns past the row hold nothing for the next mean
#pragma unroll
                    for (int e = 0; e < V; ++e)
                        if (!(on[i] >> e & 1)) v[k][i][e] = 0.0f;
                if (a.s && there[k]) at.store(a.s, row + k, i, S::pack(v[k][i]));
            }
        }
        if (a.pre != kNormNone) {
            row_statistics<V, kUnit, kR, kI, kWarp, kMean>(v, on, a.pre, a.inv_cols, a.eps, sum, mean2, rstd2);
#pragma unroll
            for (int i = 0; i < kI; ++i) {
                if (!on[i]) continue;
                float w[V];
#pragma unroll
                for (int k = 0; k < kR; ++k)
#pragma unroll
                    for (int e = 0; e < V; ++e) v[k][i][e] = kMean ? (v[k][i][e] - mean2[k]) * rstd2[k] : v[k][i][e] * rstd2[k];
                if (a.pre_gain) {
                    parameter(a.pre_gain, 0, i, w);
#pragma unroll
                    for (int k = 0; k < kR; ++k)
#pragma unroll
                        for (int e = 0; e < V; ++e) v[k][i][e] *= w[e];
                }
                if (a.pre_bias) {
                    parameter(a.pre_bias, 0, i, w);
#pragma unroll
                    for (int k = 0; k < kR; ++k)
#pragma unroll
                        for (int e = 0; e < V; ++e) v[k][i][e] += w[e];
                }
#pragma unroll
                for (int k = 0; k < kR; ++k)
                    if (there[k]) at.store(a.h, row + k, i, S::pack(v[k][i]));
            }
        }
        if (a.stats && lane == 0)
#pragma unroll
            for (int k = 0; k < kR; ++k)
                if (there[k]) a.stats[row + k] = make_float4(mean[k], rstd[k], mean2[k], rstd2[k]);
    }
}

inline void norm_launch_config(cudaLaunchConfig_t* cfg, cudaLaunchAttribute* attr, size_t grid, unsigned block, cudaStream_t st)
{
    *cfg = cudaLaunchConfig_t{};
    cfg->gridDim = dim3((unsigned)(grid < 0x7fffffffu ? grid : 0x7fffffffu));
    cfg->blockDim = dim3(block);
    cfg->stream = st;
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg->attrs = attr;
    cfg->numAttrs = 1;
}

constexpr int kNormMaxStages = 8;
constexpr int kNormRingBytes = 200 * 1024;          // of an SM's shared memory, over its resident CTAs

static __device__ unsigned g_norm_faults;           // CTAs whose wait ran out

// Element access of the any-shape kernels.
template <class S> __device__ __forceinline__ float at(const void* base, size_t i) { return S::load1(static_cast<const typename S::elem*>(base) + i); }
template <class S> __device__ __forceinline__ void put(void* base, size_t i, float v) { S::store1(static_cast<typename S::elem*>(base) + i, v); }

// Any cols, any element-aligned pointers, rows too long for registers: a CTA sweeps its row once per statistic (from
// L1 or L2 after the first sweep) and once to write.  Every element is read before its place is written, by one thread.
template <class S>
__global__ void __launch_bounds__(kBlock) norm_forward_any_kernel(const __grid_constant__ NormForwardArgs a)
{
    __shared__ float buf[2][1][32];
    RowSum<1, false> sum{buf, 0};
    for (size_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const size_t base = row * a.cols, gate = a.gate ? gate_row_of(row, a.rows_per_gate) * a.cols : 0;
        float4 st = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        auto stream = [&](uint32_t c) {                              // s of one element, from u, r and u's statistics
            float v = at<S>(a.u, base + c);
            if (a.post != kNormNone) {
                v = (v - st.x) * st.y;
                if (a.post_gain) v *= at<S>(a.post_gain, c);
                if (a.post_bias) v += at<S>(a.post_bias, c);
            }
            if (a.gate) v *= at<S>(a.gate, gate + c);
            return a.r ? fmaf(a.alpha, at<S>(a.r, base + c), v) : v;
        };
        auto statistics = [&](auto value, int kind, float* mean, float* rstd) {
            float t[1] = {0.0f}, m = 0.0f;
            if (kind == kNormLayer) {
                for (uint32_t c = threadIdx.x; c < a.cols; c += kBlock) t[0] += value(c);
                sum(t);
                m = t[0] * a.inv_cols;
            }
            t[0] = 0.0f;
            for (uint32_t c = threadIdx.x; c < a.cols; c += kBlock) {
                const float d = value(c) - m;
                t[0] = fmaf(d, d, t[0]);
            }
            sum(t);
            *mean = m;
            *rstd = reciprocal_root(fmaf(t[0], a.inv_cols, a.eps));
        };
        if (a.post != kNormNone) {
            float m, q;
            statistics([&](uint32_t c) { return at<S>(a.u, base + c); }, a.post, &m, &q);
            st.x = m; st.y = q;
        }
        if (a.pre != kNormNone) {
            float m, q;
            statistics(stream, a.pre, &m, &q);
            st.z = m; st.w = q;
        }
        for (uint32_t c = threadIdx.x; c < a.cols; c += kBlock) {
            const float v = stream(c);
            if (a.pre != kNormNone) {
                float n = (v - st.z) * st.w;
                if (a.pre_gain) n *= at<S>(a.pre_gain, c);
                if (a.pre_bias) n += at<S>(a.pre_bias, c);
                if (a.s) put<S>(a.s, base + c, v);
                put<S>(a.h, base + c, n);
            } else if (a.s) {
                put<S>(a.s, base + c, v);
            }
        }
        if (a.stats && threadIdx.x == 0) a.stats[row] = st;
    }
}

template <class S> inline bool norm_vector_ok(const void* const* p, int n, size_t cols)
{
    if (cols % S::kVec) return false;
    for (int i = 0; i < n; ++i)
        if (reinterpret_cast<uintptr_t>(p[i]) & 15u) return false;   // a null pointer passes
    return true;
}

// kUnit == V: aligned rows
template <class S, int kUnit, int kI, int kR, bool kWarp, bool kMean> cudaError_t launch_norm_forward_kernel(const NormForwardArgs& a, cudaStream_t st)
{
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute attr[1];
    const size_t rows = kWarp ? 4 * kR : kR;         // of a CTA
    const unsigned block = kWarp ? 128 : ((a.packets + kI - 1) / kI + 31) / 32 * 32;
    norm_launch_config(&cfg, attr, (a.rows + rows - 1) / rows, block, st);
    if constexpr (kUnit == S::kVec) return cudaLaunchKernelEx(&cfg, norm_forward_kernel<S, kI, kR, kWarp, kMean>, a);
    else return cudaLaunchKernelEx(&cfg, norm_forward_odd_kernel<S, kUnit, kI, kR, kWarp, kMean>, a);
}

// Packets a thread holds, and rows.  Few threads with much each: a row's reductions are shared by fewer warps, and its
// parameters by more of the work.  bf16, us, against one packet of two rows a thread: [16384, 4096] RMS pair 87 (113), LayerNorm pair
// by four packets 110 (141), [32768, 2048] 86 (102), [8192, 8192] by four 99 (112), [4096, 16384] by eight 105 (131 swept several times).
// LayerNorm pairs from 256 packets on by four of one row, against two of two rows: [6000, 2560] f16 30.4 (32.0), [16384, 2560] 75.3 (79.8),
// [16384, 4096] 105.6 (112.4), fp32 [16384, 1024] 48.2 (45.7) and [16384, 2048] 86 (85); with 2048 columns the threshold itself: 56.1 (57.1).
// A warp per row below 65 packets: [65536, 512] LayerNorm pair 49 (52 by a CTA).  Fewer rows than SMs are a matter of latency: one
// packet of one row, against two of two: three rows of 4096 2.8 (4.0), 148 of them 3.0 (4.1), their LayerNorm pair 3.5 (5.7).
template <class S, bool kMean> cudaError_t launch_norm_forward_rows(const NormForwardArgs& a, int sms, cudaStream_t st)
{
    constexpr int V = S::kVec;
    if (a.packets <= 32) return launch_norm_forward_kernel<S, V, 1, 2, true, kMean>(a, st);
    if (a.packets <= 64) return launch_norm_forward_kernel<S, V, 2, 1, true, kMean>(a, st);
    if (a.packets <= 512 && a.rows <= size_t(sms)) return launch_norm_forward_kernel<S, V, 1, 1, false, kMean>(a, st);
    if (a.packets <= (kMean ? 255 : 512)) return launch_norm_forward_kernel<S, V, 2, 2, false, kMean>(a, st);
    if (a.packets <= 1024) return launch_norm_forward_kernel<S, V, 4, 1, false, kMean>(a, st);
    return launch_norm_forward_kernel<S, V, 8, 1, false, kMean>(a, st);
}

// Rows off the 16-byte boundaries, in pieces of 4 bytes where they begin on those (an even number of 16-bit columns), else element
// by element.  bf16, us, against a CTA that sweeps its row from memory for each statistic: [14808, 100] 6 (47), [4000, 1021] 30 (43),
// [8192, 4098] 95 (184), [8192, 4097] 191 (184), [5076, 14082] 375 (727).
template <class S, int kUnit, bool kMean> cudaError_t launch_norm_forward_odd(const NormForwardArgs& a, cudaStream_t st)
{
    if (a.packets <= 32) return launch_norm_forward_kernel<S, kUnit, 1, 2, true, kMean>(a, st);
    if (a.packets <= 1024) return launch_norm_forward_kernel<S, kUnit, 4, 1, false, kMean>(a, st);
    return launch_norm_forward_kernel<S, kUnit, 8, 1, false, kMean>(a, st);
}

template <class S>
cudaError_t launch_norm_forward(const NormForwardArgs& in, cudaStream_t st)
{
    NormForwardArgs a = in;
    if (a.rows == 0 || a.cols == 0) return cudaSuccess;
    const void* p[9] = {a.u, a.r, a.post_gain, a.post_bias, a.gate, a.pre_gain, a.pre_bias, a.s, a.h};
    a.packets = (a.cols + S::kVec - 1) / S::kVec;
    DeviceInfo di;
    cudaError_t e = device_info(&di);
    if (e != cudaSuccess) return e;
    // a row in registers, eight packets a thread at most
    if (a.packets > 2048) {
        const size_t cap = size_t(di.sm_count) * 8;
        norm_forward_any_kernel<S><<<(unsigned)(a.rows < cap ? a.rows : cap), kBlock, 0, st>>>(a);
        return cudaPeekAtLastError();
    }
    const bool mean = a.post == kNormLayer || a.pre == kNormLayer;
    if (norm_vector_ok<S>(p, 9, a.cols)) return mean ? launch_norm_forward_rows<S, true>(a, di.sm_count, st) : launch_norm_forward_rows<S, false>(a, di.sm_count, st);
    constexpr int kTwo = S::kVec == 8 ? 2 : 1;       // elements in 4 bytes
    uintptr_t low = 0;
    for (const void* q : p) low |= reinterpret_cast<uintptr_t>(q);
    if (kTwo == 2 && a.cols % 2 == 0 && low % 4 == 0) return mean ? launch_norm_forward_odd<S, kTwo, true>(a, st) : launch_norm_forward_odd<S, kTwo, false>(a, st);
    return mean ? launch_norm_forward_odd<S, 1, true>(a, st) : launch_norm_forward_odd<S, 1, false>(a, st);
}

// ---------------------------------------------------------------- backward

// A chunk's sum of ds a for one gate row: straight to the result when the chunk holds all of that gate row's rows, else to
// the chunk's slot 0 (the gate row that the chunk begins with) or 1 (a later one, which the chunk ends with).
__device__ __forceinline__ float* gate_target(const NormBackwardArgs& a, size_t chunk, size_t r0, size_t r1, size_t gate_row)
{
    const size_t g0 = gate_row * a.rows_per_gate, g1 = g0 + a.rows_per_gate;
    if (g0 >= r0 && g1 <= r1) return a.grad_gate + gate_row * a.cols;
    return a.partial + (size_t(a.chunks) * kNormSums + chunk * 2 + (g0 <= r0 ? 0 : 1)) * a.cols;
}

// Two neighbours at a time: Blackwell multiplies and adds two fp32 values in one instruction.  Worth 3 % here, where most of the work
// is multiply-adds (290 -> 283 us for [32768, 4096] bf16); the forward kernels lose by it (113 -> 120 us), as their pairs have to be
// brought together first.
template <class S> __device__ __forceinline__ void widen(const uint4& p, float2 (&v)[S::kVec / 2])
{
    float w[S::kVec];
    S::unpack(p, w);
#pragma unroll
    for (int e = 0; e < S::kVec / 2; ++e) v[e] = make_float2(w[2 * e], w[2 * e + 1]);
}
template <class S> __device__ __forceinline__ uint4 narrow(const float2 (&v)[S::kVec / 2])
{
    float w[S::kVec];
#pragma unroll
    for (int e = 0; e < S::kVec / 2; ++e) { w[2 * e] = v[e].x; w[2 * e + 1] = v[e].y; }
    return S::pack(w);
}
__device__ __forceinline__ float2 twice(float a) { return make_float2(a, a); }
using hw::add2;
using hw::fma2;
using hw::mul2;

// (x - mean) rstd
template <bool kMean, int P> __device__ __forceinline__ void normalise(float2 (&v)[P], float mean, float rstd)
{
    const float2 m = twice(-mean), r = twice(rstd);
#pragma unroll
    for (int e = 0; e < P; ++e) v[e] = mul2(kMean ? add2(v[e], m) : v[e], r);
}

// Rows travel through a ring in shared memory: bulk copies of whole rows (and of their statistics), several rows ahead, so that
// reads are in flight during the two reductions that every row waits for.  Two rows go together where the registers allow:
// half the barriers, twice the independent work.  A thread owns the same columns of every row, and along a column the
// gains and the gate are constants, so the inner loop keeps few sums:
//   grad g_pre = sum dh s^;   P = sum ds u^, Q = sum ds over the rows of one gate row, from which at its end
//   grad gate = g_post P + b_post Q, grad g_post += gate P, grad b_post += gate Q.
// Measured on [32768, 4096] bf16, RMS norms and a gate (1.6 GB), graph replays: next row prefetched into registers 418 us, this ring
// 355 us, these sums 290 us, pairs of values in one instruction 283 us, with norm_reduce_kernel as it is now 276 us (calls between
// other kernels: 303 us).
// kI packets per thread, kR rows at a time; kGate: there is a gate; kFull: means and bias sums are kept too (without: RMS norms,
// no bias sums, and no post_bias in a gate's gradient that is asked for).  Aligned rows of up to 512 kI packets.  Dynamic shared
// memory: `stages` rows of the tensors that are there.
template <class S, int kI, int kR, bool kGate, bool kFull>
__global__ void __launch_bounds__(512) norm_backward_kernel(const __grid_constant__ NormBackwardArgs a, int stages)
{
    constexpr int P = S::kVec / 2, kSums = kFull ? 2 : 1;
    extern __shared__ __align__(128) unsigned char ring[];
    __shared__ float buf[2][kSums * kR][32];
    __shared__ uint64_t full[kNormMaxStages];
    __shared__ uint32_t gave_up_;
    volatile uint32_t* gave_up = &gave_up_;
    const uint32_t row_bytes = a.packets * 16;
    const bool pre = a.pre != kNormNone, post = a.post != kNormNone;
    const uint32_t at_gs = pre ? 2 * row_bytes : 0, at_u = at_gs + (a.grad_s ? row_bytes : 0), at_stats = at_u + (a.u ? row_bytes : 0);
    const uint32_t stage_bytes = at_stats + 16;
    if (threadIdx.x == 0) {
        gave_up_ = 0;
        for (int i = 0; i < stages; ++i) tc::barrier_init(tc::shared_address(&full[i]), 1);
        tc::barrier_init_done();
    }
    __syncthreads();
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    RowSum<kSums * kR, false> sum{buf, 0};
    const size_t r0 = blockIdx.x * a.chunk_rows, r1 = r0 + a.chunk_rows < a.rows ? r0 + a.chunk_rows : a.rows;
    if (r0 >= r1) return;
    auto request = [&](size_t row, int stage) {                       // by one thread
        const uint32_t bar = tc::shared_address(&full[stage]), dst = tc::shared_address(ring) + stage * stage_bytes;
        tc::barrier_expect(bar, stage_bytes);
        auto one = [&](const void* p, uint32_t at) { tc::load_run(dst + at, static_cast<const unsigned char*>(p) + row * row_bytes, row_bytes, bar); };
        if (pre) {
            one(a.grad_h, 0);
            one(a.s, row_bytes);
        }
        if (a.grad_s) one(a.grad_s, at_gs);
        if (a.u) one(a.u, at_u);
        tc::load_run(dst + at_stats, a.stats + row, 16, bar);
    };
    if (threadIdx.x == 0)
        for (int i = 0; i < stages && r0 + i < r1; ++i) request(r0 + i, i);

    uint32_t column[kI];
    bool on[kI];
#pragma unroll
    for (int i = 0; i < kI; ++i) {
        column[i] = threadIdx.x + i * blockDim.x;
        on[i] = column[i] < a.packets;
    }
    uint4 pre_gain[kI];
    float2 both[kI][P];                              // gate g_post
    float2 acc_pre[kI][P], acc_pre_bias[kFull ? kI : 1][P], acc_p[kI][P], acc_q[kFull ? kI : 1][P];
    float2 acc_post[kGate ? kI : 1][P], acc_post_bias[kGate && kFull ? kI : 1][P];
    size_t gate_row = kGate ? r0 / a.rows_per_gate : 0, gate_end = (gate_row + 1) * a.rows_per_gate;
    // a parameter's packet of this thread's columns; `none` when there is no such parameter
    auto parameter = [&](const void* base, size_t row, int i, float none, float2 (&v)[P]) {
        if (base && on[i]) {
            widen<S>(__ldg(static_cast<const uint4*>(base) + row * a.packets + column[i]), v);
        } else {
#pragma unroll
            for (int e = 0; e < P; ++e) v[e] = twice(none);
        }
    };
    auto set_both = [&]() {
#pragma unroll
        for (int i = 0; i < kI; ++i) {
            float2 w[P];
            parameter(post ? a.post_gain : nullptr, 0, i, 1.0f, both[i]);
            if (kGate) {
                parameter(a.gate, gate_row, i, 1.0f, w);
#pragma unroll
                for (int e = 0; e < P; ++e) both[i][e] = mul2(both[i][e], w[e]);
            }
            if (!on[i])                              // a mean taken from a column past the row would leave something there
#pragma unroll
                for (int e = 0; e < P; ++e) both[i][e] = twice(0.0f);
        }
    };
#pragma unroll
    for (int i = 0; i < kI; ++i) {
        pre_gain[i] = on[i] && a.pre_gain ? __ldg(static_cast<const uint4*>(a.pre_gain) + column[i]) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int e = 0; e < P; ++e) {
            acc_pre[i][e] = acc_p[i][e] = twice(0.0f);
            if (kFull) acc_pre_bias[i][e] = acc_q[i][e] = twice(0.0f);
            if (kGate) acc_post[i][e] = twice(0.0f);
            if (kGate && kFull) acc_post_bias[i][e] = twice(0.0f);
        }
    }
    set_both();
    // the end of a gate row's rows in this chunk
    auto hand_over_gate = [&]() {
#pragma unroll
        for (int i = 0; i < kI; ++i) {
            float2 gate[P], gain[P], bias[P];
            parameter(a.gate, gate_row, i, 0.0f, gate);
            parameter(post ? a.post_gain : nullptr, 0, i, 1.0f, gain);
            parameter(post ? a.post_bias : nullptr, 0, i, 0.0f, bias);
            // pairs where the place begins on eight bytes (by single floats throughout: 647 us for a gate row for each row of [32768, 4096] bf16, not
            // 617); the caller's tensor may begin on any float
            float* dst = on[i] && a.grad_gate ? gate_target(a, blockIdx.x, r0, r1, gate_row) + size_t(column[i]) * S::kVec : nullptr;
#pragma unroll
            for (int e = 0; e < P; ++e) {
                if (dst) {
                    const float2 v = kFull ? fma2(gain[e], acc_p[i][e], mul2(bias[e], acc_q[i][e])) : mul2(gain[e], acc_p[i][e]);
                    if (reinterpret_cast<uintptr_t>(dst) & 7u) {
                        dst[2 * e] = v.x;
                        dst[2 * e + 1] = v.y;
                    } else {
                        reinterpret_cast<float2*>(dst)[e] = v;
                    }
                }
                acc_post[i][e] = fma2(gate[e], acc_p[i][e], acc_post[i][e]);
                acc_p[i][e] = twice(0.0f);
                if constexpr (kFull) {
                    acc_post_bias[i][e] = fma2(gate[e], acc_q[i][e], acc_post_bias[i][e]);
                    acc_q[i][e] = twice(0.0f);
                }
            }
        }
    };

    int stage = 0;
    uint32_t phase = 0;
    bool ok = true;
    for (size_t row = r0; row < r1 && ok; row += kR) {
        float2 ds[kR][kI][P], hat[kR][kI][P], t2[kSums * kR];
        float t[kSums * kR];
        float4 st[kR];
        const bool two = kR == 1 || row + 1 < r1;
        const unsigned char* at[kR];
#pragma unroll
        for (int k = 0; k < kR; ++k) {                               // stages are a multiple of kR: no wrap inside
            if (k == 0 || two) tc::barrier_wait(tc::shared_address(&full[stage + k]), phase, gave_up);
            at[k] = ring + (stage + k) * stage_bytes;
            st[k] = k == 0 || two ? *reinterpret_cast<const float4*>(at[k] + at_stats) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        }
        // A thread whose wait ran out carries on to this row's last barrier, behind which all learn of it together.
        // Columns past the row and rows past the chunk read as zeros: they add nothing to any sum, and are not stored.
        auto in_ring = [&](int k, uint32_t tensor_at, int i) {
            return on[i] && (k == 0 || two) ? *reinterpret_cast<const uint4*>(at[k] + tensor_at + column[i] * 16) : make_uint4(0, 0, 0, 0);
        };
#pragma unroll
        for (int k = 0; k < kSums * kR; ++k) t2[k] = twice(0.0f);
        if (pre) {
            // d = dh g_pre and s^; their sums
#pragma unroll
            for (int i = 0; i < kI; ++i) {
                float2 w[P];
                widen<S>(pre_gain[i], w);
#pragma unroll
                for (int k = 0; k < kR; ++k) {
                    widen<S>(in_ring(k, 0, i), ds[k][i]);
                    widen<S>(in_ring(k, row_bytes, i), hat[k][i]);
                    normalise<kFull>(hat[k][i], st[k].z, st[k].w);
#pragma unroll
                    for (int e = 0; e < P; ++e) {
                        acc_pre[i][e] = fma2(ds[k][i][e], hat[k][i][e], acc_pre[i][e]);
                        if (kFull) acc_pre_bias[i][e] = add2(acc_pre_bias[i][e], ds[k][i][e]);
                        if (a.pre_gain) ds[k][i][e] = mul2(ds[k][i][e], w[e]);
                        t2[kSums * k] = fma2(ds[k][i][e], hat[k][i][e], t2[kSums * k]);
                        if (kFull) t2[kSums * k + 1] = add2(t2[kSums * k + 1], ds[k][i][e]);
                    }
                }
            }
#pragma unroll
            for (int k = 0; k < kSums * kR; ++k) t[k] = t2[k].x + t2[k].y;
            sum(t);
#pragma unroll
            for (int k = 0; k < kR; ++k) {
                const float2 q = twice(-t[kSums * k] * a.inv_cols), m = twice(kFull && a.pre == kNormLayer ? -t[kSums * k + 1] * a.inv_cols : 0.0f);
#pragma unroll
                for (int i = 0; i < kI; ++i) {
                    float2 v[P];
                    widen<S>(a.grad_s ? in_ring(k, at_gs, i) : make_uint4(0, 0, 0, 0), v);
#pragma unroll
                    for (int e = 0; e < P; ++e) {
                        const float2 c = fma2(hat[k][i][e], q, kFull ? add2(ds[k][i][e], m) : ds[k][i][e]);
                        ds[k][i][e] = fma2(twice(st[k].w), c, v[e]);
                    }
                }
            }
        } else {
#pragma unroll
            for (int k = 0; k < kR; ++k)
#pragma unroll
                for (int i = 0; i < kI; ++i) widen<S>(in_ring(k, at_gs, i), ds[k][i]);
        }
        // grad_r; then u^, P, Q and e = gate g_post ds, and the sums of the row
#pragma unroll
        for (int k = 0; k < kSums * kR; ++k) t2[k] = twice(0.0f);
#pragma unroll
        for (int k = 0; k < kR; ++k) {
            if (k > 0 && !two) break;
            if (kGate && row + k == gate_end) {
                hand_over_gate();
                ++gate_row;
                gate_end += a.rows_per_gate;
                set_both();
            }
#pragma unroll
            for (int i = 0; i < kI; ++i) {
                if (a.grad_r && on[i]) {
                    float2 v[P];
#pragma unroll
                    for (int e = 0; e < P; ++e) v[e] = mul2(twice(a.alpha), ds[k][i][e]);
                    store_packet<true>(static_cast<uint4*>(a.grad_r) + (row + k) * a.packets + column[i], narrow<S>(v));
                }
                if (post || kGate) {
                    widen<S>(in_ring(k, at_u, i), hat[k][i]);
                    if (post) normalise<kFull>(hat[k][i], st[k].x, st[k].y);
#pragma unroll
                    for (int e = 0; e < P; ++e) {
                        acc_p[i][e] = fma2(ds[k][i][e], hat[k][i][e], acc_p[i][e]);
                        if (kFull) acc_q[i][e] = add2(acc_q[i][e], ds[k][i][e]);
                        ds[k][i][e] = mul2(ds[k][i][e], both[i][e]);
                        t2[kSums * k] = fma2(ds[k][i][e], hat[k][i][e], t2[kSums * k]);
                        if (kFull) t2[kSums * k + 1] = add2(t2[kSums * k + 1], ds[k][i][e]);
                    }
                }
            }
        }
#pragma unroll
        for (int k = 0; k < kSums * kR; ++k) t[k] = t2[k].x + t2[k].y;
        if (post) sum(t);
        else __syncthreads();
        if (blockDim.x == 32) __syncwarp();
        ok = *gave_up == 0;
        // every thread has read the rows: their places in the ring are free
        if (threadIdx.x == 0 && ok) {
#pragma unroll
            for (int k = 0; k < kR; ++k)
                if (row + k + stages < r1) request(row + k + stages, stage + k);
        }
        stage += kR;
        if (stage >= stages) { stage = 0; phase ^= 1; }
#pragma unroll
        for (int k = 0; k < kR; ++k) {
            if (k > 0 && !two) break;
            const float2 q = twice(-t[kSums * k] * a.inv_cols), m = twice(kFull && a.post == kNormLayer ? -t[kSums * k + 1] * a.inv_cols : 0.0f);
#pragma unroll
            for (int i = 0; i < kI; ++i) {
                if (post)
#pragma unroll
                    for (int e = 0; e < P; ++e)
                        ds[k][i][e] = mul2(twice(st[k].y), fma2(hat[k][i][e], q, kFull ? add2(ds[k][i][e], m) : ds[k][i][e]));
                if (on[i]) store_packet<true>(static_cast<uint4*>(a.grad_u) + (row + k) * a.packets + column[i], narrow<S>(ds[k][i]));
            }
        }
    }
    if (!ok) {
        // copies in flight land before the CTA's memory goes away
        const long long t0 = clock64();
        while (clock64() - t0 < tc::kWaitDrain) {}
    }
    if constexpr (kGate) hand_over_gate();
#pragma unroll
    for (int i = 0; i < kI; ++i) {
        if (!on[i]) continue;
        const size_t col = size_t(column[i]) * S::kVec;
        auto keep = [&](int k, const float2 (&v)[P]) {
            if (!a.sums[k]) return;
            float4* dst = reinterpret_cast<float4*>(a.partial + (size_t(blockIdx.x) * kNormSums + k) * a.cols + col);
#pragma unroll
            for (int e = 0; e < P; e += 2) dst[e / 2] = make_float4(v[e].x, v[e].y, v[e + 1].x, v[e + 1].y);
        };
        keep(kSumPreGain, acc_pre[i]);
        if constexpr (kGate) keep(kSumPostGain, acc_post[i]);
        else keep(kSumPostGain, acc_p[i]);
        if constexpr (kFull) {
            keep(kSumPreBias, acc_pre_bias[i]);
            if constexpr (kGate) keep(kSumPostBias, acc_post_bias[i]);
            else keep(kSumPostBias, acc_q[i]);
        }
    }
    if (threadIdx.x == 0 && gave_up_) atomicAdd(&g_norm_faults, 1u);
}

// Any shape: two kernels.  A thread takes one column at a time, or a packet of them where rows are aligned (kVec: rows too long for
// registers).
template <class S, bool kVec> struct NormLanes {
    static constexpr int V = kVec ? S::kVec : 1;
    static __device__ __forceinline__ void load(const void* base, size_t i, float (&v)[V])
    {
        if constexpr (kVec) S::unpack(*reinterpret_cast<const uint4*>(static_cast<const typename S::elem*>(base) + i), v);
        else v[0] = at<S>(base, i);
    }
    static __device__ __forceinline__ void store(void* base, size_t i, const float (&v)[V])
    {
        if constexpr (kVec) *reinterpret_cast<uint4*>(static_cast<typename S::elem*>(base) + i) = S::pack(v);
        else put<S>(base, i, v[0]);
    }
    // everything of these columns up to da, from the row's statistics and (for ds) its first two means
    float d[V], shat[V], ds[V], uhat[V], a[V], da[V], gain[V];
    __device__ __forceinline__ void read(const NormBackwardArgs& g, size_t base, size_t gate, size_t c, float4 st, float m, float q)
    {
        float w[V];
#pragma unroll
        for (int e = 0; e < V; ++e) d[e] = shat[e] = ds[e] = uhat[e] = 0.0f, gain[e] = 1.0f;
        if (g.grad_s) load(g.grad_s, base + c, ds);
        if (g.pre != kNormNone) {
            load(g.grad_h, base + c, d);
            load(g.s, base + c, shat);
#pragma unroll
            for (int e = 0; e < V; ++e) w[e] = 1.0f;
            if (g.pre_gain) load(g.pre_gain, c, w);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                shat[e] = (shat[e] - st.z) * st.w;
                ds[e] = fmaf(st.w, d[e] * w[e] - m - shat[e] * q, ds[e]);
            }
        }
        if (g.u) load(g.u, base + c, uhat);
        if (g.post != kNormNone) {
#pragma unroll
            for (int e = 0; e < V; ++e) uhat[e] = (uhat[e] - st.x) * st.y;
            if (g.post_gain) load(g.post_gain, c, gain);
        }
#pragma unroll
        for (int e = 0; e < V; ++e) {
            a[e] = uhat[e] * gain[e];
            da[e] = ds[e];
        }
        if (g.gate) {
            if (g.post != kNormNone && g.post_bias) {
                load(g.post_bias, c, w);
#pragma unroll
                for (int e = 0; e < V; ++e) a[e] += w[e];
            }
            load(g.gate, gate + c, w);
#pragma unroll
            for (int e = 0; e < V; ++e) da[e] *= w[e];
        }
    }
};

// First kernel: the four row means that the gradients need, (mean d, mean d s^, mean e, mean e u^).
template <class S, bool kVec>
__global__ void __launch_bounds__(kBlock) norm_backward_means_kernel(const __grid_constant__ NormBackwardArgs a)
{
    using L = NormLanes<S, kVec>;
    constexpr int V = L::V;
    __shared__ float buf[2][2][32];
    RowSum<2, false> sum{buf, 0};
    for (size_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const size_t base = row * a.cols, gate = a.gate ? gate_row_of(row, a.rows_per_gate) * a.cols : 0;
        const float4 st = a.stats[row];
        float t[2] = {0.0f, 0.0f};
        float4 out = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (a.pre != kNormNone) {
            for (size_t c = threadIdx.x * V; c < a.cols; c += kBlock * V) {
                float d[V], x[V], w[V];
                L::load(a.grad_h, base + c, d);
                L::load(a.s, base + c, x);
#pragma unroll
                for (int e = 0; e < V; ++e) w[e] = 1.0f;
                if (a.pre_gain) L::load(a.pre_gain, c, w);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    d[e] *= w[e];
                    t[0] += d[e];
                    t[1] = fmaf(d[e], (x[e] - st.z) * st.w, t[1]);
                }
            }
            sum(t);
            out.x = a.pre == kNormLayer ? t[0] * a.inv_cols : 0.0f;
            out.y = t[1] * a.inv_cols;
        }
        if (a.post != kNormNone) {
            t[0] = t[1] = 0.0f;
            for (size_t c = threadIdx.x * V; c < a.cols; c += kBlock * V) {
                L x;
                x.read(a, base, gate, c, st, out.x, out.y);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float v = x.da[e] * x.gain[e];
                    t[0] += v;
                    t[1] = fmaf(v, x.uhat[e], t[1]);
                }
            }
            sum(t);
            out.z = a.post == kNormLayer ? t[0] * a.inv_cols : 0.0f;
            out.w = t[1] * a.inv_cols;
        }
        if (threadIdx.x == 0) a.row_means[row] = out;
    }
}

// Second kernel: a thread owns its columns of a chunk of rows, writes the two gradients and its columns' sums.
template <class S, bool kVec>
__global__ void __launch_bounds__(kBlock) norm_backward_columns_kernel(const __grid_constant__ NormBackwardArgs a)
{
    using L = NormLanes<S, kVec>;
    constexpr int V = L::V;
    const size_t c = (size_t(blockIdx.x) * kBlock + threadIdx.x) * V;
    if (c >= a.cols) return;
    const size_t r0 = blockIdx.y * a.chunk_rows, r1 = r0 + a.chunk_rows < a.rows ? r0 + a.chunk_rows : a.rows;
    if (r0 >= r1) return;
    float acc[kNormSums][V], accg[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
#pragma unroll
        for (int k = 0; k < kNormSums; ++k) acc[k][e] = 0.0f;
        accg[e] = 0.0f;
    }
    size_t gate_row = a.gate ? r0 / a.rows_per_gate : 0, gate_end = (gate_row + 1) * a.rows_per_gate;
    auto hand_over_gate = [&]() {
        float* dst = a.grad_gate ? gate_target(a, blockIdx.y, r0, r1, gate_row) + c : nullptr;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            if (dst) dst[e] = accg[e];
            accg[e] = 0.0f;
        }
    };
    for (size_t row = r0; row < r1; ++row) {
        if (a.gate && row == gate_end) {
            hand_over_gate();
            ++gate_row;
            gate_end += a.rows_per_gate;
        }
        const float4 st = __ldg(a.stats + row), mean = a.row_means[row];
        const size_t base = row * a.cols;
        L x;
        x.read(a, base, gate_row * a.cols, c, st, mean.x, mean.y);
        float gr[V], gu[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
            acc[kSumPreGain][e] = fmaf(x.d[e], x.shat[e], acc[kSumPreGain][e]);
            acc[kSumPreBias][e] += x.d[e];
            acc[kSumPostGain][e] = fmaf(x.da[e], x.uhat[e], acc[kSumPostGain][e]);
            acc[kSumPostBias][e] += x.da[e];
            accg[e] = fmaf(x.ds[e], x.a[e], accg[e]);
            gr[e] = a.alpha * x.ds[e];
            gu[e] = a.post != kNormNone ? st.y * (x.da[e] * x.gain[e] - mean.z - x.uhat[e] * mean.w) : x.da[e];
        }
        if (a.grad_r) L::store(a.grad_r, base + c, gr);
        L::store(a.grad_u, base + c, gu);
    }
#pragma unroll
    for (int k = 0; k < kNormSums; ++k)
        if (a.sums[k])
#pragma unroll
            for (int e = 0; e < V; ++e) a.partial[(size_t(blockIdx.y) * kNormSums + k) * a.cols + c + e] = acc[k][e];
    if (a.gate) hand_over_gate();
}

template <class S, bool kVec> cudaError_t launch_norm_backward_any(const NormBackwardArgs& a, int sms, cudaStream_t st)
{
    const size_t cap = size_t(sms) * 8, lanes = size_t(kBlock) * NormLanes<S, kVec>::V;
    norm_backward_means_kernel<S, kVec><<<(unsigned)(a.rows < cap ? a.rows : cap), kBlock, 0, st>>>(a);
    cudaError_t e = cudaPeekAtLastError();
    if (e != cudaSuccess) return e;
    norm_backward_columns_kernel<S, kVec><<<dim3(unsigned((a.cols + lanes - 1) / lanes), a.chunks), kBlock, 0, st>>>(a);
    return cudaPeekAtLastError();
}

// Adds the chunks' sums: blockIdx.y < kNormSums one of the parameters', beyond that a gate row's.  32 columns times kNormGroups
// runs of consecutive chunks, each run summed in order by one thread (eight loads in flight), the runs' sums then in order: the
// same bits every time.  (32 runs of a load at a time: 16 us for 147 chunks of 4096 columns.)
constexpr int kNormGroups = 8;
static __global__ void __launch_bounds__(32 * kNormGroups) norm_reduce_kernel(const __grid_constant__ NormBackwardArgs a)
{
    __shared__ float smem[kNormGroups][32];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int lane = threadIdx.x & 31, group = threadIdx.x >> 5;
    const size_t col = size_t(blockIdx.x) * 32 + lane;
    const size_t gate_rows = a.grad_gate && a.rows_per_gate > 1 ? a.rows / a.rows_per_gate : 0;          // as the launch counts them
    for (size_t job = blockIdx.y; job < kNormSums + gate_rows; job += gridDim.y) {
        const bool gate = job >= kNormSums;
        float* out = gate ? a.grad_gate + (job - kNormSums) * a.cols : a.sums[job];
        size_t c0 = 0, c1 = a.chunks, g0 = 0;
        if (gate) {
            g0 = (job - kNormSums) * a.rows_per_gate;
            c0 = g0 / a.chunk_rows;
            c1 = (g0 + a.rows_per_gate - 1) / a.chunk_rows + 1;
            if (c1 - c0 == 1) continue;                              // written by its chunk
        } else if (!out) {
            continue;
        }
        // a parameter's sums are a row of partial for each chunk; a gate row's are one of two, by where it begins
        const float* base = a.partial + (gate ? size_t(a.chunks) * kNormSums : job) * a.cols + col;
        const size_t step = size_t(gate ? 2 : kNormSums) * a.cols;
        const size_t per = (c1 - c0 + kNormGroups - 1) / kNormGroups;
        const size_t k0 = c0 + group * per, k1 = k0 + per < c1 ? k0 + per : c1;
        float s = 0.0f;
        if (col < a.cols)
            for (size_t k = k0; k < k1; k += 8) {
                float v[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const size_t second = gate && g0 > (k + j) * a.chunk_rows ? a.cols : 0;
                    v[j] = k + j < k1 ? base[(k + j) * step + second] : 0.0f;
                }
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (k + j < k1) s += v[j];
            }
        smem[group][lane] = s;
        __syncthreads();
        if (group == 0 && col < a.cols) {
            float t = smem[0][lane];
#pragma unroll
            for (int j = 1; j < kNormGroups; ++j) t += smem[j][lane];
            out[col] = t;
        }
        __syncthreads();
    }
}

// How the rows are cut: by shape, type and device alone, so that a call's scratch can be asked for beforehand.
struct NormPlan { unsigned block; int packets_per_thread; size_t chunk_rows; uint32_t chunks; };

template <class S> inline NormPlan norm_plan(size_t rows, size_t cols, int sm_count)
{
    NormPlan p;
    const size_t packets = (cols + S::kVec - 1) / S::kVec;
    p.packets_per_thread = packets <= 512 ? 1 : 2;
    size_t block = ((packets + p.packets_per_thread - 1) / p.packets_per_thread + 31) / 32 * 32;
    p.block = unsigned(block < 512 ? block : 512);
    // CTAs that stay, one per 512 threads of an SM; rows longer than their registers go by strips of columns, several to a chunk
    const size_t target = size_t(sm_count) * (packets <= 1024 ? 512 / p.block : 1);
    size_t chunks = rows < target ? rows : target;
    if (chunks == 0) chunks = 1;
    p.chunk_rows = (rows + chunks - 1) / chunks;
    if (p.chunk_rows == 0) p.chunk_rows = 1;
    p.chunks = uint32_t((rows + p.chunk_rows - 1) / p.chunk_rows);
    if (p.chunks == 0) p.chunks = 1;
    return p;
}

template <class S> inline size_t norm_backward_scratch_bytes(size_t rows, size_t cols, int sm_count)
{
    const NormPlan p = norm_plan<S>(rows, cols, sm_count);
    return rows * sizeof(float4) + size_t(p.chunks) * (kNormSums + 2) * cols * sizeof(float);
}

template <class S, int kI, int kR, bool kGate, bool kFull>
cudaError_t launch_norm_backward_kernel(const NormBackwardArgs& a, const NormPlan& p, cudaStream_t st)
{
    auto kernel = norm_backward_kernel<S, kI, kR, kGate, kFull>;
    const size_t row = size_t(a.packets) * 16 * ((a.pre != kNormNone ? 2 : 0) + (a.grad_s != nullptr) + (a.u != nullptr)) + 16;
    size_t stages = kNormRingBytes / (512 / p.block) / row;
    if (stages > kNormMaxStages) stages = kNormMaxStages;
    stages -= stages % kR;                           // rows are taken kR at a time (at least two turns: see the rule below)
    // the same limit whatever the call: one that followed the shape could be lowered by another host thread before this launch
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kNormRingBytes);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute attr[1];
    norm_launch_config(&cfg, attr, p.chunks, p.block, st);
    cfg.dynamicSmemBytes = stages * row;
    return cudaLaunchKernelEx(&cfg, kernel, a, int(stages));
}

template <class S, int kI, int kR> cudaError_t launch_norm_backward_rows(const NormBackwardArgs& a, const NormPlan& p, cudaStream_t st)
{
    // (the gate's gradient holds post_bias times the sum of ds, whether or not post_bias has a gradient of its own)
    const bool more = a.sums[kSumPreBias] || a.sums[kSumPostBias] || (a.grad_gate && a.post_bias) || a.pre == kNormLayer || a.post == kNormLayer;
    // six sums for each column beside two rows spill (310 us for a LayerNorm pair with a gate on [16384, 4096] bf16): one row then
    if (a.gate) return more ? launch_norm_backward_kernel<S, kI, 1, true, true>(a, p, st) : launch_norm_backward_kernel<S, kI, kR, true, false>(a, p, st);
    return more ? launch_norm_backward_kernel<S, kI, kR, false, true>(a, p, st) : launch_norm_backward_kernel<S, kI, kR, false, false>(a, p, st);
}

template <class S>
cudaError_t launch_norm_backward(const NormBackwardArgs& in, void* scratch, cudaStream_t st)
{
    NormBackwardArgs a = in;
    DeviceInfo di;
    cudaError_t e = device_info(&di);
    if (e != cudaSuccess) return e;
    if (a.cols == 0) return cudaSuccess;
    if (a.rows == 0) {
        for (int k = 0; k < kNormSums; ++k)
            if (a.sums[k] && (e = cudaMemsetAsync(a.sums[k], 0, a.cols * sizeof(float), st)) != cudaSuccess) return e;
        return cudaSuccess;
    }
    const NormPlan p = norm_plan<S>(a.rows, a.cols, di.sm_count);
    a.row_means = static_cast<float4*>(scratch);
    a.partial = reinterpret_cast<float*>(a.row_means + a.rows);
    a.chunk_rows = p.chunk_rows;
    a.chunks = p.chunks;
    a.packets = a.cols / S::kVec;
    const void* ptr[10] = {a.grad_h, a.grad_s, a.u, a.s, a.post_gain, a.post_bias, a.gate, a.pre_gain, a.grad_u, a.grad_r};
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute attr[1];
    // the row in registers, two packets a thread at most (beside the sums of a gate and means two already spill 280 bytes a thread for
    // bf16 and 460 for f16: [4096, 6144] f16, LayerNorm pair, 124 us)
    const bool vec = norm_vector_ok<S>(ptr, 10, a.cols);
    if (vec && a.packets <= 512) e = launch_norm_backward_rows<S, 1, 2>(a, p, st);
    else if (vec && a.packets <= 1024) e = launch_norm_backward_rows<S, 2, 1>(a, p, st);
    else e = vec ? launch_norm_backward_any<S, true>(a, di.sm_count, st) : launch_norm_backward_any<S, false>(a, di.sm_count, st);
    if (e != cudaSuccess) return e;
    const size_t gate_rows = a.grad_gate && a.rows_per_gate > 1 ? a.rows / a.rows_per_gate : 0;
    bool any = gate_rows > 0;
    for (int k = 0; k < kNormSums; ++k) any = any || a.sums[k];
    if (!any) return cudaSuccess;
    const size_t jobs = kNormSums + gate_rows;
    norm_launch_config(&cfg, attr, (a.cols + 31) / 32, 32 * kNormGroups, st);
    cfg.gridDim.y = (unsigned)(jobs < 65535 ? jobs : 65535);
    return cudaLaunchKernelEx(&cfg, norm_reduce_kernel, a);
}

}  // namespace nfad
