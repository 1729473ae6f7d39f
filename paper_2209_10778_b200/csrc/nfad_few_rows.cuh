// nfad_few_rows.cuh -- the forward products when there are few rows: single tokens, small decoding batches.
//
// Then the weights' bytes are what takes the time, and each weight is used a handful of times: what matters is that every SM
// has plenty of long contiguous reads of them in flight.  A CTA takes 16 outputs; its eight warps split the reduction, each
// reading 256 contiguous bytes of each of the 16 weight rows at once, straight into registers.  There they are the A
// operand of a small matrix instruction (16 outputs x 8 tokens), whose reduction slots are permuted so that a lane's 16 bytes
// are its own fragments: no shared memory and no shuffles between memory and the products.  The tokens' fragments are
// read the same way (they come from L1 or L2).  The warps' sums meet in shared memory, and bias, scales and activation follow.
// Bound by HBM: 24 rows over 64 experts, 2048 -> 1408, bf16 (about 20 experts' weights, 115 MB) 24 us, 0.75 of the copy rate with
// the launch in it.  Four 64-byte steps in flight per warp and four CTAs to an SM, three beside block scales or for 16 tokens at once; eight
// steps and two CTAs took 34 us.
#pragma once

#include "nfad_product.cuh"

namespace nfad {

constexpr int kFewWarps = 8;
constexpr int kFewOutputs = 16;
constexpr int kFewSteps = 4;                        // of 64 bytes of each row: what a warp has in flight
constexpr int kFewMaxRows = 256;

// d += a b of four 8-bit floating-point values each, as two pairs of halves, which hold them exactly.  (The instruction for 8-bit operands itself
// spills 172 bytes a thread and took 46 us for one token, 4096 -> 2 x 14336, where this takes 28.)
__device__ __forceinline__ void few_product_e4m3(float (&f)[4], uint32_t lo, uint32_t hi, uint32_t x)
{
    asm volatile("{\n .reg .b16 l, h;\n .reg .b32 a0, a1, a2, a3, b0, b1;\n"
        " mov.b32 {l, h}, %4;\n cvt.rn.f16x2.e4m3x2 a0, l;\n cvt.rn.f16x2.e4m3x2 a2, h;\n"
        " mov.b32 {l, h}, %5;\n cvt.rn.f16x2.e4m3x2 a1, l;\n cvt.rn.f16x2.e4m3x2 a3, h;\n"
        " mov.b32 {l, h}, %6;\n cvt.rn.f16x2.e4m3x2 b0, l;\n cvt.rn.f16x2.e4m3x2 b1, h;\n"
        " mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {a0, a1, a2, a3}, {b0, b1}, {%0, %1, %2, %3};\n}"
        : "+f"(f[0]), "+f"(f[1]), "+f"(f[2]), "+f"(f[3]) : "r"(lo), "r"(hi), "r"(x));
}

// d += a b: 16 outputs x 8 tokens, 32 bytes of the reduction
template <int kNumber> __device__ __forceinline__ void few_product(uint32_t (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    if (kNumber == tc::kNumberS8) {
        asm("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    } else {
        float f[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(d[i]);
        if (kNumber == tc::kNumberE4M3) {
            few_product_e4m3(f, a0, a1, b0);
            few_product_e4m3(f, a2, a3, b1);
        } else if (kNumber == tc::kNumberBF16)
            asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                : "+f"(f[0]), "+f"(f[1]), "+f"(f[2]), "+f"(f[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
        else
            asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                : "+f"(f[0]), "+f"(f[1]), "+f"(f[2]), "+f"(f[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
#pragma unroll
        for (int i = 0; i < 4; ++i) d[i] = __float_as_uint(f[i]);
    }
}

__device__ __forceinline__ void act1(int kind, float z, float* y, float* d)
{
    ActOut o = {z, 1.0f};
    switch (kind) {
    case kGeluErf:  o = evaluate(GeluErf{}, Fast{}, z); break;
    case kGeluTanh: o = evaluate(GeluTanh{}, Fast{}, z); break;
    case kSwish:    o = evaluate(Swish{}, Fast{}, z); break;
    case kMish:     o = evaluate(Mish{}, Fast{}, z); break;
    default: break;
    }
    *y = o.y;
    *d = o.dydx;
}

// Of operands with block scales a warp's block of 256 bytes is two scaled blocks: each one's products start from zero and are added with
// their scale.
// OP: kProdForward, kProdBytes (8-bit integers, one expert), kProdScaled or a gated one, whose CTA takes eight outputs of each of the two weights: the
// lower and the upper half of the instruction's 16 rows.  early: the weights may be read before the kernel in front has ended
// (it is the quantiser of the same call, which starts this one only after everything before it is complete).
template <int OP, int NT> struct FewResident { static constexpr int value = NT == 1 && !ProdKind<OP>::kScaled ? 4 : 3; };     // CTAs to an SM (scaled: two conversions a word, 80 registers)
template <int OP, class S, int NT>
__global__ void __launch_bounds__(kFewWarps * 32, FewResident<OP, NT>::value) few_rows_kernel(const __grid_constant__ ProdArgs g, int early)
{
    constexpr bool kBytes = OP == kProdBytes, kGated = ProdKind<OP>::kGated, kScaled = ProdKind<OP>::kScaled;
    static_assert(kFewSteps * 64 == 256, "two scaled blocks");
    constexpr int kOutputs = kFewOutputs / ProdKind<OP>::kPerResult;           // a job's
    constexpr int kNumber = kBytes ? tc::kNumberS8 : kScaled ? tc::kNumberE4M3 : IsBF16<S>::value ? tc::kNumberBF16 : tc::kNumberF16;
    constexpr int ES = kBytes || kScaled ? 1 : 2;
    __shared__ uint32_t sums[kFewWarps][kFewOutputs][8 * NT + 1];
    __shared__ int live[kFewMaxRows], first[kFewMaxRows], rows[kFewMaxRows], lives, bounds[2];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gid = lane >> 2, quad = lane & 3;
    const uint32_t groups = (g.outs + kOutputs - 1) / kOutputs;
    const uint32_t pitch = g.in * ES;                // bytes of a row of either operand
    const uint32_t blocks = (pitch + kFewSteps * 64 - 1) / (kFewSteps * 64), in_blocks = (g.in + 127) / 128;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (!early) asm volatile("griddepcontrol.wait;" ::: "memory");
    if (g.offsets) {
        // the experts' rows in groups of at most 8 NT (no more groups than rows), the ranges held inside [0, rows] and ascending
        if (warp == 0) {
            int n = 0, last = 0;
            for (uint32_t e0 = 0; e0 <= g.experts; e0 += 32) {
                const uint32_t e = e0 + lane;
                int at = e <= g.experts ? min(max(__ldg(g.offsets + e), 0), int(g.rows)) : int(g.rows);
                if (e > g.experts) at = 0;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int v = __shfl_up_sync(0xffffffffu, at, o);
                    if (lane >= o) at = max(at, v);
                }
                at = max(at, last);
                int before = __shfl_up_sync(0xffffffffu, at, 1);
                if (lane == 0) before = e0 ? last : at;
                if (e == 0) bounds[0] = at;
                if (e == g.experts) bounds[1] = at;
                const int m = e <= g.experts ? at - before : 0;       // of expert e - 1
                int mine = (m + 8 * NT - 1) / (8 * NT), upto = mine;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int v = __shfl_up_sync(0xffffffffu, upto, o);
                    if (lane >= o) upto += v;
                }
                for (int j = 0; j < mine; ++j) {
                    const int i = n + upto - mine + j;
                    live[i] = int(e) - 1;
                    first[i] = before + j * 8 * NT;
                    rows[i] = min(8 * NT, m - j * 8 * NT);
                }
                n += __shfl_sync(0xffffffffu, upto, 31);
                last = __shfl_sync(0xffffffffu, at, 31);
            }
            if (lane == 0) lives = n;
        }
        __syncthreads();
        for (size_t i = blockIdx.x * blockDim.x + threadIdx.x; i < g.rows * g.outs; i += size_t(gridDim.x) * blockDim.x) {
            const int r = int(i / g.outs);
            if (r >= bounds[0] && r < bounds[1]) continue;
            S::store1(static_cast<typename S::elem*>(g.out) + i, 0.0f);
            if (g.slope && kGated) {
                S::store1(static_cast<typename S::elem*>(g.slope) + i + size_t(r) * g.outs, 0.0f);
                S::store1(static_cast<typename S::elem*>(g.slope) + i + size_t(r + 1) * g.outs, 0.0f);
            } else if (g.slope) {
                S::store1(static_cast<typename S::elem*>(g.slope) + i, 0.0f);
            }
        }
    } else {
        if (threadIdx.x == 0) lives = (int(g.rows) + 8 * NT - 1) / (8 * NT);
        static_assert(kFewMaxRows == kFewWarps * 32, "a thread for each group");
        {
            live[threadIdx.x] = 0;
            first[threadIdx.x] = threadIdx.x * 8 * NT;
            rows[threadIdx.x] = min(8 * NT, int(g.rows) - int(threadIdx.x) * 8 * NT);
        }
        __syncthreads();
    }
    // A walk over (job, block) pairs: the next pair's weights are requested as soon as the current ones have been used, before the
    // sums of a finished job meet, so that a CTA's reads never pause.
    bool waited = !early;
    const uint32_t jobs = groups * uint32_t(lives);
    uint4 lo[kFewSteps], hi[kFewSteps];
    auto request = [&](uint32_t job, uint32_t b) {
        const uint32_t slot = job / groups, o0 = (job - slot * groups) * kOutputs;
        const unsigned char* w = static_cast<const unsigned char*>(g.b) + (size_t(live[slot]) * g.outs * ProdKind<OP>::kPerResult + o0) * pitch;
        // rows past the last output repeat it: their sums are not used
        const unsigned char* w_lo = w + size_t(min(uint32_t(gid), g.outs - 1 - o0)) * pitch;
        const unsigned char* w_hi = kGated ? w_lo + size_t(g.outs) * pitch : w + size_t(min(uint32_t(gid) + 8, g.outs - 1 - o0)) * pitch;
        const uint32_t k0 = b * (kFewSteps * 64) + quad * 16;         // this lane's first byte
#pragma unroll
        for (int i = 0; i < kFewSteps; ++i) {
            lo[i] = hi[i] = make_uint4(0, 0, 0, 0);
            if (k0 + i * 64 < pitch) {
                lo[i] = __ldcs(reinterpret_cast<const uint4*>(w_lo + k0 + i * 64));
                hi[i] = __ldcs(reinterpret_cast<const uint4*>(w_hi + k0 + i * 64));
            }
        }
    };
    uint32_t job = blockIdx.x;
    if (job < jobs && uint32_t(warp) < blocks) request(job, warp);
    for (; job < jobs; job += gridDim.x) {
        const int slot = int(job / groups);
        const uint32_t o0 = (job - slot * groups) * kOutputs;
        const int m = rows[slot];
        const unsigned char* x = static_cast<const unsigned char*>(g.a) + size_t(first[slot]) * pitch;
        uint32_t acc[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[n][0] = acc[n][1] = acc[n][2] = acc[n][3] = 0;
        if (!waited) {
            asm volatile("griddepcontrol.wait;" ::: "memory");
            waited = true;
        }
        for (uint32_t b = warp; b < blocks; b += kFewWarps) {
            const uint32_t k0 = b * (kFewSteps * 64) + quad * 16;
            // rows of the sums are outputs, of one block of weights (gated: the lower and the upper half of one of each weight)
            float sw[2][2];
            if (kScaled)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        if (!kGated && e) sw[h][e] = sw[h][0];
                        else sw[h][e] = b * 2 + h < in_blocks ? g.b_scale[(size_t(e ? (g.outs + 127) / 128 : 0) + o0 / 128) * in_blocks + b * 2 + h] : 0.0f;
                    }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                if (n * 8 >= m) break;
                // columns of the sums are tokens, two to a lane; past the row's last block all sums are 0, whatever they are scaled by
                float sx[2][2];
                if (kScaled)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int e = 0; e < 2; ++e)
                            sx[h][e] = b * 2 + h < in_blocks ? g.a_scale[size_t(b * 2 + h) * g.rows + first[slot] + min(n * 8 + int(quad) * 2 + e, m - 1)] : 0.0f;
                // tokens past the last one repeat it
                const unsigned char* row = x + size_t(min(n * 8 + gid, m - 1)) * pitch + k0;
                uint4 v[kFewSteps];
#pragma unroll
                for (int i = 0; i < kFewSteps; ++i) v[i] = k0 + i * 64 < pitch ? *reinterpret_cast<const uint4*>(row + i * 64) : make_uint4(0, 0, 0, 0);
                if constexpr (kScaled) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        uint32_t part[4] = {0, 0, 0, 0};
#pragma unroll
                        for (int i = 2 * h; i < 2 * h + 2; ++i) {
                            few_product<kNumber>(part, lo[i].x, hi[i].x, lo[i].y, hi[i].y, v[i].x, v[i].y);
                            few_product<kNumber>(part, lo[i].z, hi[i].z, lo[i].w, hi[i].w, v[i].z, v[i].w);
                        }
                        const float scale[4] = {sx[h][0] * sw[h][0], sx[h][1] * sw[h][0], sx[h][0] * sw[h][1], sx[h][1] * sw[h][1]};
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[n][e] = __float_as_uint(fmaf(__uint_as_float(part[e]), scale[e], __uint_as_float(acc[n][e])));
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < kFewSteps; ++i) {
                        few_product<kNumber>(acc[n], lo[i].x, hi[i].x, lo[i].y, hi[i].y, v[i].x, v[i].y);
                        few_product<kNumber>(acc[n], lo[i].z, hi[i].z, lo[i].w, hi[i].w, v[i].z, v[i].w);
                    }
                }
            }
            if (b + kFewWarps < blocks) request(job, b + kFewWarps);
            else if (job + gridDim.x < jobs) request(job + gridDim.x, warp);
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            sums[warp][gid][n * 8 + quad * 2] = acc[n][0];
            sums[warp][gid][n * 8 + quad * 2 + 1] = acc[n][1];
            sums[warp][gid + 8][n * 8 + quad * 2] = acc[n][2];
            sums[warp][gid + 8][n * 8 + quad * 2 + 1] = acc[n][3];
        }
        __syncthreads();
        for (int i = threadIdx.x; i < kOutputs * m; i += kFewWarps * 32) {
            const int token = i / kOutputs;
            const uint32_t o = o0 + i % kOutputs;
            if (o >= g.outs) continue;
            const size_t row = first[slot] + token;
            if constexpr (kGated) {
                float z = 0.0f, u = 0.0f, f, d;
#pragma unroll
                for (int k = 0; k < kFewWarps; ++k) {
                    z += __uint_as_float(sums[k][i % kOutputs][token]);
                    u += __uint_as_float(sums[k][i % kOutputs + kOutputs][token]);
                }
                if (g.bias) {
                    const typename S::elem* b = static_cast<const typename S::elem*>(g.bias) + size_t(live[slot]) * 2 * g.outs + o;
                    z += S::load1(b);
                    u += S::load1(b + g.outs);
                }
                act1(g.act, z, &f, &d);
                S::store1(static_cast<typename S::elem*>(g.out) + row * g.outs + o, f * u);
                if (g.slope) {
                    typename S::elem* both = static_cast<typename S::elem*>(g.slope) + row * 2 * g.outs + o;
                    S::store1(both, d * u);
                    S::store1(both + g.outs, f);
                }
                continue;
            }
            float z;
            if (kBytes) {
                int t = 0;
#pragma unroll
                for (int k = 0; k < kFewWarps; ++k) t += int(sums[k][i % kOutputs][token]);
                z = float(t) * (g.a_scale[row] * g.b_scale[o]);
            } else {
                z = 0.0f;
#pragma unroll
                for (int k = 0; k < kFewWarps; ++k) z += __uint_as_float(sums[k][i % kOutputs][token]);
            }
            if (g.bias) z += S::load1(static_cast<const typename S::elem*>(g.bias) + size_t(live[slot]) * g.outs + o);
            float y, d;
            act1(g.act, z, &y, &d);
            S::store1(static_cast<typename S::elem*>(g.out) + row * g.outs + o, y);
            if (g.slope) S::store1(static_cast<typename S::elem*>(g.slope) + row * g.outs + o, d);
        }
        __syncthreads();
    }
    if (!waited) asm volatile("griddepcontrol.wait;" ::: "memory");   // a CTA without work ends in order too
}

template <int OP, class S, int NT> cudaError_t launch_few_rows_tiles(const ProdArgs& g, int sms, int early, cudaStream_t st)
{
    const size_t live = g.rows < g.experts ? g.rows : g.experts;
    constexpr int kOutputs = kFewOutputs / ProdKind<OP>::kPerResult;
    const size_t jobs = (g.outs + kOutputs - 1) / kOutputs * live, fit = size_t(sms) * FewResident<OP, NT>::value;
    // one expert, whose jobs are known: as many for each CTA, rather than a last turn of a few (13.3 -> 12.6 us); else all that fit
    // (beside block scales, whose conversions want every warp that fits, they cost more than the last turn: 28 -> 32 us)
    const size_t turns = g.experts == 1 && !ProdKind<OP>::kScaled ? (jobs + fit - 1) / fit : 1, grid = (jobs + turns - 1) / turns;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(grid < fit ? grid : fit));
    cfg.blockDim = dim3(kFewWarps * 32);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, few_rows_kernel<OP, S, NT>, g, early);
}

// Whether there are few rows: 16 at most, or up to four for each expert.  Measured against tiles on tcgen05 (us): one token
// 4096 -> 12288 in 8 bits 12.6 (24.6), 16 tokens 4096 -> 4096 6.6 (14.0); 32 of them bf16 23.6 (16.5); 24 rows over 64 experts
// 2048 -> 1408 bf16 24.8 (44.2), 256 of them 62.7 (65.7); 64 rows over 8 experts 2048 -> 4096 34.7 (28.7).
// (Byte offsets inside a row are 32-bit there.)
inline bool few_rows(const ProdArgs& g) { return g.in < (1u << 28) && (g.rows <= 16 || (g.rows <= kFewMaxRows && g.rows <= 4 * size_t(g.experts))); }

// Tokens a job takes at once, by the rows an expert has on average: an expert with more is read once per such group.
template <int OP, class S> cudaError_t launch_few_rows(const ProdArgs& g, int sms, int early, cudaStream_t st)
{
    const size_t mean = (g.rows + g.experts - 1) / g.experts;
    if (mean <= 8) return launch_few_rows_tiles<OP, S, 1>(g, sms, early, st);
    return launch_few_rows_tiles<OP, S, 2>(g, sms, early, st);
}

}  // namespace nfad
