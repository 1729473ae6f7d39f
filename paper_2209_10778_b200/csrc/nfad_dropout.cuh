// nfad_dropout.cuh -- dropout whose mask is a function of a counter: never stored, drawn again where it is needed.
//
// Element i of a call belongs to draw i / 8; a draw is one evaluation of Philox 4x32 with ten rounds (Salmon, Moraes, Dror and
// Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011) on the counter (draw, offset + step) under the key `seed`: 128 bits, 16 for each
// of eight elements.  An element is dropped when its 16 bits are below T = rint(65536 p), and kept ones are multiplied by
// 65536 / (65536 - T): the scale belongs to the probability that is drawn, so that the mean is kept exactly.
//
// Behind an activation the mask and the scale go into both results of the nested pass: y = m f(z), and m f'(z), the derivative of that y.
// What is saved for the backward pass carries the mask, and the backward pass is Eq. 4's multiplication, unchanged.
//
// Work: a packet of 16 bytes a thread and turn, as in the streaming engine.  A packet of 16-bit values is one draw, of fp32 values half of
// one (both threads draw; fp32 has the issue slots).  What bounds it: memory, beside 20 products of 32 x 32 bits a draw (sixteen bits an
// element instead of 32 halve them).
#pragma once

#include "nfad_bias.cuh"
#include "nfad_dropout_args.h"
#include "nfad_internal.h"

namespace nfad {

struct Draw { uint32_t w[4]; };                      // element j of eight: the lower (even j) or upper half of w[j / 2]

__device__ __forceinline__ Draw philox(uint64_t index, uint64_t at, uint64_t seed)
{
    uint32_t c0 = uint32_t(index), c1 = uint32_t(index >> 32), c2 = uint32_t(at), c3 = uint32_t(at >> 32);
    uint32_t k0 = uint32_t(seed), k1 = uint32_t(seed >> 32);
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = uint64_t(c0) * 0xD2511F53u, b = uint64_t(c2) * 0xCD9E8D57u;
        c0 = uint32_t(b >> 32) ^ c1 ^ k0;
        c1 = uint32_t(b);
        c2 = uint32_t(a >> 32) ^ c3 ^ k1;
        c3 = uint32_t(a);
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return {c0, c1, c2, c3};
}

// keep[j]: element j of the draw.  `dropped` is T 2^16 (2^32 - 1 for T = 65536, when `live` is 0 and nothing is kept).
__device__ __forceinline__ bool kept(const DropoutArgs& a, uint32_t w, int j) { return ((j & 1 ? w : w << 16) & a.live) >= a.dropped; }

// V results from element 8 draw + first on; K void: no activation
template <class S, class K, class P> struct DropoutBody {
    static constexpr int V = S::kVec;
    // x, then bias or residual (null: none); out and slope
    static __device__ __forceinline__ void packet(const DropoutArgs& a, const Draw& draw, int first, const float (&x)[V], const float* other, float (&y)[V], float (&d)[V])
    {
        if constexpr (IsVoid<K>::value) {
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const bool keep = kept(a, draw.w[(first + e) >> 1], e);
                const float r = other ? other[e] : 0.0f;
                y[e] = keep ? fmaf(x[e], a.scale, r) : r;
            }
        } else {
            float z[V];
#pragma unroll
            for (int e = 0; e < V; ++e) z[e] = other ? bias_sum(x[e], other[e]) : x[e];
            // the widths of the plain pass for each kind
            if constexpr (ForwardTrainOp<K, P>::kPairs) {
#pragma unroll
                for (int e = 0; e < V; e += 2) {
                    const ActOut2 o = evaluate(K{}, Fast2{}, make_float2(z[e], z[e + 1]));
                    y[e] = o.y.x; y[e + 1] = o.y.y;
                    d[e] = o.dydx.x; d[e + 1] = o.dydx.y;
                }
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const ActOut o = evaluate<K, P>(z[e]);
                    y[e] = o.y;
                    d[e] = o.dydx;
                }
            }
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const bool keep = kept(a, draw.w[(first + e) >> 1], e);
                y[e] = keep ? __fmul_rn(y[e], a.scale) : 0.0f;
                d[e] = keep ? __fmul_rn(d[e], a.scale) : 0.0f;
            }
        }
    }
    // one element, with the packets' arithmetic
    static __device__ __forceinline__ void single(const DropoutArgs& a, uint64_t at, size_t i)
    {
        using E = typename S::elem;
        const Draw draw = philox(i >> 3, at, a.seed);
        const int j = int(i & 7);
        const uint32_t w = j < 4 ? j < 2 ? draw.w[0] : draw.w[1] : j < 6 ? draw.w[2] : draw.w[3];
        const bool keep = kept(a, w, j);
        const float x = S::load1(static_cast<const E*>(a.x) + i);
        if constexpr (IsVoid<K>::value) {
            const float r = a.other ? S::load1(static_cast<const E*>(a.other) + i) : 0.0f;
            S::store1(static_cast<E*>(a.y) + i, keep ? fmaf(x, a.scale, r) : r);
        } else {
            const ActOut o = evaluate<K, P>(a.other ? bias_sum(x, S::load1(static_cast<const E*>(a.other) + i % a.cols)) : x);
            S::store1(static_cast<E*>(a.y) + i, keep ? __fmul_rn(o.y, a.scale) : 0.0f);
            S::store1(static_cast<E*>(a.slope) + i, keep ? __fmul_rn(o.dydx, a.scale) : 0.0f);
        }
    }
};

// kWhere: where `other` is: nowhere, a residual (or a bias whose rows begin on packets) read by packets, a bias of any length
enum DropoutOther { kOtherNone, kOtherPackets, kOtherSingles };

// packets of each tensor that a thread has in flight
template <class K, int kWhere> struct DropoutTile { static constexpr int value = IsVoid<K>::value ? kWhere == kOtherNone ? 4 : 3 : 2; };

template <class S, class K, class P, int kWhere>
__global__ void __launch_bounds__(kBlock, IsVoid<K>::value ? 4 : S::kMinBlocks) dropout_kernel(const __grid_constant__ DropoutArgs a)
{
    constexpr int V = S::kVec, U = DropoutTile<K, kWhere>::value;
    constexpr bool kAct = !IsVoid<K>::value;
    using E = typename S::elem;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const uint64_t at = a.offset + (a.step ? *a.step : 0);
    const size_t packets = a.n / V, tile = size_t(kBlock) * U;
    for (size_t t0 = size_t(blockIdx.x) * tile; t0 < packets; t0 += size_t(gridDim.x) * tile) {
        uint4 raw[U], more[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const size_t pk = t0 + size_t(u) * kBlock + threadIdx.x;
            if (pk < packets) {
                raw[u] = load_packet(static_cast<const uint4*>(a.x) + pk);
                if (kWhere == kOtherPackets && !kAct) more[u] = load_packet(static_cast<const uint4*>(a.other) + pk);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const size_t pk = t0 + size_t(u) * kBlock + threadIdx.x;
            if (pk >= packets) break;
            const Draw draw = philox(V == 8 ? pk : pk >> 1, at, a.seed);
            Draw mine = draw;
            if (V == 4 && (pk & 1)) { mine.w[0] = draw.w[2]; mine.w[1] = draw.w[3]; }
            float x[V], r[V], y[V], d[V];
            S::unpack(raw[u], x);
            if (kWhere == kOtherPackets) S::unpack(kAct ? __ldg(static_cast<const uint4*>(a.other) + pk % a.row_packets) : more[u], r);
            if (kWhere == kOtherSingles) {
                uint32_t c = uint32_t(pk * V % a.cols);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    r[e] = S::load1(static_cast<const E*>(a.other) + c);
                    if (++c == a.cols) c = 0;
                }
            }
            DropoutBody<S, K, P>::packet(a, mine, 0, x, kWhere == kOtherNone ? nullptr : r, y, d);
            store_packet<true>(static_cast<uint4*>(a.y) + pk, S::pack(y));
            if (kAct) store_packet<false>(static_cast<uint4*>(a.slope) + pk, S::pack(d));
        }
    }
    if (blockIdx.x == 0 && threadIdx.x < a.n - packets * V) DropoutBody<S, K, P>::single(a, at, packets * V + threadIdx.x);
}

// Tensors that begin off the 16-byte boundaries: one element a thread.
template <class S, class K, class P> __global__ void __launch_bounds__(kBlock) dropout_single_kernel(const __grid_constant__ DropoutArgs a)
{
    const uint64_t at = a.offset + (a.step ? *a.step : 0);
    const size_t stride = size_t(gridDim.x) * kBlock;
    for (size_t i = size_t(blockIdx.x) * kBlock + threadIdx.x; i < a.n; i += stride) DropoutBody<S, K, P>::single(a, at, i);
}

template <class S, class K, class P, int kWhere> cudaError_t launch_dropout_packets(const DropoutArgs& a, cudaStream_t st)
{
    constexpr int U = DropoutTile<K, kWhere>::value;
    const size_t tiles = (a.n / S::kVec + size_t(kBlock) * U - 1) / (size_t(kBlock) * U);
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute attr[1];
    bias_launch_config(&cfg, attr, tiles == 0 ? 1 : tiles < 0x7fffffff ? tiles : 0x7fffffff, kBlock, st, true);
    return cudaLaunchKernelEx(&cfg, dropout_kernel<S, K, P, kWhere>, a);
}

template <class S, class K, class P> cudaError_t launch_dropout_kind(const DropoutArgs& in, cudaStream_t st)
{
    DropoutArgs a = in;
    constexpr bool kAct = !IsVoid<K>::value;
    if (!aligned16(a.x) || !aligned16(a.y) || (kAct && !aligned16(a.slope)) || (!kAct && !aligned16(a.other)))
    {
        const unsigned grid = edge_grid_blocks(a.n, kBlock);
        dropout_single_kernel<S, K, P><<<grid, kBlock, 0, st>>>(a);
        return cudaPeekAtLastError();
    }
    if (!a.other) return launch_dropout_packets<S, K, P, kOtherNone>(a, st);
    a.row_packets = kAct ? a.cols / S::kVec : 0;
    if (!kAct || (a.cols % S::kVec == 0 && aligned16(a.other))) return launch_dropout_packets<S, K, P, kOtherPackets>(a, st);
    if constexpr (kAct) return launch_dropout_packets<S, K, P, kOtherSingles>(a, st);
    return cudaErrorInvalidValue;
}

template <class S, class P> cudaError_t launch_dropout_store(int kind, const DropoutArgs& a, cudaStream_t st)
{
    switch (kind) {
    case -1:        return launch_dropout_kind<S, void, P>(a, st);
    case kGeluErf:  return launch_dropout_kind<S, GeluErf, P>(a, st);
    case kGeluTanh: return launch_dropout_kind<S, GeluTanh, P>(a, st);
    case kSwish:    return launch_dropout_kind<S, Swish, P>(a, st);
    case kMish:     return launch_dropout_kind<S, Mish, P>(a, st);
    }
    return cudaErrorInvalidValue;
}

}  // namespace nfad
