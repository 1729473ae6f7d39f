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

// whether element j of the draw is kept; `dropped` is T 2^16 (T = 65536, where nothing is, never gets here)
__device__ __forceinline__ bool kept(const DropoutArgs& a, uint32_t w, int j) { return (j & 1 ? w : w << 16) >= a.dropped; }

// V results, whose bits are the first V halves of the draw; K void: no activation
template <class S, class K, class P> struct DropoutBody {
    static constexpr int V = S::kVec;
    // x, then bias or residual (null: none); out and slope
    static __device__ __forceinline__ void packet(const DropoutArgs& a, const Draw& draw, const float (&x)[V], const float* other, float (&y)[V], float (&d)[V])
    {
        if constexpr (IsVoid<K>::value) {
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const bool keep = kept(a, draw.w[e >> 1], e);
                const float r = other ? other[e] : 0.0f;
                y[e] = keep ? fmaf(x[e], a.scale, r) : r;
            }
        } else {
            // a dropped element goes in as 0, where every f is 0 and every f' finite: so nothing that it held comes out, and the factor
            // may be a product's
            float z[V], factor[V];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const bool keep = kept(a, draw.w[e >> 1], e);
                z[e] = keep ? (other ? bias_sum(x[e], other[e]) : x[e]) : 0.0f;
                factor[e] = keep ? a.scale : 0.0f;
            }
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
            for (int e = 0; e < V; e += 2) {
                const float2 f = make_float2(factor[e], factor[e + 1]);
                const float2 y2 = hw::mul2(make_float2(y[e], y[e + 1]), f), d2 = hw::mul2(make_float2(d[e], d[e + 1]), f);
                y[e] = y2.x; y[e + 1] = y2.y;
                d[e] = d2.x; d[e + 1] = d2.y;
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
            const ActOut o = evaluate<K, P>(!keep ? 0.0f : a.other ? bias_sum(x, S::load1(static_cast<const E*>(a.other) + i % a.cols)) : x);
            S::store1(static_cast<E*>(a.y) + i, __fmul_rn(o.y, keep ? a.scale : 0.0f));
            S::store1(static_cast<E*>(a.slope) + i, __fmul_rn(o.dydx, keep ? a.scale : 0.0f));
        }
    }
};

// kWhere: where `other` is: nowhere, a residual, a bias of any length
enum DropoutOther { kOtherNone, kOtherPackets, kOtherSingles };

// packets of each tensor that a thread has in flight
template <class K, int kWhere> struct DropoutTile { static constexpr int value = IsVoid<K>::value ? kWhere == kOtherNone ? 4 : 3 : 2; };

template <class S, class K, class P, int kWhere>
__global__ void __launch_bounds__(kBlock, 4) dropout_kernel(const __grid_constant__ DropoutArgs a)
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
                if (kWhere == kOtherPackets) more[u] = load_packet(static_cast<const uint4*>(a.other) + pk);
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
            if (kWhere == kOtherPackets) S::unpack(more[u], r);
            if (kWhere == kOtherSingles) {
                uint32_t c = uint32_t(pk * V % a.cols);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    r[e] = S::load1(static_cast<const E*>(a.other) + c);
                    if (++c == a.cols) c = 0;
                }
            }
            DropoutBody<S, K, P>::packet(a, mine, x, kWhere == kOtherNone ? nullptr : r, y, d);
            store_packet<true>(static_cast<uint4*>(a.y) + pk, S::pack(y));
            if (kAct) store_packet<false>(static_cast<uint4*>(a.slope) + pk, S::pack(d));
        }
    }
    if (blockIdx.x == 0 && threadIdx.x < a.n - packets * V) DropoutBody<S, K, P>::single(a, at, packets * V + threadIdx.x);
}

// With a bias whose rows begin on packets: a thread has one column packet of kBiasRows rows, as in the pass without dropout, and reads
// the bias once.  (Flat, with the packet's place in its row from a 64-bit division: 171 us for 8192 x 12288 bf16, GELU-erf.)
template <class S, class K, class P>
__global__ void __launch_bounds__(kBiasMaxBlock, 4) dropout_rows_kernel(const __grid_constant__ DropoutArgs a)
{
    constexpr int V = S::kVec, U = kBiasRows;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const uint32_t cp = blockIdx.x * blockDim.x + threadIdx.x;
    if (cp >= a.row_packets) return;
    const uint64_t at = a.offset + (a.step ? *a.step : 0);
    const size_t rows = a.n / a.cols, chunks = (rows + U - 1) / U;
    float bias[V];
    S::unpack(__ldg(static_cast<const uint4*>(a.other) + cp), bias);
    for (size_t chunk = blockIdx.y; chunk < chunks; chunk += gridDim.y) {
        const size_t row0 = chunk * U, pk0 = row0 * a.row_packets + cp;
        uint4 raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (row0 + u < rows) raw[u] = load_packet(static_cast<const uint4*>(a.x) + pk0 + size_t(u) * a.row_packets);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (row0 + u >= rows) break;
            const size_t pk = pk0 + size_t(u) * a.row_packets;
            Draw draw = philox(V == 8 ? pk : pk >> 1, at, a.seed);
            if (V == 4 && (pk & 1)) { draw.w[0] = draw.w[2]; draw.w[1] = draw.w[3]; }
            float x[V], y[V], d[V];
            S::unpack(raw[u], x);
            DropoutBody<S, K, P>::packet(a, draw, x, bias, y, d);
            store_packet<true>(static_cast<uint4*>(a.y) + pk, S::pack(y));
            store_packet<false>(static_cast<uint4*>(a.slope) + pk, S::pack(d));
        }
    }
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
    if constexpr (kAct) {
        if (a.cols % S::kVec || !aligned16(a.other)) return launch_dropout_packets<S, K, P, kOtherSingles>(a, st);
        a.row_packets = a.cols / S::kVec;
        const unsigned block = bias_block(a.row_packets);
        const size_t chunks = (a.n / a.cols + kBiasRows - 1) / kBiasRows;
        cudaLaunchConfig_t cfg;
        cudaLaunchAttribute attr[1];
        bias_launch_config(&cfg, attr, (a.row_packets + block - 1) / block, block, st, true);
        cfg.gridDim.y = unsigned(chunks < 65535 ? chunks : 65535);
        return cudaLaunchKernelEx(&cfg, dropout_rows_kernel<S, K, P>, a);
    } else {
        return launch_dropout_packets<S, K, P, kOtherPackets>(a, st);
    }
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
