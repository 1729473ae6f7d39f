// nfad_scaled_launch.cuh -- launches of the products in 8-bit floating point with block scales.
#pragma once

#include "nfad_product_launch.cuh"
#include "nfad_scaled.cuh"
#include "nfad_scaled_split.cuh"

namespace nfad {

template <int OP, int BN, class S, bool kGather, bool kPair = false>
cudaError_t launch_scaled_tile(const ProdArgs& g, int sms, cudaStream_t st)
{
    using Kind = ProdKind<OP>;
    using Tile = ProdTile<BN, kPair>;
    auto kernel = scaled_kernel<OP, BN, S, kGather, kPair>;
    static std::atomic<bool> ready[64] = {};         // the shared-memory opt-in of this kernel, by device (setting it twice is harmless)
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64 || !ready[dev]) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kScaledSmem);
        if (e != cudaSuccess) return e;
        if (dev >= 0 && dev < 64) ready[dev] = true;
    }
    CUtensorMap map_a = {}, map_b = {}, map_out = {};
    // results leave by tensor copies of 64 to a row where rows of them begin on 16-byte boundaries and a warp has as many
    const int kOut = BN / Kind::kPerResult / (ScaledWarps<kGather>::kResult / 4);
    const int out_copies = kOut >= 64 && g.outs % 8 == 0 && reinterpret_cast<uintptr_t>(g.out) % 16 == 0;
    if (out_copies) {
        e = make_map(&map_out, IsBF16<S>::value ? tc::kNumberBF16 : tc::kNumberF16, g.out, g.outs, g.rows, 0, 32);
        if (e != cudaSuccess) return e;
    }
    if (!kGather) {
        e = make_map(&map_a, tc::kNumberE4M3, g.a, g.in, g.rows, 0, Tile::kBoxRows);
        if (e != cudaSuccess) return e;
        e = make_map(&map_b, tc::kNumberE4M3, g.b, g.in, g.outs, Kind::kPerResult, Kind::kGated ? BN / 2 : Tile::kOwnColumns);
        if (e != cudaSuccess) return e;
    }
    constexpr size_t kResults = BN / Kind::kPerResult;
    size_t grid = ((g.rows + Tile::kRows - 1) / Tile::kRows) * ((g.outs + kResults - 1) / kResults);
    if (grid >= (size_t(1) << 31)) return cudaErrorInvalidValue;     // beyond what any device's memory holds
    if (grid > size_t(sms / (kPair ? 2 : 1))) grid = sms / (kPair ? 2 : 1);
    if (kPair) grid *= 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(grid));
    cfg.blockDim = dim3(ScaledWarps<kGather>::kThreads);
    cfg.dynamicSmemBytes = kScaledSmem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 2;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = kPair ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, g, map_a, map_b, map_out, out_copies);
}

template <int OP, class S> cudaError_t launch_scaled_split(const ProdArgs& g, unsigned ranks, cudaStream_t st)
{
    using Kind = ProdKind<OP>;
    auto kernel = scaled_split_kernel<OP, S>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kThinSmem);
    if (e != cudaSuccess) return e;
    CUtensorMap map_a = {}, map_b = {};
    e = make_map(&map_a, tc::kNumberE4M3, g.a, g.in, g.rows, 0, 32);
    if (e != cudaSuccess) return e;
    e = make_map(&map_b, tc::kNumberE4M3, g.b, g.in, g.outs, Kind::kPerResult, kSplitColumns / Kind::kPerResult);
    if (e != cudaSuccess) return e;
    constexpr size_t kResults = kSplitColumns / Kind::kPerResult;
    const size_t tiles = ((g.rows + kTileRows - 1) / kTileRows) * ((g.outs + kResults - 1) / kResults);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(tiles * ranks));     // no more than SMs
    cfg.blockDim = dim3(kSplitThreads);
    cfg.dynamicSmemBytes = kThinSmem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = ranks;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, g, map_a, map_b, uint32_t(ranks));
}

// Over how many CTAs a tile's reduction is split (0: not at all; tiles of another size, which CTAs walk over): as many as one to an SM allows,
// with eight blocks left for each.  Measured (us a call with its quantiser, captured calls on inputs in turn that the caches do not hold; in
// brackets by tiles that are walked over): 100 rows 4096 -> 1024 over 4: 11.1 (17.4), over 8: 19.2; 400 rows 4096 -> 1024 over 2: 15.5 (18.6),
// over 4: 22.5; 40 rows 8192 -> 2048 over 4: 15.4 (29.5); gated 100 rows 8192 -> 2 x 2048 over 2: 22.3 (29.4).  One CTA to a tile of this size
// was never the fastest (40 rows 4096 -> 28672: 57, by tiles of 256 26.9).
template <int OP> unsigned scaled_split_ranks(const ProdArgs& g, int sms)
{
    if (g.outs % 8 || (reinterpret_cast<uintptr_t>(g.out) | reinterpret_cast<uintptr_t>(g.bias)) % 16) return 0;      // its results go by packets
    constexpr size_t kResults = kSplitColumns / ProdKind<OP>::kPerResult;
    const size_t tiles = ((g.rows + kTileRows - 1) / kTileRows) * ((g.outs + kResults - 1) / kResults), blocks = (g.in + kScaleBlock - 1) / kScaleBlock;
    for (unsigned ranks = 8; ranks > 1; ranks /= 2)
        if (tiles * ranks <= size_t(sms) && blocks >= 8 * ranks) return ranks;
    return 0;
}

template <int OP, class S> cudaError_t launch_scaled_store(const ProdArgs& g, cudaStream_t st)
{
    DeviceInfo di;
    cudaError_t e = device_info(&di);
    if (e != cudaSuccess) return e;
    const uintptr_t low = reinterpret_cast<uintptr_t>(g.a) | reinterpret_cast<uintptr_t>(g.b) | uintptr_t(g.in);
    // a tensor copy needs rows that begin on 16-byte boundaries (and something to copy)
    if (low % 16 || g.in == 0) return launch_scaled_tile<OP, 64, S, true>(g, di.sm_count, st);
    // Up to eight rows, a column each of the small matrix instruction.  Against tiles (us, measured as above): 8 rows 4096 -> 4096 8.2 (11.1 split
    // over 4, 15.1 walked over), gated 4096 -> 2 x 14336 30.4 (31.5), 1 row of it 28.0 (32.9); with two such groups 16 rows of it take 93 (30.8).
    if (few_rows(g) && g.rows <= 8) return launch_few_rows_tiles<OP, S, 1>(g, di.sm_count, g.b_ready, st);
    if (const unsigned ranks = scaled_split_ranks<OP>(g, di.sm_count)) return launch_scaled_split<OP, S>(g, ranks, st);
    // The rule of the other products, by turns of all SMs, holds for these too.  Alone, in turn as above (us, by 128 / 256 columns / pairs): 128 rows
    // 4096 -> 8192 19.6 / 21.0 / 21.4; 40 rows 4096 -> 28672 31.8 / 25.1 / 37.4, gated 4096 -> 2 x 14336 32.6 / 26.7 / 40.3; 300 rows 2048 -> 8192
    // 17.0 / 13.4 / 14.0; 1024 rows 4096 -> 4096 31.2 / 22.6 / 23.4; 4096 rows 88.8 / 71.9 / 70.4, gated 185 / 137 / 122.
    switch (product_tile<OP>(g, di.sm_count)) {
    case kPairTile: return launch_scaled_tile<OP, 256, S, false, true>(g, di.sm_count, st);
    case 256: return launch_scaled_tile<OP, 256, S, false>(g, di.sm_count, st);
    default:  return launch_scaled_tile<OP, 128, S, false>(g, di.sm_count, st);
    }
}

template <int OP> cudaError_t launch_scaled_op(int dtype, const ProdArgs& g, cudaStream_t st)
{
    if (dtype == kBF16) return launch_scaled_store<OP, StoreBF16>(g, st);
    if (dtype == kF16) return launch_scaled_store<OP, StoreF16>(g, st);
    return cudaErrorInvalidValue;
}

}  // namespace nfad
