// nfad_product_launch.cuh -- tensor maps, tile widths and launches of the matrix products.
#pragma once

#include <atomic>
#include <mutex>

#include "nfad_few_rows.cuh"
#include "nfad_product.cuh"
#include "nfad_split.cuh"

namespace nfad {

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                 const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline cudaError_t encode_function(EncodeTiled* out)
{
    static std::mutex lock;
    static EncodeTiled found = nullptr;
    std::lock_guard<std::mutex> hold(lock);
    if (!found) {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult r;
        cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &r);
        if (e != cudaSuccess) return e;
        if (r != cudaDriverEntryPointSuccess || !p) return cudaErrorNotSupported;
        found = reinterpret_cast<EncodeTiled>(p);
    }
    *out = found;
    return cudaSuccess;
}

// [d2, d1, d0] contiguous elements in boxes of b1 rows of 128 bytes; d2 == 0: two dimensions.  What lies outside reads as zero.
inline cudaError_t make_map(CUtensorMap* m, int number, const void* p, uint64_t d0, uint64_t d1, uint64_t d2, uint32_t b1)
{
    EncodeTiled encode;
    cudaError_t e = encode_function(&encode);
    if (e != cudaSuccess) return e;
    const bool bytes = number == tc::kNumberS8 || number == tc::kNumberE4M3;
    const uint32_t es = bytes ? 1 : 2;
    const CUtensorMapDataType type = bytes ? CU_TENSOR_MAP_DATA_TYPE_UINT8
                                     : number == tc::kNumberBF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    const cuuint64_t dims[3] = {d0, d1, d2}, strides[2] = {d0 * es, d0 * d1 * es};
    const cuuint32_t box[3] = {128 / es, b1, 1}, step[3] = {1, 1, 1};
    const CUresult r = encode(m, type, d2 ? 3 : 2, const_cast<void*>(p), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

template <int OP, int BN, class S, bool kGather, bool kPair = false>
cudaError_t launch_product_tile(const ProdArgs& g, int sms, cudaStream_t st)
{
    using Kind = ProdKind<OP>;
    using Tile = ProdTile<BN, kPair>;
    auto kernel = product_kernel<OP, BN, S, kGather, kPair>;
    static std::atomic<bool> ready[64] = {};         // the shared-memory opt-in of this kernel, by device (setting it twice is harmless)
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64 || !ready[dev]) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kProdSmem);
        if (e != cudaSuccess) return e;
        if (dev >= 0 && dev < 64) ready[dev] = true;
    }
    CUtensorMap map_a = {}, map_b = {};
    if (!kGather) {
        const int number = Kind::kBytes ? tc::kNumberS8 : IsBF16<S>::value ? tc::kNumberBF16 : tc::kNumberF16;
        const uint64_t pitch_a = Kind::kInput || OP == kProdWeight ? g.outs : g.in;
        e = make_map(&map_a, number, g.a, pitch_a, g.rows, 0, Kind::kTurnA ? 64 : Tile::kBoxRows);
        if (e != cudaSuccess) return e;
        e = OP == kProdWeight ? make_map(&map_b, number, g.b, g.in, g.rows, 0, 64)
            : Kind::kGated    ? make_map(&map_b, number, g.b, g.in, g.outs, uint64_t(g.experts) * 2, BN / 2)
                              : make_map(&map_b, number, g.b, g.in, g.outs, g.experts, Kind::kTurnB ? 64 : Tile::kOwnColumns);
        if (e != cudaSuccess) return e;
    }
    constexpr size_t kResults = BN / Kind::kPerResult;
    const size_t width = Kind::kInput || OP == kProdWeight ? g.in : g.outs, b_tiles = (width + kResults - 1) / kResults;
    const size_t a_tiles = OP == kProdWeight ? size_t(g.experts) * ((g.outs + Tile::kRows - 1) / Tile::kRows)
                                             : (g.rows + Tile::kRows - 1) / Tile::kRows + (g.offsets ? g.experts : 0);
    size_t grid = a_tiles * b_tiles;                 // at most this many tiles
    if (grid >= (size_t(1) << 31)) return cudaErrorInvalidValue;     // beyond what any device's memory holds
    if (grid > size_t(sms / (kPair ? 2 : 1))) grid = sms / (kPair ? 2 : 1);
    if (kPair) grid *= 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(grid));
    cfg.blockDim = dim3(ProdWarps<kGather>::kThreads);
    cfg.dynamicSmemBytes = kProdSmem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 2;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = kPair ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, g, map_a, map_b);
}

template <int OP, class S> cudaError_t launch_split(const ProdArgs& g, unsigned ranks, cudaStream_t st)
{
    using Kind = ProdKind<OP>;
    auto kernel = split_kernel<OP, S>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSplitSmem);
    if (e != cudaSuccess) return e;
    CUtensorMap map_a = {}, map_b = {};
    const int number = Kind::kBytes ? tc::kNumberS8 : IsBF16<S>::value ? tc::kNumberBF16 : tc::kNumberF16;
    e = make_map(&map_a, number, g.a, Kind::kInput || OP == kProdWeight ? g.outs : g.in, g.rows, 0, Kind::kTurnA ? 64 : 32);
    if (e != cudaSuccess) return e;
    e = OP == kProdWeight ? make_map(&map_b, number, g.b, g.in, g.rows, 0, 64)
        : Kind::kGated    ? make_map(&map_b, number, g.b, g.in, g.outs, uint64_t(g.experts) * 2, kSplitColumns / 2)
                          : make_map(&map_b, number, g.b, g.in, g.outs, g.experts, 64);
    if (e != cudaSuccess) return e;
    constexpr size_t kResults = kSplitColumns / Kind::kPerResult;
    const size_t width = Kind::kInput || OP == kProdWeight ? g.in : g.outs, b_tiles = (width + kResults - 1) / kResults;
    const size_t a_tiles = OP == kProdWeight ? size_t(g.experts) * ((g.outs + kTileRows - 1) / kTileRows)
                                             : (g.rows + kTileRows - 1) / kTileRows + (g.offsets ? g.experts : 0);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(a_tiles * b_tiles * ranks));          // at most this many tiles; clusters past the last leave
    cfg.blockDim = dim3(kSplitThreads);
    cfg.dynamicSmemBytes = kSplitSmem;
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

// Over how many CTAs a tile's reduction is split (0: not at all; single CTAs or pairs walk over the tiles): as many as two to an
// SM allow, with ten steps left for each.  Measured (us, against tiles that are walked over): 77 rows 5120 -> 2048 in 8 bits over 4:
// 10.7 (16.2); 64 rows 4096 -> 4096 bf16 over 4: 15.7 (23.3); 200 rows over 2: 19.6 (25.1); weight gradient 8192 rows of 256 x 256 over
// 8: 13.3 (41.8).  With eight steps each no gain (1024 x 1024 x 1024 over 2: 10.8, 10.8); with more CTAs than fit twice what it was.
template <int OP> unsigned split_ranks(const ProdArgs& g, int sms)
{
    using Kind = ProdKind<OP>;
    constexpr size_t kResults = kSplitColumns / Kind::kPerResult;
    const size_t width = Kind::kInput || OP == kProdWeight ? g.in : g.outs;
    const uintptr_t results = reinterpret_cast<uintptr_t>(g.out) | reinterpret_cast<uintptr_t>(g.slope) | reinterpret_cast<uintptr_t>(g.bias) | reinterpret_cast<uintptr_t>(g.prev);
    if (width % 8 || results % 16) return 0;         // its results go by packets
    const size_t a_tiles = OP == kProdWeight ? size_t(g.experts) * ((g.outs + kTileRows - 1) / kTileRows)
                                             : (g.rows + kTileRows - 1) / kTileRows + (g.offsets ? g.experts - 1 : 0);
    const size_t tiles = a_tiles * ((width + kResults - 1) / kResults), fit = 2 * size_t(sms);
    const size_t steps = (Kind::kInput ? g.outs : OP == kProdWeight ? g.rows / g.experts : g.in) / ProdKind<OP>::kStep;
    for (unsigned ranks = 8; ranks > 1; ranks /= 2)
        if (tiles * ranks <= fit && steps >= 10 * ranks) return ranks;
    return 0;
}

// Tiles of 128 rows by 256, 128 or 64 columns for single CTAs, or of 256 x 256 for pairs (kPairTile): what takes the fewest turns of
// all SMs, each turn counted by the rows of operands that a CTA copies in a step (128 and the columns; 256 for half a pair).
// Experts' tiles are counted with half a tile of padding each.  Measured (us, by 128 / 256 columns / pairs): 1024 rows 4096 -> 4096 bf16
// 45 / 30 / 29, its gradient of the input 44 / 28 / 26; 512 rows 26 / 28 / 28 (by 64: 48), in 8 bits 17 / 21 / 21; 2048 x 2048 x 2048
// 26 / 19 / 19; 512 rows 512 -> 2048 by 64: 7.1, by 128 8.1; 2000 rows of 16 experts 1024 -> 1024 16 / 14 / 15, 3000 of them 2048 -> 1408
// 38 / 40 / 33; 61 experts of 67 rows 1000 -> 1416 47 / 46 / 56; 32768 rows of 8 experts 2048 -> 8192 by 256: 550, by pairs 450.
// Pairs only where their second 128 rows are not empty as a rule (900 rows of 8 experts 4096 -> 4096: 56 us by 256, 63 by pairs) and, in the
// weight gradient, where the reduction is long enough to pay for the pair's hand-shakes (128 to 256 rows an expert: 55 and 196 us in
// pairs, 47 and 187 by single CTAs; 1024 and more: 377 against 410).
constexpr int kPairTile = 512;
template <int OP> int product_tile(const ProdArgs& g, int sms)
{
    using Kind = ProdKind<OP>;
    const size_t width = (Kind::kInput || OP == kProdWeight ? g.in : g.outs) * size_t(Kind::kPerResult);
    const size_t live = g.rows < g.experts ? g.rows : g.experts;
    auto turns = [&](size_t tile_rows, size_t columns, size_t workers) {
        size_t a = (g.rows + tile_rows - 1) / tile_rows + (live > 1 ? live / 2 : 0);
        if (a < live) a = live;
        if (OP == kProdWeight) a = size_t(g.experts) * ((g.outs + tile_rows - 1) / tile_rows);
        return (a * ((width + columns - 1) / columns) + workers - 1) / workers;
    };
    int best = 256;
    size_t least = turns(128, 256, sms) * 384;
    // 64: a gated tile has results for two warps of each lane quarter, and one with block scales is no narrower than a block
    for (int columns = 128; columns >= (Kind::kGated || Kind::kScaled ? 128 : 64); columns /= 2)
        if (const size_t cost = turns(128, columns, sms) * (128 + columns); cost < least) {
            least = cost;
            best = columns;
        }
    if (g.rows / g.experts >= (OP == kProdWeight ? 512 : 128) && turns(256, 256, sms / 2) * 256 < least) best = kPairTile;
    return best;
}

template <int OP, class S> cudaError_t launch_product_store(const ProdArgs& g, cudaStream_t st)
{
    using Kind = ProdKind<OP>;
    DeviceInfo di;
    cudaError_t e = device_info(&di);
    if (e != cudaSuccess) return e;
    const size_t reduction = Kind::kInput ? g.outs : OP == kProdWeight ? g.rows : g.in;
    const uintptr_t low = reinterpret_cast<uintptr_t>(g.a) | reinterpret_cast<uintptr_t>(g.b) | uintptr_t(g.in) * Kind::kElem |
                          (Kind::kTurnB ? uintptr_t(g.outs) * Kind::kElem : 0);
    // a tensor copy needs rows that begin on 16-byte boundaries (and something to copy)
    if (low % 16 || reduction == 0) return launch_product_tile<OP, 128, S, true>(g, di.sm_count, st);
    if constexpr (Kind::kForward)
        if (few_rows(g)) return launch_few_rows<OP, S>(g, di.sm_count, g.b_ready, st);
    if (const unsigned ranks = split_ranks<OP>(g, di.sm_count)) return launch_split<OP, S>(g, ranks, st);
    switch (product_tile<OP>(g, di.sm_count)) {
    case kPairTile: return launch_product_tile<OP, 256, S, false, true>(g, di.sm_count, st);
    case 256: return launch_product_tile<OP, 256, S, false>(g, di.sm_count, st);
    case 128: return launch_product_tile<OP, 128, S, false>(g, di.sm_count, st);
    default:
        if constexpr (!Kind::kGated) return launch_product_tile<OP, 64, S, false>(g, di.sm_count, st);
        return cudaErrorInvalidValue;
    }
}

template <int OP> cudaError_t launch_product_op(int dtype, const ProdArgs& g, cudaStream_t st)
{
    if (dtype == kBF16) return launch_product_store<OP, StoreBF16>(g, st);
    if (dtype == kF16) return launch_product_store<OP, StoreF16>(g, st);
    return cudaErrorInvalidValue;
}

inline cudaError_t product_faults_here(unsigned* n) { return cudaMemcpyFromSymbol(n, g_product_faults, sizeof *n); }

}  // namespace nfad
