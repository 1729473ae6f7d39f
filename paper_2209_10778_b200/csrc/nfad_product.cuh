// nfad_product.cuh -- matrix products grouped by expert, and the 8-bit product, on the fifth-generation tensor cores, with
// the nested activation in the epilogue: z = x W_e^T + b_e lives only in tensor memory; y = f(z) and f'(z) leave the kernel.
//
// One CTA per SM stays for the whole launch and walks over result tiles of 128 x BN.  Its warps have roles:
//   copy      (one thread) tensor copies of the operands' 128-byte wide boxes into a ring of stages;
//   products  (one thread) 128 x BN x 64 (128 bytes of the reduction) per stage into one of two accumulators;
//   results   (eight warps, four beside a gather) read the other accumulator, apply the epilogue, store.
// So copies, products and epilogues of neighbouring tiles overlap.  Which rows a tile has comes from the offsets on the
// device: every CTA builds the table of row ranges in shared memory and finds its tiles in it, with no word from the host.
// A tile's last rows may belong to the next expert (forward, input gradient): they are computed and not stored, as rows do
// not mix.  In the weight gradient rows are the reduction, so rows past the expert's end are cleared in shared memory
// (both operands: 0 times a NaN of the neighbour would be one).
//
// Operands that no tensor copy can take (rows that do not start on 16-byte boundaries) are gathered by eight further warps
// with plain loads into the same swizzled stages (kGather); everything behind the stages is shared.
//
// What bounds it: the tensor cores for long inputs (2 rows in out operations, 32 KB + 16 KB of operands for each 128 x 256 x
// 64 step); the weights' bytes when an expert has few rows.  BN is chosen by how many turns the tiles take (see product_tile).
#pragma once

#include "nfad_internal.h"
#include "nfad_ops.cuh"
#include "nfad_product_args.h"
#include "nfad_storage.cuh"
#include "nfad_stream.cuh"
#include "nfad_tcgen.cuh"

namespace nfad {

constexpr int kTileRows = 128;
constexpr int kStepBytes = 128;                    // of the reduction, per stage
constexpr int kGatherWarps = 8;
constexpr int kFirstResultWarp = 4;                // a warp reads the 32 tensor-memory lanes of its index modulo 4
constexpr int kRingBytes = 163840;
constexpr int kMaxStages = 9;

template <int OP> struct ProdKind {
    static constexpr bool kBytes = OP == kProdBytes;
    static constexpr bool kScaled = OP == kProdScaled || OP == kProdScaledGated;
    static constexpr bool kGated = OP == kProdGated || OP == kProdScaledGated;                      // half of a tile's columns are a's, half are u's of the same outputs
    static constexpr bool kInput = OP == kProdInput || OP == kProdInputGated;
    static constexpr bool kForward = OP == kProdForward || OP == kProdBytes || kGated || kScaled;
    static constexpr bool kTurnA = OP == kProdWeight;                     // operand A runs along its rows' dimension in memory
    static constexpr bool kTurnB = OP == kProdWeight || kInput;
    static constexpr int kPerResult = kGated ? 2 : 1;                     // a tile's columns for each column of the result
    static constexpr int kElem = kBytes || kScaled ? 1 : 2;
    static constexpr int kStep = kStepBytes / kElem;                      // reduction steps per stage: 64, 128 for bytes
};
template <class S> struct IsBF16 { static constexpr bool value = false; };
template <> struct IsBF16<StoreBF16> { static constexpr bool value = true; };

// kPair: two CTAs share a tile of twice the rows; each holds its own 128 rows of A and half of B's columns
template <int BN, bool kPair> struct ProdTile {
    static constexpr int kRows = kTileRows * (kPair ? 2 : 1);
    static constexpr int kOwnColumns = kPair ? BN / 2 : BN;
    static constexpr int kBoxRows = BN > 64 ? 128 : 32;              // rows of A that one copy brings
    static constexpr int kStage = (kTileRows + kOwnColumns) * kStepBytes;
    static constexpr int kStages = kRingBytes / kStage < kMaxStages ? kRingBytes / kStage : kMaxStages;
};

struct ProdShared {
    uint64_t full[kMaxStages], empty[kMaxStages], landed[kMaxStages], acc_full[2], acc_empty[2], drained;
    uint32_t tmem, gave_up;
    int start[kMaxExperts + 1];                     // first row of each expert
    int tiles[kMaxExperts + 1];                     // row tiles before each expert
};
constexpr int kStageBytes = 32 * 128;             // a result warp's 32 rows of 128 bytes
constexpr int kMostResultWarps = 8;
// The bias and the weights' scales of a result warp's columns, fetched while it waits for the tile: eight packets for each 32 columns
// straight from memory cost a third of the epilogue (8192 x 8192 results of a reduction of 64, bf16, us: without activation 79, now
// 51; GELU-erf and f' 157, now 130; of 1024: 181, now 150).
constexpr int kColumns = 128;
constexpr int kColumnBytes = kColumns * 2 * 4;
// Result warps: beside gathering warps four, whose registers those need.
template <bool kGather> struct ProdWarps {
    static constexpr int kResult = kGather ? 4 : kMostResultWarps;
    static constexpr int kThreads = (kFirstResultWarp + kResult + (kGather ? kGatherWarps : 0)) * 32;
};
constexpr int kProdSmem = 1024 + kRingBytes + kMostResultWarps * (kStageBytes + kColumnBytes) + int(sizeof(ProdShared));

// CTAs one of whose waits ran out; one counter for each translation unit that includes this file
static __device__ unsigned g_product_faults;

struct ProdTileAt {
    uint32_t expert;
    int a0, b0;                                     // first index of the tile along A's and B's own dimension (A: a row or an output)
    int a_end;                                      // end of A's valid indices
    int r0, r_end;                                  // kProdWeight: the reduction's rows; else [0, reduction)
};

// Tile t, for one role's walk over its tiles (t ascending).  Within an expert, bands of kBand tiles along A's dimension, B's tile
// changing slowest inside a band: the CTAs that run at one time then share a few tiles of each operand through L2.  32-bit
// arithmetic throughout: tiles are counted below 2^31 (the launch sees to it), and every role does this once per tile.  Bands of 8, 16
// and 64 tiles, us, 8192 rows 2048 -> 8192 bf16: forward 187, 185, 183; gradient of the input 199, 203, 211; of the weights 221, 221, 228.
constexpr uint32_t kBand = 16;
template <int OP, int BN, bool kPair> struct TileWalk {
    uint32_t b_tiles, expert = 0;
    __device__ __forceinline__ ProdTileAt at(const ProdArgs& g, const int* start, const int* tiles, uint32_t t)
    {
        constexpr int kRows = ProdTile<BN, kPair>::kRows;
        ProdTileAt q;
        uint32_t a_tiles, local;
        if (OP == kProdWeight) {
            a_tiles = (g.outs + kRows - 1) / kRows;
            expert = t / (a_tiles * b_tiles);
            local = t - expert * a_tiles * b_tiles;
        } else {
            while (uint32_t(tiles[expert + 1]) * b_tiles <= t) ++expert;
            a_tiles = tiles[expert + 1] - tiles[expert];
            local = t - uint32_t(tiles[expert]) * b_tiles;
        }
        const uint32_t band = local / (kBand * b_tiles);
        const uint32_t in_band = local - band * kBand * b_tiles;
        const uint32_t height = min(kBand, a_tiles - band * kBand);
        const uint32_t bt = in_band / height, at = band * kBand + in_band - bt * height;
        const int r0 = start[expert], r1 = start[expert + 1];
        q.expert = expert;
        q.b0 = int(bt) * (BN / ProdKind<OP>::kPerResult);
        if (OP == kProdWeight) {
            q.a0 = int(at) * kRows;
            q.a_end = int(g.outs);
            q.r0 = r0;
            q.r_end = r1;
        } else {
            q.a0 = r0 + int(at) * kRows;
            q.a_end = r1;
            q.r0 = 0;
            q.r_end = int(ProdKind<OP>::kInput ? g.outs : g.in);
        }
        return q;
    }
};

// One warp: the experts' row ranges, held inside [0, rows] whatever the offsets say, and the row tiles of kRows before each.
template <int kRows> __device__ __forceinline__ void row_table(const ProdArgs& g, int* start, int* tiles, int lane)
{
    int before = 0, last = 0;
    for (uint32_t e0 = 0; e0 <= g.experts; e0 += 32) {
        const uint32_t e = e0 + lane;
        int first = e < g.experts ? 0 : int(g.rows);
        if (g.offsets && e <= g.experts) first = min(max(__ldg(g.offsets + e), 0), int(g.rows));
        // ranges that run backwards are empty: an expert begins no earlier than the largest offset before it
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, first, o);
            if (lane >= o) first = max(first, v);
        }
        first = max(first, last);
        int prev = __shfl_up_sync(0xffffffffu, first, 1);
        if (lane == 0) prev = e0 ? last : first;
        int n = (first - prev + kRows - 1) / kRows;      // of the expert before this one
        if (e > g.experts) n = 0;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, n, o);
            if (lane >= o) n += v;
        }
        n += before;
        if (e <= g.experts) {
            start[e] = first;
            tiles[e] = n;
        }
        before = __shfl_sync(0xffffffffu, n, 31);
        last = __shfl_sync(0xffffffffu, first, 31);
    }
}

// The weight gradient's last step of an expert: `keep` of its 64 rows are the expert's.  Products are issued by 16 rows, as many as hold one of
// them, so only the rows up to the next multiple of 16 have to be cleared: here, in `runs` boxes of 128-byte rows, by one warp.  (All 64
// cleared and multiplied: 77 us for 61 experts of 67 rows, 1000 x 1416 f16; 46 us for 64 rows each.)
constexpr int kProductRows = 16;
__device__ __forceinline__ void clear_runs(unsigned char* at, int runs, int keep, int lane)
{
    const int end = (keep + kProductRows - 1) / kProductRows * kProductRows * 8;
    for (int j = 0; j < runs; ++j)
        for (int i = keep * 8 + lane; i < end; i += 32) *reinterpret_cast<uint4*>(at + j * 64 * 128 + i * 16) = make_uint4(0, 0, 0, 0);
}

// ---------------------------------------------------------------- gathering without tensor copies

// One operand's 128 (kRows) x 128 bytes of a stage, swizzled as tensor copies would leave them: 1024 packets of 16 bytes, four to a thread.
// Not turned: 128 rows of the operand's own dimension, 128 bytes of the reduction.  Turned: two boxes of 64 reduction steps (128
// for bytes there are none) by 128 bytes along the own dimension.  Elements outside read as zeros.  A packet that starts
// anywhere comes from the two aligned ones that hold it, shifted; at the ends of a row and of the whole operand ([begin, end))
// it comes element by element.  (By ordinary loads, not the read-only path: a kernel in front that has not ended yet when this one begins may
// write either operand.)
struct GatherSource {
    const unsigned char *begin, *end, *at;
    uint32_t pitch;
    int own, own_end, red, red_end;                  // first index and end along the own dimension and along the reduction
    size_t second;                                   // kHalves: bytes from the first half of the box's rows to the second
};
// kHalves: the second half of the box's kRows rows has the first one's indices in another matrix (the two weights of a gated layer)
template <int ES, bool kTurn, bool kHalves = false, int kRows = kTileRows> struct GatherPackets {
    static constexpr int kGatherPackets = kRows * 8 / (kGatherWarps * 32);
    static constexpr int PER = 16 / ES;
    uint4 lo[kGatherPackets], hi[kGatherPackets];
    uint32_t whole;
    // where packet i of the box begins, and how many of its elements there are
    static __device__ __forceinline__ const unsigned char* place(const GatherSource& src, int i, int* n)
    {
        const int row = kTurn ? src.red + ((i & 511) >> 3) : src.own + (kHalves ? i % (kRows * 4) >> 3 : i >> 3), end = kTurn ? src.red_end : src.own_end;
        const int col = kTurn ? src.own + (i >> 9) * (128 / ES) + (i & 7) * PER : src.red + (i & 7) * PER, width = kTurn ? src.own_end : src.red_end;
        *n = row < end ? width - col : 0;
        return src.at + size_t(row) * src.pitch + size_t(col) * ES + (kHalves && i >= kRows * 4 ? src.second : 0);
    }
    __device__ __forceinline__ void load(const GatherSource& src, int thread)
    {
        whole = 0;
#pragma unroll
        for (int j = 0; j < kGatherPackets; ++j) {
            int n;
            const unsigned char* p = place(src, thread + j * kGatherWarps * 32, &n);
            const unsigned char* q = reinterpret_cast<const unsigned char*>(reinterpret_cast<uintptr_t>(p) & ~uintptr_t(15));
            lo[j] = hi[j] = make_uint4(0, 0, 0, 0);
            if (n >= PER && q >= src.begin && q + (p == q ? 16 : 32) <= src.end) {
                whole |= 1u << j;
                lo[j] = *reinterpret_cast<const uint4*>(q);
                if (p != q) hi[j] = reinterpret_cast<const uint4*>(q)[1];
            }
        }
    }
    __device__ __forceinline__ void store(unsigned char* dst, const GatherSource& src, int thread)
    {
#pragma unroll
        for (int j = 0; j < kGatherPackets; ++j) {
            const int i = thread + j * kGatherWarps * 32;
            int n;
            const unsigned char* p = place(src, i, &n);
            uint4 v = make_uint4(0, 0, 0, 0);
            if (whole >> j & 1) {
                // bytes [s, s + 16) of the 32: whole words first, then within the words
                const uint32_t s = uint32_t(reinterpret_cast<uintptr_t>(p)) & 15u, bits = (s & 3u) * 8;
                uint32_t w[8] = {lo[j].x, lo[j].y, lo[j].z, lo[j].w, hi[j].x, hi[j].y, hi[j].z, hi[j].w};
                if (s & 8u) {
#pragma unroll
                    for (int k = 0; k < 6; ++k) w[k] = w[k + 2];
                }
                if (s & 4u) {
#pragma unroll
                    for (int k = 0; k < 5; ++k) w[k] = w[k + 1];
                }
                v = make_uint4(__funnelshift_r(w[0], w[1], bits), __funnelshift_r(w[1], w[2], bits), __funnelshift_r(w[2], w[3], bits), __funnelshift_r(w[3], w[4], bits));
            } else if (n > 0) {
                uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
                for (int e = 0; e < PER; ++e)
                    if (e < n) {
                        if (ES == 2) w[e >> 1] |= uint32_t(reinterpret_cast<const unsigned short*>(p)[e]) << (16 * (e & 1));
                        else w[e >> 2] |= uint32_t(p[e]) << (8 * (e & 3));
                    }
                v = make_uint4(w[0], w[1], w[2], w[3]);
            }
            const int r = i >> 3;
            *reinterpret_cast<uint4*>(dst + r * 128 + (((i & 7) ^ (r & 7)) << 4)) = v;
        }
    }
};

// ---------------------------------------------------------------- epilogue

// a lane's 32 values: z -> y in place (and f' when it is asked for)
template <class K, bool kSlope> __device__ __forceinline__ void act32(float (&z)[32], float (&d)[32])
{
#pragma unroll
    for (int e = 0; e < 32; e += 2) {
        if (kSlope) {
            const ActOut2 o = evaluate(K{}, Fast2{}, make_float2(z[e], z[e + 1]));
            z[e] = o.y.x; z[e + 1] = o.y.y;
            d[e] = o.dydx.x; d[e + 1] = o.dydx.y;
        } else {
            const float2 y = evaluate_value(K{}, Fast2{}, make_float2(z[e], z[e + 1]));
            z[e] = y.x; z[e + 1] = y.y;
        }
    }
}

template <bool kSlope> __device__ __forceinline__ void act32(int kind, float (&z)[32], float (&d)[32])
{
    switch (kind) {
    case kGeluErf:  act32<GeluErf, kSlope>(z, d); break;
    case kGeluTanh: act32<GeluTanh, kSlope>(z, d); break;
    case kSwish:    act32<Swish, kSlope>(z, d); break;
    case kMish:     act32<Mish, kSlope>(z, d); break;
    default: break;                                  // no activation (and then no slope is asked for)
    }
}

// the same for one packet
template <class K, bool kSlope> __device__ __forceinline__ void act8(float (&z)[8], float (&d)[8])
{
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
        if (kSlope) {
            const ActOut2 o = evaluate(K{}, Fast2{}, make_float2(z[e], z[e + 1]));
            z[e] = o.y.x; z[e + 1] = o.y.y;
            d[e] = o.dydx.x; d[e + 1] = o.dydx.y;
        } else {
            const float2 y = evaluate_value(K{}, Fast2{}, make_float2(z[e], z[e + 1]));
            z[e] = y.x; z[e + 1] = y.y;
        }
    }
}
template <bool kSlope> __device__ __forceinline__ void act8(int kind, float (&z)[8], float (&d)[8])
{
    switch (kind) {
    case kGeluErf:  act8<GeluErf, kSlope>(z, d); break;
    case kGeluTanh: act8<GeluTanh, kSlope>(z, d); break;
    case kSwish:    act8<Swish, kSlope>(z, d); break;
    case kMish:     act8<Mish, kSlope>(z, d); break;
    default: break;
    }
}

// eight neighbours of a [*, width] tensor from column c on
template <class S> __device__ __forceinline__ void load8(const void* base, size_t row, uint32_t width, uint32_t c, float (&v)[8])
{
    S::unpack(*reinterpret_cast<const uint4*>(static_cast<const typename S::elem*>(base) + row * width + c), v);
}
template <class S> __device__ __forceinline__ uint4 pack8(const float (&z)[32], int p)
{
    float o[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = z[p * 8 + e];
    return S::pack(o);
}

// A lane holds results of its own row; memory wants whole lines.  So packets of eight go through the warp's 4 KB of shared
// memory: 32 rows of eight packets, their places rotated so that neither side meets bank conflicts.  The eight packets are 64
// neighbouring results (whole 128-byte lines on the way out), or 32 results and their 32 slopes, or 32 factors on the way in.
// (Half rows of two neighbours are read together: the rotation puts them into different halves.)
// Written straight from the rows, every access touched 32 lines, and the stores alone took 5 us a tile.
struct RowPackets {
    int lane, rows;                                 // how many of the warp's 32 rows there are
    uint32_t width;
    size_t row0;                                    // the first one
    size_t pitch;                                   // elements from one row to the next
    uint4* stage;
    static __device__ __forceinline__ int at(int row, int packet) { return row * 8 + (packet ^ (row << 2 & 4 | row >> 1 & 3)); }
    __device__ __forceinline__ void put(int packet, const uint4& v) const { stage[at(lane, packet)] = v; }
    __device__ __forceinline__ uint4 get(int packet) const { return stage[at(lane, packet)]; }
    // Calls f(i, place in the stage, address) for each packet of this lane that is inside: packet lane % kPackets, counted from
    // column `col` and from the stage's packet `first`, of every 32 / kPackets-th row.
    template <class E, int kPackets, class F> __device__ __forceinline__ void each(E* base, uint32_t col, int first, F f) const
    {
        const int r0 = lane / kPackets, c = lane % kPackets;
        if (col + c * 8 >= width) return;
        E* p = base + ((row0 + r0) * pitch + col + c * 8);
        const size_t step = size_t(32 / kPackets) * pitch;
#pragma unroll
        for (int i = 0; i < kPackets; ++i, p += step) {
            const int r = r0 + i * (32 / kPackets);
            if (r < rows) f(i, at(r, first + c), p);
        }
    }
    template <class S, int kPackets> __device__ __forceinline__ void store(void* base, uint32_t col, int first) const
    {
        each<typename S::elem, kPackets>(static_cast<typename S::elem*>(base), col, first,
                                         [&](int, int place, typename S::elem* p) { *reinterpret_cast<uint4*>(p) = stage[place]; });
    }
    // the same where rows start anywhere: kPackets * 8 elements of each row, one by one, neighbours by neighbouring lanes
    template <class S, int kPackets> __device__ __forceinline__ void store_odd(void* base, uint32_t col, int first) const
    {
        using E = typename S::elem;
        E* p = static_cast<E*>(base) + row0 * pitch + col;
        for (int r = 0; r < rows; ++r, p += pitch)
#pragma unroll
            for (int e = lane; e < kPackets * 8; e += 32)
                if (col + e < width) p[e] = reinterpret_cast<const E*>(stage + at(r, first + (e >> 3)))[e & 7];
    }
    template <class S> __device__ __forceinline__ void fetch_odd(const void* base, uint32_t col, int first) const
    {
        using E = typename S::elem;
        const E* p = static_cast<const E*>(base) + row0 * pitch + col;
        for (int r = 0; r < rows; ++r, p += pitch)
            if (col + lane < width) reinterpret_cast<E*>(stage + at(r, first + (lane >> 3)))[lane & 7] = p[lane];
    }
    // four packets of each row, on their way in
    template <class S> __device__ __forceinline__ void fetch(const void* base, uint32_t col, uint4 (&v)[4]) const
    {
        each<const typename S::elem, 4>(static_cast<const typename S::elem*>(base), col, 0,
                                        [&](int i, int, const typename S::elem* p) { v[i] = *reinterpret_cast<const uint4*>(p); });
    }
    // what fetch brought, to the stage's packets from `first` on (values of packets outside are never used)
    __device__ __forceinline__ void settle(const uint4 (&v)[4], int first) const
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) stage[at((lane >> 2) + i * 8, first + (lane & 3))] = v[i];
    }
};

// rows that belong to no expert: zeros (kGated: `slope` has two such rows to each of `out`; kInputGated: `out` does)
template <class S, int kThreads, int OP> __device__ __forceinline__ void clear_rows(const ProdArgs& g, int first, int end, uint32_t result_width, int thread)
{
    const size_t width = OP == kProdInputGated ? size_t(result_width) * 2 : result_width;
    const size_t n0 = size_t(first) * width, n1 = size_t(end) * width;
    for (size_t i = n0 + size_t(blockIdx.x) * kThreads + thread; i < n1; i += size_t(gridDim.x) * kThreads) {
        S::store1(static_cast<typename S::elem*>(g.out) + i, 0.0f);
        if (!ProdKind<OP>::kGated && g.slope) S::store1(static_cast<typename S::elem*>(g.slope) + i, 0.0f);
    }
    if (ProdKind<OP>::kGated && g.slope)
        for (size_t i = 2 * n0 + size_t(blockIdx.x) * kThreads + thread; i < 2 * n1; i += size_t(gridDim.x) * kThreads)
            S::store1(static_cast<typename S::elem*>(g.slope) + i, 0.0f);
}

// ---------------------------------------------------------------- the kernel

template <int OP, int BN, class S, bool kGather, bool kPair>
__global__ void __launch_bounds__(ProdWarps<kGather>::kThreads, 1)
product_kernel(const __grid_constant__ ProdArgs g, const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b)
{
    using Kind = ProdKind<OP>;
    using Tile = ProdTile<BN, kPair>;
    constexpr int kStages = Tile::kStages, kStep = Kind::kStep, kOwn = Tile::kOwnColumns;
    constexpr uint32_t kTmem = 2 * BN;
    constexpr int kBoxRows = Tile::kBoxRows, kResultWarps = ProdWarps<kGather>::kResult;
    extern __shared__ unsigned char raw[];
    unsigned char* ring = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
    ProdShared& s = *reinterpret_cast<ProdShared*>(ring + kRingBytes + kMostResultWarps * (kStageBytes + kColumnBytes));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = kPair ? tc::rank_in_pair() : 0;
    const uint32_t unit = kPair ? blockIdx.x >> 1 : blockIdx.x, units = kPair ? gridDim.x >> 1 : gridDim.x;
    const uint32_t ring_at = tc::shared_address(ring);
    auto full = [&](int i) { return tc::shared_address(&s.full[i]); };
    auto empty = [&](int i) { return tc::shared_address(&s.empty[i]); };
    auto acc_full = [&](int i) { return tc::shared_address(&s.acc_full[i]); };
    auto acc_empty = [&](int i) { return tc::shared_address(&s.acc_empty[i]); };
    auto landed = [&](int i) { return tc::shared_address(&s.landed[i]); };
    volatile uint32_t* gave_up = &s.gave_up;

    if (threadIdx.x == 0) {
        s.gave_up = 0;
        for (int i = 0; i < kStages; ++i) {
            // per stage: both copying warps of each CTA (or every gathering thread); the products' one commit
            tc::barrier_init(full(i), kGather ? kGatherWarps * 32 : kPair ? 4 : 2);
            tc::barrier_init(empty(i), 1);
            tc::barrier_init(landed(i), 2);
        }
        for (int i = 0; i < 2; ++i) {
            tc::barrier_init(acc_full(i), 1);
            tc::barrier_init(acc_empty(i), kResultWarps * (kPair ? 2 : 1));
        }
        tc::barrier_init(tc::shared_address(&s.drained), 1);
        tc::barrier_init_done();
        if (!kGather) {
            tc::prefetch_map(&map_a);
            tc::prefetch_map(&map_b);
        }
    }
    if (warp == 2) tc::tmem_alloc<kPair>(tc::shared_address(&s.tmem), kTmem);
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");

    if (warp == 3) row_table<Tile::kRows>(g, s.start, s.tiles, lane);
    tc::fence_before_sync();
    __syncthreads();
    if (kPair) tc::pair_sync();                      // the other CTA's barriers exist
    tc::fence_after_sync();
    const uint32_t tmem = s.tmem;
    const uint32_t width = Kind::kInput || OP == kProdWeight ? g.in : g.outs;       // of a result's row
    constexpr uint32_t kResults = BN / Kind::kPerResult;                             // a tile's
    TileWalk<OP, BN, kPair> walk;
    walk.b_tiles = (width + kResults - 1) / kResults;
    const uint32_t total = (OP == kProdWeight ? g.experts * ((g.outs + Tile::kRows - 1) / Tile::kRows) : uint32_t(s.tiles[g.experts])) * walk.b_tiles;
    // the last tile along a result's row is a narrower product (a multiple of 16 columns, of 32 for a pair, which halves it)
    auto columns = [&](const ProdTileAt& q) {
        if (Kind::kGated) return uint32_t(BN);       // u's columns keep their place: what lies behind the last output is zeros, times x
        const uint32_t unit_n = kPair ? 32 : 16, left = (width - q.b0 + unit_n - 1) / unit_n * unit_n;
        return left < uint32_t(BN) ? left : uint32_t(BN);
    };
    // a step of the weight gradient whose products reach past the expert's end (gathered operands come without those rows)
    auto ragged = [&](const ProdTileAt& q, int r) { return OP == kProdWeight && !kGather && r + kStep > q.r_end && (q.r_end - r) % kProductRows; };
    // clears those rows in every 128-byte run of this CTA's two operands
    auto clear_ragged = [&](const ProdTileAt& q, int r, uint32_t stage) {
        clear_runs(ring + stage * Tile::kStage, 2 + kOwn / 64, q.r_end - r, lane);
        tc::writes_to_async();
        if (kPair) tc::pair_fence();
        __syncwarp();
    };

    if (!kGather && (warp == 0 || warp == 3)) {
        // ------------------------------------------------ tensor copies into the ring: one thread for A, one for B (issuing a
        // copy takes a thread longer than a pair's product step of 512 cycles leaves for four of them)
        uint32_t stage = 0, phase = 0;
        const bool for_a = warp == 0;
        if (lane == 0)
            for (uint32_t t = unit; t < total; t += units) {
                const ProdTileAt q = walk.at(g, s.start, s.tiles, t);
                const int a0 = q.a0 + int(rank) * kTileRows, b0 = q.b0 + (rank && !Kind::kGated ? int(columns(q)) / 2 : 0);
                const int a_rows = max(0, min(kTileRows, q.a_end - a0));
                const int boxes = (a_rows + kBoxRows - 1) / kBoxRows;     // of A, when it is not turned
                const uint32_t bytes = !for_a ? kOwn * kStepBytes : Kind::kTurnA ? kTileRows * kStepBytes : uint32_t(boxes) * kBoxRows * kStepBytes;
                bool ok = true;
                for (int r = q.r0; r < q.r_end; r += kStep) {
                    if (!(ok = tc::barrier_wait(empty(stage), phase ^ 1, gave_up))) break;
                    const uint32_t at_a = ring_at + stage * Tile::kStage, at_b = at_a + kTileRows * kStepBytes;
                    // a ragged step is announced by the warp that clears it, once it has landed
                    uint32_t bar;
                    if (ragged(q, r)) {
                        bar = landed(stage);
                        tc::barrier_expect(bar, bytes);
                    } else if (kPair) {
                        bar = tc::first_of_pair(full(stage));
                        tc::barrier_expect_first(bar, bytes);
                    } else {
                        bar = full(stage);
                        tc::barrier_expect(bar, bytes);
                    }
                    if (for_a) {
                        if (Kind::kTurnA) {
#pragma unroll
                            for (int j = 0; j < 2; ++j) tc::load_box<kPair>(at_a + j * 64 * 128, &map_a, bar, a0 + j * 64, r);
                        } else {
                            for (int j = 0; j < boxes; ++j) tc::load_box<kPair>(at_a + j * kBoxRows * 128, &map_a, bar, r, a0 + j * kBoxRows);
                        }
                    } else if (OP == kProdWeight) {
#pragma unroll
                        for (int j = 0; j < kOwn / 64; ++j) tc::load_box<kPair>(at_b + j * 64 * 128, &map_b, bar, b0 + j * 64, r);
                    } else if (Kind::kTurnB) {
#pragma unroll
                        for (int j = 0; j < kOwn / 64; ++j) tc::load_box<kPair>(at_b + j * 64 * 128, &map_b, bar, b0 + j * 64, r, int(q.expert));
                    } else if (Kind::kGated) {
                        // a pair's first CTA holds a's columns, the second u's
                        tc::load_box<kPair>(at_b, &map_b, bar, r, b0, int(q.expert * 2 + rank));
                        if (!kPair) tc::load_box<kPair>(at_b + kOwn / 2 * kStepBytes, &map_b, bar, r, b0, int(q.expert * 2 + 1));
                    } else {
                        tc::load_box<kPair>(at_b, &map_b, bar, r, b0, int(q.expert));
                    }
                    if (++stage == kStages) { stage = 0; phase ^= 1; }
                }
                if (!ok) {
                    // a wait ran out: the copies in flight land before the CTA's memory goes away
                    const long long t0 = clock64();
                    while (clock64() - t0 < tc::kWaitDrain) {}
                    break;
                }
            }
    } else if (kGather && warp >= kFirstResultWarp + kResultWarps) {
        // ------------------------------------------------ the same by plain loads
        uint32_t stage = 0, phase = 0;
        bool ok = true;
        for (uint32_t t = unit; t < total && ok; t += units) {
            const ProdTileAt q = walk.at(g, s.start, s.tiles, t);
            static_assert(!kGather || BN == kTileRows, "both operands' boxes are 128 by 128 bytes");
            constexpr int ES = Kind::kElem;
            const int thread = threadIdx.x - (kFirstResultWarp + kResultWarps) * 32;
            GatherSource a, b;
            a.pitch = (Kind::kInput || OP == kProdWeight ? g.outs : g.in) * ES;
            b.pitch = g.in * ES;
            b.second = size_t(g.outs) * b.pitch;
            const size_t weight = Kind::kPerResult * b.second;                    // bytes of an expert's
            a.begin = a.at = static_cast<const unsigned char*>(g.a);
            a.end = a.begin + g.rows * a.pitch;
            a.own = q.a0;
            a.own_end = q.a_end;
            b.begin = static_cast<const unsigned char*>(g.b);
            b.end = b.begin + (OP == kProdWeight ? g.rows * b.pitch : g.experts * weight);
            b.at = b.begin + (OP == kProdWeight ? 0 : q.expert * weight);
            b.own = q.b0;
            b.own_end = int(width);
            a.red_end = b.red_end = q.r_end;
            for (int r = q.r0; r < q.r_end; r += kStep) {
                a.red = b.red = r;
                // requested before the stage is free, so that the wait covers the loads
                GatherPackets<ES, Kind::kTurnA> pa;
                GatherPackets<ES, Kind::kTurnB, Kind::kGated> pb;
                pa.load(a, thread);
                pb.load(b, thread);
                if (!(ok = tc::barrier_wait(empty(stage), phase ^ 1, gave_up))) break;
                unsigned char* at = ring + stage * Tile::kStage;
                pa.store(at, a, thread);
                pb.store(at + kTileRows * kStepBytes, b, thread);
                tc::writes_to_async();
                tc::barrier_arrive(full(stage));
                if (++stage == kStages) { stage = 0; phase ^= 1; }
            }
        }
    } else if (warp == 1 && rank == 0) {
        // ------------------------------------------------ products
        // By one elected lane of a warp that goes through the steps together, and looks at a barrier before it sleeps: 16384 rows 2048 -> 8192
        // bf16, against lane 0 and a sleeping wait (us): with GELU-erf and f' 373 (416), gradient of the input 340 (347), of the weights 369
        // (444), in 8 bits 179 (192).
        const bool leader = tc::elected();
        uint32_t stage = 0, phase = 0, turn = 0, turn_phase = 0, landed_phases = 0;              // landed_phases: a bit for each stage
        bool ok = true;
        for (uint32_t t = unit; t < total && ok; t += units) {
            const ProdTileAt q = walk.at(g, s.start, s.tiles, t);
            if (!(ok = tc::barrier_wait(acc_empty(turn), turn_phase ^ 1, gave_up))) break;
            tc::fence_after_sync();
            const uint32_t what = tc::instruction(Kind::kBytes ? tc::kNumberS8 : IsBF16<S>::value ? tc::kNumberBF16 : tc::kNumberF16, Kind::kTurnA, Kind::kTurnB,
                                                  Tile::kRows, columns(q));
            for (int r = q.r0; r < q.r_end; r += kStep) {
                if (ragged(q, r)) {
                    if (!(ok = tc::barrier_wait(landed(stage), landed_phases >> stage & 1, gave_up))) break;
                    landed_phases ^= 1u << stage;
                    clear_ragged(q, r, stage);
                    if (lane < 2) tc::barrier_arrive(full(stage));       // in the copying threads' place
                }
                if (!(ok = tc::barrier_poll(full(stage), phase, gave_up))) break;
                if (kPair && ragged(q, r)) {
                    tc::pair_fence();
                    tc::writes_to_async();
                }
                tc::fence_after_sync();
                const uint32_t at_a = ring_at + stage * Tile::kStage, at_b = at_a + kTileRows * kStepBytes;
                if (leader) {
#pragma unroll
                    for (int k = 0; k < kStepBytes / 32; ++k) {
                        if (OP == kProdWeight && k * kProductRows >= q.r_end - r) break;
                        // 32 bytes of the reduction: along the 128-byte rows, or 16 reduction steps of 128 bytes further
                        const uint64_t da = Kind::kTurnA ? tc::operand(at_a + k * 2048, 64 * 128, 1024) : tc::operand(at_a + k * 32, 16, 1024);
                        const uint64_t db = Kind::kTurnB ? tc::operand(at_b + k * 2048, 64 * 128, 1024) : tc::operand(at_b + k * 32, 16, 1024);
                        tc::product<Kind::kBytes, kPair>(tmem + turn * BN, da, db, what, r > q.r0 || k > 0);
                    }
                    tc::products_to<kPair>(empty(stage));
                }
                __syncwarp();
                if (++stage == kStages) { stage = 0; phase ^= 1; }
            }
            if (leader && ok) tc::products_to<kPair>(acc_full(turn));
            __syncwarp();
            turn ^= 1;
            if (turn == 0) turn_phase ^= 1;
        }
        if (!ok && leader) {
            tc::products_to<kPair>(tc::shared_address(&s.drained));
            const long long t0 = clock64();
            while (!tc::barrier_try(tc::shared_address(&s.drained), 0) && clock64() - t0 < tc::kWaitDrain) {}
        }
    } else if (warp == 1 && OP == kProdWeight) {
        // ------------------------------------------------ the second CTA's ragged steps
        uint32_t stage = 0, landed_phases = 0;
        bool ok = true;
        for (uint32_t t = unit; t < total && ok; t += units) {
            const ProdTileAt q = walk.at(g, s.start, s.tiles, t);
            for (int r = q.r0; r < q.r_end; r += kStep) {
                if (ragged(q, r)) {
                    if (!(ok = tc::barrier_wait(landed(stage), landed_phases >> stage & 1, gave_up))) break;
                    landed_phases ^= 1u << stage;
                    clear_ragged(q, r, stage);
                    if (lane < 2) tc::barrier_arrive_first(tc::first_of_pair(full(stage)));
                }
                if (++stage == kStages) stage = 0;
            }
        }
    } else if (warp >= kFirstResultWarp && warp < kFirstResultWarp + kResultWarps) {
        // ------------------------------------------------ results
        const int lanes = (warp & 3) * 32, half = (warp - kFirstResultWarp) >> 2;
        if (OP != kProdWeight && g.offsets) {
            clear_rows<S, kResultWarps * 32, OP>(g, 0, s.start[0], width, threadIdx.x - kFirstResultWarp * 32);
            clear_rows<S, kResultWarps * 32, OP>(g, s.start[g.experts], int(g.rows), width, threadIdx.x - kFirstResultWarp * 32);
        }
        // whole 16-byte packets: rows start on packets and no packet crosses a row's end
        const bool vec = width % 8 == 0 && ((reinterpret_cast<uintptr_t>(g.out) | reinterpret_cast<uintptr_t>(g.slope) | reinterpret_cast<uintptr_t>(g.prev)) & 15u) == 0;
        float* columns = reinterpret_cast<float*>(ring + kRingBytes + kMostResultWarps * kStageBytes + (warp - kFirstResultWarp) * kColumnBytes);
        uint32_t turn = 0, turn_phase = 0;
        for (uint32_t t = unit; t < total; t += units) {
            const ProdTileAt q = walk.at(g, s.start, s.tiles, t);
            const int row = q.a0 + int(rank) * kTileRows + lanes + lane;
            const bool mine = row < q.a_end, none = q.r0 >= q.r_end;
            const size_t out_row = OP == kProdWeight ? size_t(q.expert) * g.outs + row : size_t(row);
            const float scale = Kind::kBytes && mine ? g.a_scale[row] : 0.0f;
            RowPackets rows;
            rows.lane = lane;
            rows.rows = min(32, q.a_end - (row - lane));
            rows.width = width;
            rows.pitch = OP == kProdInputGated ? size_t(width) * 2 : width;
            rows.row0 = out_row - lane;
            rows.stage = reinterpret_cast<uint4*>(ring + kRingBytes + (warp - kFirstResultWarp) * kStageBytes);
            // 32 columns at a time; without slopes two of them leave together; the factors of the next are fetched during the current
            constexpr int kChunks = kResults / 32, kOwnChunks = kChunks / (kResultWarps / 4);
            static_assert(kOwnChunks > 0, "results for every result warp");
            constexpr bool kTwo = kOwnChunks > 1;
            const bool slopes = (OP == kProdForward || Kind::kGated) && g.slope;
            uint4 prev[4] = {}, prev_u[4] = {};
            if constexpr (OP == kProdInputGated)
                if (vec) {
                    rows.template fetch<S>(g.prev, q.b0 + half * kOwnChunks * 32, prev);
                    rows.template fetch<S>(static_cast<const typename S::elem*>(g.prev) + width, q.b0 + half * kOwnChunks * 32, prev_u);
                }
            if (OP == kProdInput && g.prev && vec) rows.template fetch<S>(g.prev, q.b0 + half * kOwnChunks * 32, prev);
            if constexpr (Kind::kForward) {
                static_assert(kOwnChunks * 32 <= kColumns, "a result warp's columns");
                float bias[kOwnChunks], scales[kOwnChunks];           // kGated: a's bias and u's
#pragma unroll
                for (int j = 0; j < kOwnChunks; ++j) {
                    const uint32_t col = q.b0 + (half * kOwnChunks + j) * 32 + lane;
                    const bool inside = col < width;
                    const typename S::elem* own = static_cast<const typename S::elem*>(g.bias) + size_t(q.expert) * width * Kind::kPerResult + col;
                    bias[j] = g.bias && inside ? S::load1(own) : 0.0f;
                    if (Kind::kGated) scales[j] = g.bias && inside ? S::load1(own + width) : 0.0f;
                    else scales[j] = Kind::kBytes && inside ? g.b_scale[col] : 0.0f;
                }
#pragma unroll
                for (int j = 0; j < kOwnChunks; ++j) {
                    columns[j * 32 + lane] = bias[j];
                    if (Kind::kBytes || Kind::kGated) columns[kColumns + j * 32 + lane] = scales[j];
                }
                __syncwarp();
            }
            if (!tc::barrier_wait(acc_full(turn), turn_phase, gave_up)) break;
            tc::fence_after_sync();
            for (int c = half * kOwnChunks; c < (half + 1) * kOwnChunks; ++c) {
                const uint32_t col0 = q.b0 + c * 32;
                if (col0 >= width || rows.rows <= 0) break;     // past the result's columns; a warp without rows
                const bool second = kTwo && !slopes && OP != kProdInputGated && (c & 1);
                uint32_t v[32];
                tc::tmem_load32(tmem + (uint32_t(lanes) << 16) + turn * BN + c * 32, v);
                if constexpr (Kind::kGated) {
                    const float4* own = reinterpret_cast<const float4*>(columns) + (c - half * kOwnChunks) * 8;
                    uint32_t w[32];
                    tc::tmem_load32(tmem + (uint32_t(lanes) << 16) + turn * BN + kResults + c * 32, w);
                    tc::tmem_load_wait();
                    float z[32], u[32], d[32];
#pragma unroll
                    for (int p = 0; p < 8; ++p) {
                        const float4 ba = own[p], bu = own[kColumns / 4 + p];
                        const float add_a[4] = {ba.x, ba.y, ba.z, ba.w}, add_u[4] = {bu.x, bu.y, bu.z, bu.w};
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const int e = p * 4 + k;
                            z[e] = (none ? 0.0f : __uint_as_float(v[e])) + add_a[k];
                            u[e] = (none ? 0.0f : __uint_as_float(w[e])) + add_u[k];
                            d[e] = 1.0f;             // of no activation
                        }
                    }
                    if (slopes) {
                        act32<true>(g.act, z, d);
#pragma unroll
                        for (int e = 0; e < 32; ++e) d[e] *= u[e];
#pragma unroll
                        for (int e = 0; e < 32; ++e) u[e] *= z[e];
#pragma unroll
                        for (int p = 0; p < 4; ++p) {
                            rows.put(p, pack8<S>(u, p));
                            rows.put(4 + p, pack8<S>(d, p));
                        }
                        __syncwarp();
                        RowPackets both = rows;      // the derivatives' rows
                        both.pitch = size_t(width) * 2;
                        typename S::elem* by_u = static_cast<typename S::elem*>(g.slope) + width;
                        if (vec) {
                            rows.template store<S, 4>(g.out, col0, 0);
                            both.template store<S, 4>(g.slope, col0, 4);
                        } else {
                            rows.template store_odd<S, 4>(g.out, col0, 0);
                            both.template store_odd<S, 4>(g.slope, col0, 4);
                        }
                        __syncwarp();
#pragma unroll
                        for (int p = 0; p < 4; ++p) rows.put(p, pack8<S>(z, p));
                        __syncwarp();
                        if (vec) both.template store<S, 4>(by_u, col0, 0);
                        else both.template store_odd<S, 4>(by_u, col0, 0);
                        __syncwarp();
                        continue;
                    }
                    act32<false>(g.act, z, d);
#pragma unroll
                    for (int e = 0; e < 32; ++e) u[e] *= z[e];
#pragma unroll
                    for (int p = 0; p < 4; ++p) rows.put((second ? 4 : 0) + p, pack8<S>(u, p));
                    if (kTwo && !second && c + 1 < (half + 1) * kOwnChunks && col0 + 32 < width) continue;
                    __syncwarp();
                    if (kTwo && second) {
                        if (vec) rows.template store<S, 8>(g.out, col0 - 32, 0);
                        else rows.template store_odd<S, 8>(g.out, col0 - 32, 0);
                    } else {
                        if (vec) rows.template store<S, 4>(g.out, col0, 0);
                        else rows.template store_odd<S, 4>(g.out, col0, 0);
                    }
                    __syncwarp();
                    continue;
                }
                tc::tmem_load_wait();
                float z[32], d[32];
#pragma unroll
                for (int e = 0; e < 32; ++e) z[e] = Kind::kBytes ? float(int(v[e])) : __uint_as_float(v[e]);
                if (none)
#pragma unroll
                    for (int e = 0; e < 32; ++e) z[e] = 0.0f;
                const float4* own = reinterpret_cast<const float4*>(columns) + (c - half * kOwnChunks) * 8;
                if (Kind::kBytes) {
#pragma unroll
                    for (int p = 0; p < 8; ++p) {
                        const float4 w = own[kColumns / 4 + p];
                        z[p * 4] *= scale * w.x; z[p * 4 + 1] *= scale * w.y; z[p * 4 + 2] *= scale * w.z; z[p * 4 + 3] *= scale * w.w;
                    }
                }
                if ((OP == kProdForward || OP == kProdBytes) && g.bias) {
#pragma unroll
                    for (int p = 0; p < 8; ++p) {
                        const float4 b = own[p];
                        z[p * 4] += b.x; z[p * 4 + 1] += b.y; z[p * 4 + 2] += b.z; z[p * 4 + 3] += b.w;
                    }
                }
                if (OP == kProdInput && g.prev) {
                    const int first = second ? 4 : 0;                 // the places that this chunk's results will take
                    if (vec) rows.settle(prev, first);
                    else rows.template fetch_odd<S>(g.prev, col0, first);
                    __syncwarp();
                    if (vec && c + 1 < (half + 1) * kOwnChunks) rows.template fetch<S>(g.prev, col0 + 32, prev);
#pragma unroll
                    for (int p = 0; p < 4; ++p) {
                        float f[8];
                        S::unpack(rows.get(first + p), f);
#pragma unroll
                        for (int e = 0; e < 8; ++e) z[p * 8 + e] *= f[e];
                    }
                    __syncwarp();
                }
                if constexpr (OP == kProdInputGated) {
                    // both factors in, both products out, through this lane's own places
                    typename S::elem* by_u = static_cast<typename S::elem*>(g.out) + width;
                    const typename S::elem* prev_by_u = static_cast<const typename S::elem*>(g.prev) + width;
                    if (vec) {
                        rows.settle(prev, 0);
                        rows.settle(prev_u, 4);
                    } else {
                        rows.template fetch_odd<S>(g.prev, col0, 0);
                        rows.template fetch_odd<S>(prev_by_u, col0, 4);
                    }
                    __syncwarp();
                    if (vec && c + 1 < (half + 1) * kOwnChunks) {
                        rows.template fetch<S>(g.prev, col0 + 32, prev);
                        rows.template fetch<S>(prev_by_u, col0 + 32, prev_u);
                    }
#pragma unroll
                    for (int p = 0; p < 8; ++p) {
                        float f[8];
                        S::unpack(rows.get(p), f);
#pragma unroll
                        for (int e = 0; e < 8; ++e) f[e] *= z[(p & 3) * 8 + e];
                        rows.put(p, S::pack(f));
                    }
                    __syncwarp();
                    if (vec) {
                        rows.template store<S, 4>(g.out, col0, 0);
                        rows.template store<S, 4>(by_u, col0, 4);
                    } else {
                        rows.template store_odd<S, 4>(g.out, col0, 0);
                        rows.template store_odd<S, 4>(by_u, col0, 4);
                    }
                    __syncwarp();
                    continue;
                }
                if constexpr (OP == kProdForward) {
                    if (slopes) act32<true>(g.act, z, d);
                    else act32<false>(g.act, z, d);
                } else if constexpr (OP == kProdBytes) {
                    act32<false>(g.act, z, d);
                }
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    rows.put((second ? 4 : 0) + p, pack8<S>(z, p));
                    if (OP == kProdForward && slopes) rows.put(4 + p, pack8<S>(d, p));
                }
                if (kTwo && !slopes && !second && c + 1 < (half + 1) * kOwnChunks && col0 + 32 < width) continue;   // the next 32 first
                __syncwarp();
                if (kTwo && second) {
                    if (vec) rows.template store<S, 8>(g.out, col0 - 32, 0);
                    else rows.template store_odd<S, 8>(g.out, col0 - 32, 0);
                } else {
                    if (vec) rows.template store<S, 4>(g.out, col0, 0);
                    else rows.template store_odd<S, 4>(g.out, col0, 0);
                    if (OP == kProdForward && slopes) {
                        if (vec) rows.template store<S, 4>(g.slope, col0, 4);
                        else rows.template store_odd<S, 4>(g.slope, col0, 4);
                    }
                }
                __syncwarp();
            }
            tc::fence_before_sync();
            __syncwarp();
            if (lane == 0) {
                if (kPair) tc::barrier_arrive_first(tc::first_of_pair(acc_empty(turn)));
                else tc::barrier_arrive(acc_empty(turn));
            }
            turn ^= 1;
            if (turn == 0) turn_phase ^= 1;
        }
    }
    __syncwarp();
    tc::fence_before_sync();
    __syncthreads();
    if (kPair) tc::pair_sync();                      // nothing of the pair arrives on this CTA's barriers or reads its memory any more
    tc::fence_after_sync();
    if (warp == 2) tc::tmem_free<kPair>(tmem, kTmem);
    if (threadIdx.x == 0 && s.gave_up) atomicAdd(&g_product_faults, 1u);
}

}  // namespace nfad
