// nfad_scaled.cuh -- matrix products in 8-bit floating point (four exponent bits, three of the significand) whose operands carry a scale for
// each block of 128 along the reduction: z[m, o] = sum_b sx[b, m] sw[o / 128, b] sum_{k in block b} xq[m, k] wq[o, k], then the epilogues of
// the other products, plain or gated.
//
// A stage of the ring holds 128 bytes of the reduction: one block.  So a step's products (four of 32) start from zero in a buffer of
// tensor memory of their own, and the result warps take every step's buffer, times its scale, into sums that stay in their registers:
// 128 columns of a row to a thread, as 64 pairs of packed multiply-adds.  Two buffers of 256 columns (four of 128) let the products
// run ahead.  The copying and issuing warps give registers to the result warps (setmaxnreg), which hold their sums, a chunk of 32
// on its way and the next.
//
// Roles, tiles, pairs of CTAs, the walk over tiles and the gather for rows off the 16-byte boundaries are those of nfad_product.cuh.
// Each step costs a result warp's reads of its share of tensor memory (128 columns: 128 cycles of an SM quarter) and as many
// multiply-adds, beside 512 cycles of a pair's products.
#pragma once

#include "nfad_product.cuh"

namespace nfad {

constexpr int kScaleBlock = 128;

template <bool kGather> struct ScaledWarps {
    static constexpr int kResult = kGather ? 4 : 8;
    static constexpr int kThreads = (kFirstResultWarp + kResult + (kGather ? kGatherWarps : 0)) * 32;
};

struct ScaledShared {
    uint64_t full[kMaxStages], empty[kMaxStages], acc_full[4], acc_empty[4], drained;
    uint32_t tmem, gave_up;
    int start[2], tiles[2];
};
constexpr int kScaledSmem = 1024 + kRingBytes + kMostResultWarps * kStageBytes + int(sizeof(ScaledShared));

// 64 pairs of sums += 32 columns of a buffer at a time: the next chunk is on its way while one is added
template <int kColumns> __device__ __forceinline__ void add_chunk(float2 (&acc)[kColumns / 2], int chunk, const uint32_t (&v)[32], float scale)
{
    const float2 s = make_float2(scale, scale);
#pragma unroll
    for (int i = 0; i < 16; ++i)
        acc[chunk * 16 + i] = hw::fma2(make_float2(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1])), s, acc[chunk * 16 + i]);
}

template <int OP, int BN, class S, bool kGather, bool kPair>
__global__ void __launch_bounds__(ScaledWarps<kGather>::kThreads, 1)
scaled_kernel(const __grid_constant__ ProdArgs g, const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b)
{
    using Kind = ProdKind<OP>;
    using Tile = ProdTile<BN, kPair>;
    static_assert(Kind::kScaled && Kind::kStep == kScaleBlock, "a stage is a block");
    constexpr int kStages = Tile::kStages, kStep = Kind::kStep, kOwn = Tile::kOwnColumns;
    constexpr int kBuffers = BN > 128 ? 2 : 4;
    constexpr uint32_t kTmem = kBuffers * BN, kResults = BN / Kind::kPerResult;
    constexpr int kBoxRows = Tile::kBoxRows, kResultWarps = ScaledWarps<kGather>::kResult;
    constexpr int kColumns = BN / (kResultWarps / 4), kChunks = kColumns / 32;            // a result warp's
    constexpr bool kMoveRegisters = BN > 128;        // 168 a thread at launch: 40 for four warps leave 232 for the other eight
    extern __shared__ unsigned char raw[];
    unsigned char* ring = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
    ScaledShared& s = *reinterpret_cast<ScaledShared*>(ring + kRingBytes + kMostResultWarps * kStageBytes);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = kPair ? tc::rank_in_pair() : 0;
    const uint32_t unit = kPair ? blockIdx.x >> 1 : blockIdx.x, units = kPair ? gridDim.x >> 1 : gridDim.x;
    const uint32_t ring_at = tc::shared_address(ring);
    auto full = [&](int i) { return tc::shared_address(&s.full[i]); };
    auto empty = [&](int i) { return tc::shared_address(&s.empty[i]); };
    auto acc_full = [&](int i) { return tc::shared_address(&s.acc_full[i]); };
    auto acc_empty = [&](int i) { return tc::shared_address(&s.acc_empty[i]); };
    volatile uint32_t* gave_up = &s.gave_up;

    if (threadIdx.x == 0) {
        s.gave_up = 0;
        for (int i = 0; i < kStages; ++i) {
            // per stage: both copying threads of each CTA (or every gathering thread); the products' one commit
            tc::barrier_init(full(i), kGather ? kGatherWarps * 32 : kPair ? 4 : 2);
            tc::barrier_init(empty(i), 1);
        }
        for (int i = 0; i < kBuffers; ++i) {
            tc::barrier_init(acc_full(i), 1);
            tc::barrier_init(acc_empty(i), kResultWarps * (kPair ? 2 : 1));
        }
        tc::barrier_init(tc::shared_address(&s.drained), 1);
        tc::barrier_init_done();
        if (!kGather) {
            tc::prefetch_map(&map_a);
            tc::prefetch_map(&map_b);
        }
        s.start[0] = 0;
        s.start[1] = int(g.rows);
        s.tiles[0] = 0;
        s.tiles[1] = (int(g.rows) + Tile::kRows - 1) / Tile::kRows;
    }
    if (warp == 2) tc::tmem_alloc<kPair>(tc::shared_address(&s.tmem), kTmem);
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    tc::fence_before_sync();
    __syncthreads();
    if (kPair) tc::pair_sync();                      // the other CTA's barriers exist
    tc::fence_after_sync();
    const uint32_t tmem = s.tmem, width = g.outs, blocks = (g.in + kScaleBlock - 1) / kScaleBlock;
    TileWalk<OP, BN, kPair> walk;
    walk.b_tiles = (width + kResults - 1) / kResults;
    const uint32_t total = uint32_t(s.tiles[1]) * walk.b_tiles;
    auto columns = [&](const ProdTileAt& q) {
        if (Kind::kGated) return uint32_t(BN);
        const uint32_t unit_n = kPair ? 32 : 16, left = (width - q.b0 + unit_n - 1) / unit_n * unit_n;
        return left < uint32_t(BN) ? left : uint32_t(BN);
    };
    if (warp < kFirstResultWarp) {
        if (kMoveRegisters) asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
        if (!kGather && (warp == 0 || warp == 3)) {
            // ------------------------------------------------ tensor copies into the ring: one thread for A, one for B
            uint32_t stage = 0, phase = 0;
            const bool for_a = warp == 0;
            if (lane == 0)
                for (uint32_t t = unit; t < total; t += units) {
                    const ProdTileAt q = walk.at(g, s.start, s.tiles, t);
                    const int a0 = q.a0 + int(rank) * kTileRows, b0 = q.b0 + (rank && !Kind::kGated ? int(columns(q)) / 2 : 0);
                    const int a_rows = max(0, min(kTileRows, q.a_end - a0)), boxes = (a_rows + kBoxRows - 1) / kBoxRows;
                    const uint32_t bytes = for_a ? uint32_t(boxes) * kBoxRows * kStepBytes : kOwn * kStepBytes;
                    bool ok = true;
                    for (int r = 0; r < q.r_end; r += kStep) {
                        if (!(ok = tc::barrier_wait(empty(stage), phase ^ 1, gave_up))) break;
                        const uint32_t at_a = ring_at + stage * Tile::kStage, at_b = at_a + kTileRows * kStepBytes;
                        uint32_t bar = full(stage);
                        if (kPair) {
                            bar = tc::first_of_pair(bar);
                            tc::barrier_expect_first(bar, bytes);
                        } else {
                            tc::barrier_expect(bar, bytes);
                        }
                        if (for_a) {
                            for (int j = 0; j < boxes; ++j) tc::load_box<kPair>(at_a + j * kBoxRows * 128, &map_a, bar, r, a0 + j * kBoxRows);
                        } else if (Kind::kGated) {
                            tc::load_box<kPair>(at_b, &map_b, bar, r, b0, int(rank));
                            if (!kPair) tc::load_box<kPair>(at_b + kOwn / 2 * kStepBytes, &map_b, bar, r, b0, 1);
                        } else {
                            tc::load_box<kPair>(at_b, &map_b, bar, r, b0, 0);
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
        } else if (warp == 1 && rank == 0) {
            // ------------------------------------------------ products: a buffer for each step
            uint32_t stage = 0, phase = 0, turn = 0, turn_phase = 0;
            bool ok = true;
            for (uint32_t t = unit; t < total && ok; t += units) {
                const ProdTileAt q = walk.at(g, s.start, s.tiles, t);
                const uint32_t what = tc::instruction(tc::kNumberE4M3, false, false, Tile::kRows, columns(q));
                for (int r = 0; r < q.r_end; r += kStep) {
                    if (!(ok = tc::barrier_wait(acc_empty(turn), turn_phase ^ 1, gave_up))) break;
                    if (!(ok = tc::barrier_wait(full(stage), phase, gave_up))) break;
                    tc::fence_after_sync();
                    const uint32_t at_a = ring_at + stage * Tile::kStage, at_b = at_a + kTileRows * kStepBytes;
                    if (lane == 0) {
#pragma unroll
                        for (int k = 0; k < kStepBytes / 32; ++k)
                            tc::product_e4m3<kPair>(tmem + turn * BN, tc::operand(at_a + k * 32, 16, 1024), tc::operand(at_b + k * 32, 16, 1024), what, k > 0);
                        tc::products_to<kPair>(empty(stage));
                        tc::products_to<kPair>(acc_full(turn));
                    }
                    __syncwarp();
                    if (++stage == kStages) { stage = 0; phase ^= 1; }
                    if (++turn == kBuffers) { turn = 0; turn_phase ^= 1; }
                }
            }
            if (!ok && lane == 0) {
                tc::products_to<kPair>(tc::shared_address(&s.drained));
                const long long t0 = clock64();
                while (!tc::barrier_try(tc::shared_address(&s.drained), 0) && clock64() - t0 < tc::kWaitDrain) {}
            }
        }
    } else if (warp < kFirstResultWarp + kResultWarps) {
        if (kMoveRegisters) asm volatile("setmaxnreg.inc.sync.aligned.u32 232;");
        // ------------------------------------------------ results
        const int lanes = (warp & 3) * 32, half = (warp - kFirstResultWarp) >> 2;
        const bool vec = width % 8 == 0 && (reinterpret_cast<uintptr_t>(g.out) & 15u) == 0;
        constexpr int kOut = kColumns / Kind::kPerResult;                    // this warp's results of a row, from half kOut on
        // chunk c's first column in a buffer: a gated warp has columns of a first, then those of u
        auto column = [&](int c) { return Kind::kGated && c >= kChunks / 2 ? kResults + half * kOut + (c - kChunks / 2) * 32 : half * kOut + c * 32; };
        uint32_t turn = 0, turn_phase = 0;
        for (uint32_t t = unit; t < total; t += units) {
            const ProdTileAt q = walk.at(g, s.start, s.tiles, t);
            const int row = q.a0 + int(rank) * kTileRows + lanes + lane;
            RowPackets rows;
            rows.lane = lane;
            rows.rows = min(32, q.a_end - (row - lane));
            rows.width = width;
            rows.pitch = width;
            rows.row0 = size_t(row - lane);
            rows.stage = reinterpret_cast<uint4*>(ring + kRingBytes + (warp - kFirstResultWarp) * kStageBytes);
            const uint32_t first = q.b0 + half * kOut;                        // of this warp's results: all in one block of outputs
            float2 acc[kColumns / 2];
#pragma unroll
            for (int i = 0; i < kColumns / 2; ++i) acc[i] = make_float2(0.0f, 0.0f);
            // scales, one block ahead; a row or column outside has any valid one's, for sums that nobody uses
            const float* sx = g.a_scale + min(row, int(g.rows) - 1);
            const float* sw = g.b_scale + size_t(min(first, width - 1) / kScaleBlock) * blocks;
            const size_t second = size_t((width + kScaleBlock - 1) / kScaleBlock) * blocks;
            float next_x = 0.0f, next_a = 0.0f, next_u = 0.0f;
            auto request = [&](uint32_t b) {
                if (b >= blocks) return;
                next_x = __ldg(sx + size_t(b) * g.rows);
                next_a = __ldg(sw + b);
                if (Kind::kGated) next_u = __ldg(sw + second + b);
            };
            request(0);
            bool ok = true;
            for (uint32_t b = 0; b < blocks; ++b) {
                const float scale = next_x * next_a, scale_u = next_x * next_u;
                request(b + 1);
                if (!(ok = tc::barrier_wait(acc_full(turn), turn_phase, gave_up))) break;
                tc::fence_after_sync();
                const uint32_t at = tmem + (uint32_t(lanes) << 16) + turn * BN;
                uint32_t v[2][32];
                tc::tmem_load32(at + column(0), v[0]);
#pragma unroll
                for (int c = 0; c < kChunks; ++c) {
                    tc::tmem_load_wait(v[c & 1]);
                    if (c + 1 < kChunks) tc::tmem_load32(at + column(c + 1), v[(c + 1) & 1]);
                    else {
                        // everything of this buffer is in registers
                        tc::fence_before_sync();
                        __syncwarp();
                        if (lane == 0) {
                            if (kPair) tc::barrier_arrive_first(tc::first_of_pair(acc_empty(turn)));
                            else tc::barrier_arrive(acc_empty(turn));
                        }
                    }
                    add_chunk<kColumns>(acc, c, v[c & 1], Kind::kGated && c >= kChunks / 2 ? scale_u : scale);
                }
                if (++turn == kBuffers) { turn = 0; turn_phase ^= 1; }
            }
            if (!ok) break;
            // 32 results at a time; two of them leave together
            constexpr int kOutChunks = kOut / 32;
#pragma unroll
            for (int c = 0; c < kOutChunks; ++c) {
                const uint32_t col0 = first + c * 32;
                if (col0 >= width || rows.rows <= 0) break;
                float z[32], d[32];
                const uint32_t col = col0 + lane;
                const typename S::elem* bias = static_cast<const typename S::elem*>(g.bias) + col;
                const float own = g.bias && col < width ? S::load1(bias) : 0.0f;
#pragma unroll
                for (int e = 0; e < 32; ++e) z[e] = (e & 1 ? acc[c * 16 + e / 2].y : acc[c * 16 + e / 2].x) + __shfl_sync(0xffffffffu, own, e);
                act32<false>(g.act, z, d);
                if constexpr (Kind::kGated) {
                    const float own_u = g.bias && col < width ? S::load1(bias + width) : 0.0f;
                    constexpr int u0 = kChunks / 2 * 16;
#pragma unroll
                    for (int e = 0; e < 32; ++e)
                        z[e] *= (e & 1 ? acc[u0 + c * 16 + e / 2].y : acc[u0 + c * 16 + e / 2].x) + __shfl_sync(0xffffffffu, own_u, e);
                }
                const bool odd = c & 1;
#pragma unroll
                for (int p = 0; p < 4; ++p) rows.put((odd ? 4 : 0) + p, pack8<S>(z, p));
                if (!odd && c + 1 < kOutChunks && col0 + 32 < width) continue;                // the next 32 first
                __syncwarp();
                if (odd) {
                    if (vec) rows.template store<S, 8>(g.out, col0 - 32, 0);
                    else rows.template store_odd<S, 8>(g.out, col0 - 32, 0);
                } else {
                    if (vec) rows.template store<S, 4>(g.out, col0, 0);
                    else rows.template store_odd<S, 4>(g.out, col0, 0);
                }
                __syncwarp();
            }
        }
    } else if (kGather) {
        // ------------------------------------------------ the same by plain loads
        uint32_t stage = 0, phase = 0;
        bool ok = true;
        for (uint32_t t = unit; t < total && ok; t += units) {
            const ProdTileAt q = walk.at(g, s.start, s.tiles, t);
            const int thread = threadIdx.x - (kFirstResultWarp + kResultWarps) * 32;
            GatherSource a, b;
            a.pitch = b.pitch = g.in;
            b.second = size_t(g.outs) * g.in;
            a.begin = a.at = static_cast<const unsigned char*>(g.a);
            a.end = a.begin + g.rows * a.pitch;
            a.own = q.a0;
            a.own_end = q.a_end;
            b.begin = b.at = static_cast<const unsigned char*>(g.b);
            b.end = b.begin + Kind::kPerResult * b.second;
            b.own = q.b0;
            b.own_end = int(width);
            a.red_end = b.red_end = q.r_end;
            for (int r = 0; r < q.r_end; r += kStep) {
                a.red = b.red = r;
                GatherPackets<1, false> pa;
                GatherPackets<1, false, Kind::kGated, BN> pb;
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
