// nfad_split.cuh -- the products when there are fewer tiles than SMs: the reduction is split over a cluster of CTAs.
//
// Every CTA of a cluster takes the same 128 x 64 tile and its own run of the reduction (tcgen05, as nfad_product.cuh, but one
// tile and one accumulator); then each leaves its sums in its shared memory, and the cluster's CTAs add them up, each for its
// share of the packets, in rank order (the same bits every time) and finish them.  Two CTAs fit an SM, so that up to two
// clusters' worth of loads are in flight on each.  Bound by latency: fill, a few steps, one exchange.
// 77 rows 5120 -> 2048 in 8 bits: 10.9 us by four CTAs a tile, 16.2 by one (the launch's rule has more).
#pragma once

#include "nfad_product.cuh"

namespace nfad {

constexpr int kSplitColumns = 64;
constexpr int kSplitStage = (kTileRows + kSplitColumns) * kStepBytes;
constexpr int kSplitStages = 4;
constexpr int kSplitThreads = (kFirstResultWarp + 8) * 32;

struct SplitShared {
    uint64_t full[kSplitStages], empty[kSplitStages], landed[kSplitStages], done;
    uint32_t tmem, gave_up;
    int start[kMaxExperts + 1], tiles[kMaxExperts + 1];
};
constexpr int kSplitSmem = 1024 + kSplitStages * kSplitStage + int(sizeof(SplitShared));

// 16 bytes of another CTA's shared memory (`address` as this CTA has it)
__device__ __forceinline__ uint4 peer_packet(uint32_t address, uint32_t rank)
{
    uint32_t at;
    uint4 v;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(address), "r"(rank));
    asm volatile("ld.shared::cluster.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}

template <int OP, class S>
__global__ void __launch_bounds__(kSplitThreads, 2)
split_kernel(const __grid_constant__ ProdArgs g, const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, uint32_t ranks)
{
    using Kind = ProdKind<OP>;
    constexpr int kStep = Kind::kStep;
    extern __shared__ unsigned char raw[];
    unsigned char* ring = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
    SplitShared& s = *reinterpret_cast<SplitShared*>(ring + kSplitStages * kSplitStage);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = tc::rank_in_pair(), tile = blockIdx.x / ranks;
    const uint32_t ring_at = tc::shared_address(ring), done = tc::shared_address(&s.done);
    auto full = [&](int i) { return tc::shared_address(&s.full[i]); };
    auto empty = [&](int i) { return tc::shared_address(&s.empty[i]); };
    auto landed = [&](int i) { return tc::shared_address(&s.landed[i]); };
    volatile uint32_t* gave_up = &s.gave_up;
    if (threadIdx.x == 0) {
        s.gave_up = 0;
        for (int i = 0; i < kSplitStages; ++i) {
            tc::barrier_init(full(i), 2);
            tc::barrier_init(empty(i), 1);
            tc::barrier_init(landed(i), 2);
        }
        tc::barrier_init(done, 1);
        tc::barrier_init_done();
        tc::prefetch_map(&map_a);
        tc::prefetch_map(&map_b);
    }
    if (warp == 2) tc::tmem_alloc<false>(tc::shared_address(&s.tmem), kSplitColumns);
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (warp == 3) row_table<kTileRows>(g, s.start, s.tiles, lane);
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    const uint32_t tmem = s.tmem;
    const uint32_t width = Kind::kInput || OP == kProdWeight ? g.in : g.outs;
    constexpr uint32_t kResults = kSplitColumns / Kind::kPerResult;          // a tile's
    TileWalk<OP, kSplitColumns, false> walk;
    walk.b_tiles = (width + kResults - 1) / kResults;
    const uint32_t total = (OP == kProdWeight ? g.experts * ((g.outs + kTileRows - 1) / kTileRows) : uint32_t(s.tiles[g.experts])) * walk.b_tiles;
    const bool mine = tile < total;                  // the same for every CTA of the cluster
    ProdTileAt q = {};
    int r0 = 0, r1 = 0;                              // this CTA's run of the reduction
    if (mine) {
        q = walk.at(g, s.start, s.tiles, tile);
        const int steps = (q.r_end - q.r0 + kStep - 1) / kStep, per = (steps + int(ranks) - 1) / int(ranks);
        r0 = min(q.r_end, q.r0 + int(rank) * per * kStep);
        r1 = min(q.r_end, r0 + per * kStep);
    }
    const uint32_t n = Kind::kGated ? kSplitColumns : min(uint32_t(kSplitColumns), (width - q.b0 + 15) / 16 * 16);
    auto ragged = [&](int r) { return OP == kProdWeight && r + kStep > q.r_end && (q.r_end - r) % kProductRows; };
    bool ok = true;
    if (warp == 0 || warp == 3) {
        const bool for_a = warp == 0;
        if (lane == 0) {
            const int boxes = (min(kTileRows, q.a_end - q.a0) + 31) / 32;
            const uint32_t bytes = !for_a ? kSplitColumns * kStepBytes : Kind::kTurnA ? kTileRows * kStepBytes : uint32_t(boxes) * 32 * kStepBytes;
            int stage = 0;
            uint32_t phase = 0;
            for (int r = r0; r < r1; r += kStep) {
                if (!(ok = tc::barrier_wait(empty(stage), phase ^ 1, gave_up))) break;
                const uint32_t at_a = ring_at + stage * kSplitStage, at_b = at_a + kTileRows * kStepBytes;
                const uint32_t bar = ragged(r) ? landed(stage) : full(stage);
                tc::barrier_expect(bar, bytes);
                if (for_a) {
                    if (Kind::kTurnA) {
#pragma unroll
                        for (int j = 0; j < 2; ++j) tc::load_box<false>(at_a + j * 64 * 128, &map_a, bar, q.a0 + j * 64, r);
                    } else {
                        for (int j = 0; j < boxes; ++j) tc::load_box<false>(at_a + j * 32 * 128, &map_a, bar, r, q.a0 + j * 32);
                    }
                } else if (OP == kProdWeight) {
                    tc::load_box<false>(at_b, &map_b, bar, q.b0, r);
                } else if (Kind::kTurnB) {
                    tc::load_box<false>(at_b, &map_b, bar, q.b0, r, int(q.expert));
                } else if (Kind::kGated) {
                    tc::load_box<false>(at_b, &map_b, bar, r, q.b0, int(q.expert * 2));
                    tc::load_box<false>(at_b + kSplitColumns / 2 * kStepBytes, &map_b, bar, r, q.b0, int(q.expert * 2 + 1));
                } else {
                    tc::load_box<false>(at_b, &map_b, bar, r, q.b0, int(q.expert));
                }
                if (++stage == kSplitStages) { stage = 0; phase ^= 1; }
            }
            if (!ok) {
                const long long t0 = clock64();
                while (clock64() - t0 < tc::kWaitDrain) {}
            }
        }
    } else if (warp == 1) {
        const uint32_t what = tc::instruction(Kind::kBytes ? tc::kNumberS8 : IsBF16<S>::value ? tc::kNumberBF16 : tc::kNumberF16, Kind::kTurnA, Kind::kTurnB, kTileRows, n);
        const bool leader = tc::elected();
        int stage = 0;
        uint32_t phase = 0, landed_phases = 0;
        for (int r = r0; r < r1; r += kStep) {
            if (ragged(r)) {
                if (!(ok = tc::barrier_wait(landed(stage), landed_phases >> stage & 1, gave_up))) break;
                landed_phases ^= 1u << stage;
                clear_runs(ring + stage * kSplitStage, 2 + kSplitColumns / 64, q.r_end - r, lane);
                tc::writes_to_async();
                __syncwarp();
                if (lane < 2) tc::barrier_arrive(full(stage));
            }
            if (!(ok = tc::barrier_poll(full(stage), phase, gave_up))) break;
            tc::fence_after_sync();
            const uint32_t at_a = ring_at + stage * kSplitStage, at_b = at_a + kTileRows * kStepBytes;
            if (leader) {
#pragma unroll
                for (int k = 0; k < kStepBytes / 32; ++k) {
                    if (OP == kProdWeight && k * kProductRows >= q.r_end - r) break;
                    const uint64_t da = Kind::kTurnA ? tc::operand(at_a + k * 2048, 64 * 128, 1024) : tc::operand(at_a + k * 32, 16, 1024);
                    const uint64_t db = Kind::kTurnB ? tc::operand(at_b + k * 2048, 64 * 128, 1024) : tc::operand(at_b + k * 32, 16, 1024);
                    tc::product<Kind::kBytes, false>(tmem, da, db, what, r > r0 || k > 0);
                }
                tc::products_to<false>(empty(stage));
            }
            __syncwarp();
            if (++stage == kSplitStages) { stage = 0; phase ^= 1; }
        }
        // every product issued is done when this arrives, after a wait that ran out too
        if (leader) tc::products_to<false>(done);
        __syncwarp();
    }
    // every CTA's sums into its own shared memory: the ring is free once its products are done
    if (!tc::barrier_wait(done, 0, gave_up)) ok = false;
    tc::fence_after_sync();
    __syncwarp();
    constexpr int kPackets = kSplitColumns / 4;      // of a row: four 32-bit sums each, their places rotated against bank conflicts
    auto place = [](int row, int p) { return (row * kPackets + (p ^ (row & (kPackets - 1)))) * 16; };
    if (warp >= kFirstResultWarp && mine) {
        const int row = (warp & 3) * 32 + lane, c = (warp - kFirstResultWarp) >> 2;
        if (q.a0 + (warp & 3) * 32 < q.a_end) {
            uint32_t v[32];
            tc::tmem_load32(tmem + (uint32_t((warp & 3) * 32) << 16) + c * 32, v);
            tc::tmem_load_wait();
#pragma unroll
            for (int p = 0; p < 8; ++p) {
                uint4 t = make_uint4(v[4 * p], v[4 * p + 1], v[4 * p + 2], v[4 * p + 3]);
                if (r0 >= r1) t = make_uint4(0, 0, 0, 0);            // nothing was summed here
                *reinterpret_cast<uint4*>(ring + place(row, c * 8 + p)) = t;
            }
        }
    }
    tc::fence_before_sync();
    __syncthreads();
    tc::pair_sync();                                 // of the whole cluster
    if (mine) {
        // packets of eight results, shared out over the cluster
        const int rows = min(kTileRows, q.a_end - q.a0);
        constexpr int kOut = kResults / 8;                            // packets of a row
        for (int i = rank * kSplitThreads + threadIdx.x; i < rows * kOut; i += ranks * kSplitThreads) {
            const int row = i / kOut, p = i % kOut;
            const uint32_t col = q.b0 + p * 8;
            if (col >= width) continue;
            float z[8];
            int t[8];
            auto sums = [&](int p) {
#pragma unroll
                for (int e = 0; e < 8; ++e) { z[e] = 0.0f; t[e] = 0; }
                for (uint32_t k = 0; k < ranks; ++k)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint4 w = peer_packet(ring_at + place(row, p * 2 + h), k);
                        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            if (Kind::kBytes) t[h * 4 + e] += int(u[e]);
                            else z[h * 4 + e] += __uint_as_float(u[e]);
                        }
                    }
            };
            if constexpr (Kind::kGated) {
                float u[8], f[8], d[8];
                sums(p + kOut);
#pragma unroll
                for (int e = 0; e < 8; ++e) { u[e] = z[e]; d[e] = 1.0f; }
                sums(p);
                if (g.bias) {
                    load8<S>(g.bias, q.expert * 2, width, col, f);
#pragma unroll
                    for (int e = 0; e < 8; ++e) z[e] += f[e];
                    load8<S>(g.bias, q.expert * 2 + 1, width, col, f);
#pragma unroll
                    for (int e = 0; e < 8; ++e) u[e] += f[e];
                }
                const size_t r = size_t(q.a0) + row;
                if (g.slope) {
                    act8<true>(g.act, z, d);
#pragma unroll
                    for (int e = 0; e < 8; ++e) d[e] *= u[e];
                    typename S::elem* both = static_cast<typename S::elem*>(g.slope) + r * 2 * width + col;
                    *reinterpret_cast<uint4*>(both) = S::pack(d);
                    *reinterpret_cast<uint4*>(both + width) = S::pack(z);
                } else {
                    act8<false>(g.act, z, d);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) z[e] *= u[e];
                *reinterpret_cast<uint4*>(static_cast<typename S::elem*>(g.out) + r * width + col) = S::pack(z);
                continue;
            }
            sums(p);
            const size_t out_row = OP == kProdWeight ? size_t(q.expert) * g.outs + q.a0 + row : size_t(q.a0) + row, at = out_row * width + col;
            if (Kind::kBytes) {
                const float scale = g.a_scale[q.a0 + row];
#pragma unroll
                for (int e = 0; e < 8; ++e) z[e] = float(t[e]) * (scale * g.b_scale[col + e]);
            }
            float f[8];
            if (Kind::kForward && g.bias) {
                load8<S>(g.bias, q.expert, width, col, f);
#pragma unroll
                for (int e = 0; e < 8; ++e) z[e] += f[e];
            }
            if constexpr (OP == kProdInputGated) {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    load8<S>(g.prev, out_row * 2 + j, width, col, f);
#pragma unroll
                    for (int e = 0; e < 8; ++e) f[e] *= z[e];
                    *reinterpret_cast<uint4*>(static_cast<typename S::elem*>(g.out) + (out_row * 2 + j) * width + col) = S::pack(f);
                }
                continue;
            }
            if (OP == kProdInput && g.prev) {
                load8<S>(g.prev, out_row, width, col, f);
#pragma unroll
                for (int e = 0; e < 8; ++e) z[e] *= f[e];
            }
            if constexpr (OP == kProdForward || OP == kProdBytes) {
                if (OP == kProdForward && g.slope) {
                    act8<true>(g.act, z, f);
                    *reinterpret_cast<uint4*>(static_cast<typename S::elem*>(g.slope) + at) = S::pack(f);
                } else {
                    act8<false>(g.act, z, f);
                }
            }
            *reinterpret_cast<uint4*>(static_cast<typename S::elem*>(g.out) + at) = S::pack(z);
        }
    }
    if (OP != kProdWeight && g.offsets) {
        clear_rows<S, kSplitThreads, OP>(g, 0, s.start[0], width, threadIdx.x);
        clear_rows<S, kSplitThreads, OP>(g, s.start[g.experts], int(g.rows), width, threadIdx.x);
    }
    __syncthreads();
    tc::pair_sync();                                 // no CTA reads this one's sums any more
    tc::fence_after_sync();
    if (warp == 2) tc::tmem_free<false>(tmem, kSplitColumns);
    if (threadIdx.x == 0 && s.gave_up) atomicAdd(&g_product_faults, 1u);
}

}  // namespace nfad
