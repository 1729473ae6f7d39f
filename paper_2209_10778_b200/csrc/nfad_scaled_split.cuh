// nfad_scaled_split.cuh -- the products in 8-bit floating point with block scales when there are few rows or few tiles.
//
// Tiles of 128 rows x 64 columns, at most half as many as SMs: a cluster of two, four or eight CTAs splits each tile's reduction and adds up
// through its shared memory, as nfad_split.cuh does; one CTA to an SM (see scaled_split_ranks).  A step is a block of 128 of the reduction, its
// products in one of four buffers of 64 columns, times its scale into 32 sums a thread.  (Registers for a second CTA that never comes, 80 a
// thread of the 94 wanted: 100 rows 4096 -> 1024 in calls one behind another 11.4 us, now 10.5; 40 rows 8192 -> 2048 15.4, now 14.3.)
//
// For few rows the weights' bytes are what takes the time, and the ring is laid out for them: a stage holds as many rows of x as there are, to
// the next 32, beside the weights' 8 KB, so that up to eight stages (64 KB of weights) are on their way.  (The products read
// 128 rows whatever the stage holds: what lies behind its rows of x are weights or another stage's bytes, in rows of the sums that nobody
// reads.)
#pragma once

#include "nfad_scaled.cuh"
#include "nfad_split.cuh"

namespace nfad {

constexpr int kThinStages = 8;
constexpr int kThinRing = kSplitStages * kSplitStage;
constexpr int kThinBuffers = 4;

struct ThinShared {
    uint64_t full[kThinStages], done[kThinStages], taken[kThinBuffers], drained;
    uint32_t tmem, gave_up;
};
constexpr int kThinSmem = 1024 + kThinRing + int(sizeof(ThinShared));

template <int OP, class S>
__global__ void __launch_bounds__(kSplitThreads, 1)
scaled_split_kernel(const __grid_constant__ ProdArgs g, const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, uint32_t ranks)
{
    using Kind = ProdKind<OP>;
    constexpr uint32_t kResults = kSplitColumns / Kind::kPerResult;          // a tile's
    extern __shared__ unsigned char raw[];
    unsigned char* ring = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
    ThinShared& s = *reinterpret_cast<ThinShared*>(ring + kThinRing);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = tc::rank_in_pair(), tile = blockIdx.x / ranks;
    const uint32_t ring_at = tc::shared_address(ring);
    auto full = [&](int i) { return tc::shared_address(&s.full[i]); };
    auto done = [&](int i) { return tc::shared_address(&s.done[i]); };       // as in scaled_kernel: a stage is free, a buffer full
    auto taken = [&](int i) { return tc::shared_address(&s.taken[i]); };
    volatile uint32_t* gave_up = &s.gave_up;
    const uint32_t width = g.outs, rows = uint32_t(g.rows), blocks = (g.in + kScaleBlock - 1) / kScaleBlock, b_tiles = (width + kResults - 1) / kResults;
    const uint32_t a0 = tile / b_tiles * kTileRows, b0 = tile % b_tiles * kResults;
    const uint32_t boxes = (min(uint32_t(kTileRows), rows - a0) + 31) / 32, stage_a = boxes * 32 * kStepBytes, stage_bytes = stage_a + kSplitColumns * kStepBytes;
    // 128 rows from any stage's beginning on are inside the ring
    const int stages = int(min(uint32_t(kThinStages), min((uint32_t(kThinRing) - kTileRows * kStepBytes) / stage_bytes + 1, uint32_t(kThinRing) / stage_bytes)));
    // this CTA's run of the reduction
    const uint32_t per = (blocks + ranks - 1) / ranks, first_block = min(blocks, rank * per), end_block = min(blocks, first_block + per);
    if (threadIdx.x == 0) {
        s.gave_up = 0;
        for (int i = 0; i < kThinStages; ++i) {
            tc::barrier_init(full(i), 2);
            tc::barrier_init(done(i), 1);
        }
        for (int i = 0; i < kThinBuffers; ++i) tc::barrier_init(taken(i), 8);
        tc::barrier_init(tc::shared_address(&s.drained), 1);
        tc::barrier_init_done();
        tc::prefetch_map(&map_a);
        tc::prefetch_map(&map_b);
    }
    if (warp == 2) tc::tmem_alloc<false>(tc::shared_address(&s.tmem), kThinBuffers * kSplitColumns);
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    // the weights may be read before the kernel in front has ended, where that is the quantiser of the same call
    if (!(g.b_ready && warp == 3)) asm volatile("griddepcontrol.wait;" ::: "memory");
    const uint32_t tmem = s.tmem;
    float2 acc[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] = make_float2(0.0f, 0.0f);
    bool ok = true;
    if (warp == 0 || warp == 3) {
        if (lane == 0) {
            int stage = 0;
            uint32_t phase = 0;
            for (uint32_t b = first_block; b < end_block; ++b) {
                if (!(ok = tc::barrier_wait(done(stage), phase ^ 1, gave_up))) break;
                const uint32_t at_a = ring_at + stage * stage_bytes, at_b = at_a + stage_a;
                tc::barrier_expect(full(stage), warp == 0 ? stage_a : kSplitColumns * kStepBytes);
                if (warp == 0) {
                    for (uint32_t j = 0; j < boxes; ++j) tc::load_box<false>(at_a + j * 32 * 128, &map_a, full(stage), int(b * kScaleBlock), int(a0 + j * 32));
                } else if (Kind::kGated) {
                    tc::load_box<false>(at_b, &map_b, full(stage), int(b * kScaleBlock), int(b0), 0);
                    tc::load_box<false>(at_b + kSplitColumns / 2 * kStepBytes, &map_b, full(stage), int(b * kScaleBlock), int(b0), 1);
                } else {
                    tc::load_box<false>(at_b, &map_b, full(stage), int(b * kScaleBlock), int(b0), 0);
                }
                if (++stage == stages) { stage = 0; phase ^= 1; }
            }
            if (!ok) {
                const long long t0 = clock64();
                while (clock64() - t0 < tc::kWaitDrain) {}
            }
        }
        __syncwarp();
        // the tail of the launch order: whatever read ahead waits here
        if (g.b_ready && warp == 3) asm volatile("griddepcontrol.wait;" ::: "memory");
    } else if (warp == 1) {
        const uint32_t what = tc::instruction(tc::kNumberE4M3, false, false, kTileRows, kSplitColumns);
        const bool leader = tc::elected();
        int stage = 0, turn = 0;
        uint32_t phase = 0, turn_phase = 0;
        bool ready = false;
        for (uint32_t b = first_block; b < end_block; ++b) {
            if (!ready) {
                if (!(ok = tc::barrier_poll(full(stage), phase, gave_up))) break;
                if (!(ok = tc::barrier_poll(taken(turn), turn_phase ^ 1, gave_up))) break;
            }
            tc::fence_after_sync();
            const uint64_t at_a = tc::operand(ring_at + stage * stage_bytes, 16, 1024), at_b = tc::operand(ring_at + stage * stage_bytes + stage_a, 16, 1024);
            const uint32_t to = tmem + turn * kSplitColumns, bar = done(stage);
            if (++stage == stages) { stage = 0; phase ^= 1; }
            if (++turn == kThinBuffers) { turn = 0; turn_phase ^= 1; }
            ready = tc::barrier_test(full(stage), phase) & tc::barrier_test(taken(turn), turn_phase ^ 1);        // ahead, as in scaled_kernel
            if (leader) {
#pragma unroll
                for (int k = 0; k < kStepBytes / 32; ++k) tc::product_e4m3<false>(to, at_a + k * 2, at_b + k * 2, what, k > 0);
                tc::products_to<false>(bar);
            }
            __syncwarp();
        }
        if (!ok && leader) {
            tc::products_to<false>(tc::shared_address(&s.drained));
            const long long t0 = clock64();
            while (!tc::barrier_try(tc::shared_address(&s.drained), 0) && clock64() - t0 < tc::kWaitDrain) {}
        }
        __syncwarp();
    } else if (warp >= kFirstResultWarp) {
        // 32 rows and 32 columns to a warp (gated: those of a, or of u)
        const uint32_t lanes = (warp & 3) * 32, c = (warp - kFirstResultWarp) >> 2;
        const bool live = a0 + lanes < rows;
        const uint32_t sx = min(a0 + lanes + lane, rows - 1), out_blocks = (width + kScaleBlock - 1) / kScaleBlock;
        const uint32_t sw = Kind::kGated ? c * out_blocks + b0 / kScaleBlock : min(b0 + c * 32, width - 1) / kScaleBlock;
        float next_x = 0.0f, next_w = 0.0f;
        auto request = [&](uint32_t b) {
            if (b >= end_block || !live) return;
            next_x = load_now(g.a_scale + (size_t(b) * rows + sx));
            next_w = load_now(g.b_scale + (size_t(sw) * blocks + b));
        };
        request(first_block);
        int stage = 0, turn = 0;
        uint32_t phase = 0;
        for (uint32_t b = first_block; b < end_block; ++b) {
            if (!(ok = tc::barrier_poll(done(stage), phase, gave_up))) break;
            tc::fence_after_sync();
            if (live) {
                uint32_t v[32];
                tc::tmem_load32(tmem + (lanes << 16) + turn * kSplitColumns + c * 32, v);
                const float scale = next_x * next_w;
                request(b + 1);
                tc::tmem_load_wait(v);
                tc::fence_before_sync();
                __syncwarp();
                if (lane == 0) tc::barrier_arrive(taken(turn));
                const float2 s2 = make_float2(scale, scale);
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[i] = hw::fma2(make_float2(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1])), s2, acc[i]);
            } else {
                if (lane == 0) tc::barrier_arrive(taken(turn));
            }
            if (++stage == stages) { stage = 0; phase ^= 1; }
            if (++turn == kThinBuffers) turn = 0;
        }
    }
    // every step's products are done once all roles are here (or one gave up): the ring takes the sums
    __syncwarp();
    __syncthreads();
    constexpr int kPackets = kSplitColumns / 4;      // of a row: four sums each, their places rotated against bank conflicts
    auto place = [](int row, int p) { return (row * kPackets + (p ^ (row & (kPackets - 1)))) * 16; };
    if (warp >= kFirstResultWarp && a0 + (warp & 3) * 32 < rows) {
        const int row = (warp & 3) * 32 + lane, c = (warp - kFirstResultWarp) >> 2;
#pragma unroll
        for (int p = 0; p < 8; ++p)
            *reinterpret_cast<float4*>(ring + place(row, c * 8 + p)) = make_float4(acc[2 * p].x, acc[2 * p].y, acc[2 * p + 1].x, acc[2 * p + 1].y);
    }
    __syncthreads();
    tc::pair_sync();                                 // of the whole cluster
    {
        // packets of eight results, shared out over the cluster
        const int live_rows = int(min(uint32_t(kTileRows), rows - a0));
        constexpr int kOut = kResults / 8;
        for (int i = rank * kSplitThreads + threadIdx.x; i < live_rows * kOut; i += ranks * kSplitThreads) {
            const int row = i / kOut, p = i % kOut;
            const uint32_t col = b0 + p * 8;
            if (col >= width) continue;
            float z[8], f[8];
            auto sums = [&](int p, float (&z)[8]) {
#pragma unroll
                for (int e = 0; e < 8; ++e) z[e] = 0.0f;
                for (uint32_t k = 0; k < ranks; ++k)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint4 w = peer_packet(ring_at + place(row, p * 2 + h), k);
                        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                        for (int e = 0; e < 4; ++e) z[h * 4 + e] += __uint_as_float(u[e]);
                    }
            };
            auto add_bias = [&](int matrix, float (&z)[8]) {
                if (!g.bias) return;
                load8<S>(g.bias, matrix, width, col, f);
#pragma unroll
                for (int e = 0; e < 8; ++e) z[e] += f[e];
            };
            sums(p, z);
            add_bias(0, z);
            act8<false>(g.act, z, f);
            if constexpr (Kind::kGated) {
                float u[8];
                sums(p + kOut, u);
                add_bias(1, u);
#pragma unroll
                for (int e = 0; e < 8; ++e) z[e] *= u[e];
            }
            *reinterpret_cast<uint4*>(static_cast<typename S::elem*>(g.out) + (size_t(a0) + row) * width + col) = S::pack(z);
        }
    }
    __syncthreads();
    tc::pair_sync();                                 // no CTA reads this one's sums any more
    tc::fence_after_sync();
    if (warp == 2) tc::tmem_free<false>(tmem, kThinBuffers * kSplitColumns);
    if (threadIdx.x == 0 && s.gave_up) atomicAdd(&g_product_faults, 1u);
}

}  // namespace nfad
