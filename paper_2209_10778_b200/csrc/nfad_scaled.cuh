// nfad_scaled.cuh -- matrix products in 8-bit floating point (four exponent bits, three of the significand) whose operands carry a scale for
// each block of 128 along the reduction: z[m, o] = sum_b sx[b, m] sw[o / 128, b] sum_{k in block b} xq[m, k] wq[o, k], then the epilogues of
// the other products, plain or gated.
//
// A stage of the ring holds 128 bytes of the reduction: one block.  So a step's products (four of 32) start from zero in a buffer of
// tensor memory of their own, and the result warps take every step's buffer, times its scale, into sums that stay in their registers:
// 128 columns of a row to a thread, as 64 pairs of packed multiply-adds.  Two buffers of 256 columns (four of 128) let the products
// run ahead.  The copying and issuing warps give registers to the result warps (setmaxnreg).
//
// Roles, tiles, pairs of CTAs and the gather for rows off the 16-byte boundaries are those of nfad_product.cuh; results leave by tensor
// copies, while the next tile's steps run.
//
// What bounds it: a step takes 440 ns where its products take 277 (the result warps' reads of tensor memory, 55 cycles for 16 columns, eight
// in turn, and the way there and back), and the epilogue, whose sums are the next tile's registers, follows the steps: 1.9 us for a tile
// without an activation, 3.9 with Swish (two special-function results an element).  8000 rows 4096 -> 16384 bf16, the product alone, twenty
// captured calls in turn: 483 to 533 us by the device's clock, with Swish 569 to 584, with GELU-tanh and bias 535 to 581; the quantiser takes 18
// to 22 more, and calls one behind another until the power limit sets the clock 640 in all (GELU-tanh and bias).
#pragma once

#include <stddef.h>

#include "nfad_dropout_args.h"
#include "nfad_product.cuh"

namespace nfad {

constexpr int kScaleBlock = 128;
template <class T> struct TypeTag { using type = T; };

template <bool kGather> struct ScaledWarps {
    static constexpr int kResult = kGather ? 4 : 8;
    static constexpr int kThreads = (kFirstResultWarp + kResult + (kGather ? kGatherWarps : 0)) * 32;
};

struct ScaledShared {
    uint64_t full[kMaxStages], done[kMaxStages], taken[4], drained;
    uint32_t tmem, gave_up;
};

// Tile t's first row and first result, in the bands of TileWalk
struct ScaledAt { uint32_t a0, b0; };
__device__ __forceinline__ ScaledAt scaled_at(uint32_t t, uint32_t a_tiles, uint32_t b_tiles, uint32_t tile_rows, uint32_t results)
{
    const uint32_t band = t / (kBand * b_tiles), in_band = t - band * kBand * b_tiles, height = min(kBand, a_tiles - band * kBand);
    const uint32_t bt = in_band / height;
    return {(band * kBand + in_band - bt * height) * tile_rows, bt * results};
}
// a result warp's 32 rows of up to 128 results, as two boxes of 64 (128 bytes) that tensor copies store
constexpr int kOutBytes = 2 * kStageBytes;
constexpr int kScaledSmem = 1024 + kRingBytes + kMostResultWarps * kOutBytes + int(sizeof(ScaledShared));

// 16 columns of a buffer, times their scale, into the sums.  (Chunks of 32 leave a warp fewer, longer waits, but the 32 registers more spill
// within the steps: 515 ns a step against 485.)
constexpr int kChunk = 16;
template <int kColumns> __device__ __forceinline__ void add_chunk(float2 (&acc)[kColumns / 2], int chunk, const uint32_t (&v)[kChunk], float scale)
{
    const float2 s = make_float2(scale, scale);
#pragma unroll
    for (int i = 0; i < kChunk / 2; ++i)
        acc[chunk * (kChunk / 2) + i] = hw::fma2(make_float2(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1])), s, acc[chunk * (kChunk / 2) + i]);
}

// Eight results from sums: bias, activation (K void: none), the other factor of a gated layer, one rounding.
template <class K, class S, bool kGated> __device__ __forceinline__ uint4 finish8(const float2* a, const float2* u, const float (&bias)[8], const float (&bias_u)[8])
{
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
        float2 z = make_float2(a[e / 2].x + bias[e], a[e / 2].y + bias[e + 1]);
        if constexpr (!IsVoid<K>::value) z = evaluate_value(K{}, Fast2{}, z);
        if (kGated) z = make_float2(z.x * (u[e / 2].x + bias_u[e]), z.y * (u[e / 2].y + bias_u[e + 1]));
        y[e] = z.x;
        y[e + 1] = z.y;
    }
    return S::pack(y);
}

// a value whose origin the compiler does not see: it is formed where this stands, and what is formed of it further down
__device__ __forceinline__ uint32_t fresh(uint32_t v)
{
    asm volatile("" : "+r"(v));
    return v;
}

// A load that stays where it stands: left to itself it sinks to its use, a step later, and every step waits for it (500 of 1000 cycles).
// (An ordinary one, like all loads of what a kernel in front may write: these kernels begin before that one has ended, and the read-only
// path asks for data that nothing writes while the kernel lives.)
__device__ __forceinline__ float load_now(const float* p)
{
    float v;
    asm volatile("ld.global.f32 %0, [%1];" : "=f"(v) : "l"(p));
    return v;
}

template <int OP, int BN, class S, bool kGather, bool kPair>
__global__ void __launch_bounds__(ScaledWarps<kGather>::kThreads, 1)
scaled_kernel(const __grid_constant__ ProdArgs g, const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
              const __grid_constant__ CUtensorMap map_out, int out_copies)
{
    using Kind = ProdKind<OP>;
    using Tile = ProdTile<BN, kPair>;
    static_assert(Kind::kScaled && Kind::kStep == kScaleBlock, "a stage is a block");
    constexpr int kStages = Tile::kStages, kStep = Kind::kStep, kOwn = Tile::kOwnColumns;
    constexpr int kBuffers = BN > 128 ? 2 : 4;
    constexpr uint32_t kTmem = kBuffers * BN, kResults = BN / Kind::kPerResult;
    constexpr int kBoxRows = Tile::kBoxRows, kResultWarps = ScaledWarps<kGather>::kResult;
    constexpr int kColumns = BN / (kResultWarps / 4), kChunks = kColumns / kChunk;        // a result warp's
    constexpr bool kMoveRegisters = BN > 128;        // 168 a thread at launch: 40 for four warps leave 232 for the other eight
    extern __shared__ unsigned char raw[];
    unsigned char* ring = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
    ScaledShared& s = *reinterpret_cast<ScaledShared*>(ring + kRingBytes + kMostResultWarps * kOutBytes);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = kPair ? tc::rank_in_pair() : 0;
    const uint32_t unit = kPair ? blockIdx.x >> 1 : blockIdx.x, units = kPair ? gridDim.x >> 1 : gridDim.x;
    const uint32_t ring_at = tc::shared_address(ring);
    auto full = [&](int i) { return tc::shared_address(&s.full[i]); };
    // a step's products are done: its stage is free and its buffer full.  One barrier says both, as a commit takes a place in the tensor
    // cores' queue.  Copies and results each see every phase: the next one needs the stage copied to and the buffer taken.
    auto done = [&](int i) { return tc::shared_address(&s.done[i]); };
    auto taken = [&](int i) { return tc::shared_address(&s.taken[i]); };          // a buffer's sums are in registers
    volatile uint32_t* gave_up = &s.gave_up;

    if (threadIdx.x == 0) {
        s.gave_up = 0;
        for (int i = 0; i < kStages; ++i) {
            // per stage: both copying threads of each CTA (or every gathering thread); the products' one commit
            tc::barrier_init(full(i), kGather ? kGatherWarps * 32 : kPair ? 4 : 2);
            tc::barrier_init(done(i), 1);
        }
        for (int i = 0; i < kBuffers; ++i) tc::barrier_init(taken(i), kResultWarps * (kPair ? 2 : 1));
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
    tc::fence_before_sync();
    __syncthreads();
    if (kPair) tc::pair_sync();                      // the other CTA's barriers exist
    tc::fence_after_sync();
    const uint32_t tmem = s.tmem, width = g.outs, blocks = (g.in + kScaleBlock - 1) / kScaleBlock;
    const uint32_t rows = uint32_t(g.rows), a_tiles = (rows + Tile::kRows - 1) / Tile::kRows, b_tiles = (width + kResults - 1) / kResults;
    const uint32_t total = a_tiles * b_tiles;
    auto tile_at = [&](uint32_t t) { return scaled_at(t, a_tiles, b_tiles, Tile::kRows, kResults); };
    // the last tile along a result's row is a narrower product (a multiple of 16 columns, of 32 for a pair, which halves it)
    auto columns = [&](const ScaledAt& q) {
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
                    const ScaledAt q = tile_at(t);
                    const int a0 = int(q.a0 + rank * kTileRows), b0 = int(q.b0 + (rank && !Kind::kGated ? columns(q) / 2 : 0));
                    const int a_rows = max(0, min(kTileRows, int(rows) - a0)), boxes = (a_rows + kBoxRows - 1) / kBoxRows;
                    const uint32_t bytes = for_a ? uint32_t(boxes) * kBoxRows * kStepBytes : kOwn * kStepBytes;
                    bool ok = true;
                    for (uint32_t b = 0; b < blocks; ++b) {
                        if (!(ok = tc::barrier_wait(done(stage), phase ^ 1, gave_up))) break;
                        const uint32_t at_a = ring_at + stage * Tile::kStage, at_b = at_a + kTileRows * kStepBytes;
                        uint32_t bar = full(stage);
                        if (kPair) {
                            bar = tc::first_of_pair(bar);
                            tc::barrier_expect_first(bar, bytes);
                        } else {
                            tc::barrier_expect(bar, bytes);
                        }
                        if (for_a) {
                            for (int j = 0; j < boxes; ++j) tc::load_box<kPair>(at_a + j * kBoxRows * 128, &map_a, bar, int(b * kStep), a0 + j * kBoxRows);
                        } else if (Kind::kGated) {
                            // a pair's first CTA holds a's columns, the second u's
                            tc::load_box<kPair>(at_b, &map_b, bar, int(b * kStep), b0, int(rank));
                            if (!kPair) tc::load_box<kPair>(at_b + kOwn / 2 * kStepBytes, &map_b, bar, int(b * kStep), b0, 1);
                        } else {
                            tc::load_box<kPair>(at_b, &map_b, bar, int(b * kStep), b0, 0);
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
            // ------------------------------------------------ products: a buffer for each step.  The next step's barriers are looked at before
            // this step's products are issued, which hides the looks: by one lane alone, step after step, 780 cycles (350 of them looks).
            const bool leader = tc::elected();
            uint32_t stage = 0, phase = 0, turn = 0, turn_phase = 0;
            bool ok = true, ready = false;
            for (uint32_t t = unit; t < total && ok; t += units) {
                const uint32_t what = tc::instruction(tc::kNumberE4M3, false, false, Tile::kRows, columns(tile_at(t)));
                for (uint32_t b = 0; b < blocks; ++b) {
                    if (!ready) {
                        if (!(ok = tc::barrier_poll(full(stage), phase, gave_up))) break;
                        if (!(ok = tc::barrier_poll(taken(turn), turn_phase ^ 1, gave_up))) break;
                    }
                    tc::fence_after_sync();
                    const uint64_t at_a = tc::operand(ring_at + stage * Tile::kStage, 16, 1024), at_b = tc::operand(ring_at + stage * Tile::kStage + kTileRows * kStepBytes, 16, 1024);
                    const uint32_t to = tmem + turn * BN, bar = done(stage);
                    if (++stage == kStages) { stage = 0; phase ^= 1; }
                    if (++turn == kBuffers) { turn = 0; turn_phase ^= 1; }
                    ready = tc::barrier_test(full(stage), phase) & tc::barrier_test(taken(turn), turn_phase ^ 1);
                    if (leader) {
#pragma unroll
                        for (int k = 0; k < kStepBytes / 32; ++k) tc::product_e4m3<kPair>(to, at_a + k * 2, at_b + k * 2, what, k > 0);
                        tc::products_to<kPair>(bar);
                    }
                    __syncwarp();
                }
            }
            if (!ok && leader) {
                tc::products_to<kPair>(tc::shared_address(&s.drained));
                const long long t0 = clock64();
                while (!tc::barrier_try(tc::shared_address(&s.drained), 0) && clock64() - t0 < tc::kWaitDrain) {}
            }
        }
    } else if (warp < kFirstResultWarp + kResultWarps) {
        if (kMoveRegisters) asm volatile("setmaxnreg.inc.sync.aligned.u32 232;");
        // ------------------------------------------------ results.  Little besides the sums may live through the steps.
        // What the roles share is formed anew here, hidden from the compiler: a value that lives across the roles is put into local memory
        // and fetched from there in every step.
        const uint32_t thread = fresh(threadIdx.x), warp = thread >> 5, lane = thread & 31;
        const uint32_t rows = fresh(uint32_t(g.rows)), width = fresh(g.outs), blocks = (fresh(g.in) + kScaleBlock - 1) / kScaleBlock;
        const uint32_t rank = kPair ? fresh(tc::rank_in_pair()) : 0, block = fresh(blockIdx.x), step = fresh(gridDim.x);
        const uint32_t unit = kPair ? block >> 1 : block, units = kPair ? step >> 1 : step;
        const uint32_t a_tiles = (rows + Tile::kRows - 1) / Tile::kRows, b_tiles = (width + kResults - 1) / kResults, total = a_tiles * b_tiles;
        const uint32_t base = fresh(tc::shared_address(raw)), shared_at = ((base + 1023) & ~1023u) + kRingBytes + kMostResultWarps * kOutBytes;
        auto done = [&](int i) { return shared_at + uint32_t(offsetof(ScaledShared, done)) + i * 8; };
        auto taken = [&](int i) { return shared_at + uint32_t(offsetof(ScaledShared, taken)) + i * 8; };
        uint32_t tmem;
        asm volatile("ld.shared.u32 %0, [%1];" : "=r"(tmem) : "r"(shared_at + uint32_t(offsetof(ScaledShared, tmem))));
        const int lanes = (warp & 3) * 32, half = (warp - kFirstResultWarp) >> 2;
        constexpr int kOut = kColumns / Kind::kPerResult;                    // this warp's results of a row, from half kOut on
        // chunk c's first column in a buffer: a gated warp has columns of a first, then those of u
        auto column = [&](int c) { return Kind::kGated && c >= kChunks / 2 ? int(kResults) + half * kOut + (c - kChunks / 2) * kChunk : half * kOut + c * kChunk; };
        uint32_t turn = 0, stage = 0, phase = 0;
        for (uint32_t t = unit; t < total; t += units) {
            const ScaledAt q = scaled_at(t, a_tiles, b_tiles, Tile::kRows, kResults);
            const uint32_t row0 = q.a0 + rank * kTileRows + lanes;            // this warp's first row
            const uint32_t first = q.b0 + half * kOut;                        // and result: all of its results are in one block of outputs
            float2 acc[kColumns / 2];
#pragma unroll
            for (int i = 0; i < kColumns / 2; ++i) acc[i] = make_float2(0.0f, 0.0f);
            // scales, one block ahead; a row or column outside has any valid one's, for sums that nobody uses
            const uint32_t sx = min(row0 + lane, rows - 1), sw = min(first, width - 1) / kScaleBlock;
            float next_x = 0.0f, next_a = 0.0f, next_u = 0.0f;
            auto request = [&](uint32_t b) {
                if (b >= blocks) return;
                next_x = load_now(g.a_scale + (size_t(b) * rows + sx));
                next_a = load_now(g.b_scale + (size_t(sw) * blocks + b));
                if (Kind::kGated) next_u = load_now(g.b_scale + ((size_t((width + kScaleBlock - 1) / kScaleBlock) + sw) * blocks + b));
            };
            request(0);
            if (g.bias && first + lane * (kOut / 32) < width) {
                // needed behind the steps; not held through them
                const typename S::elem* bias = static_cast<const typename S::elem*>(g.bias) + first + lane * (kOut / 32);
                asm volatile("prefetch.global.L1 [%0];" ::"l"(bias));
                if (Kind::kGated) asm volatile("prefetch.global.L1 [%0];" ::"l"(bias + width));
            }
            bool ok = true;
            for (uint32_t b = 0; b < blocks; ++b) {
                if (!(ok = tc::barrier_wait(done(stage), phase, gave_up))) break;
                tc::fence_after_sync();
                const uint32_t at = tmem + (uint32_t(lanes) << 16) + turn * BN;
                uint32_t v[2][kChunk];
                tc::tmem_load16(at + column(0), v[0]);
                // while the first chunk is on its way
                const float scale = next_x * next_a, scale_u = next_x * next_u;
                request(b + 1);
#pragma unroll
                for (int c = 0; c < kChunks; ++c) {
                    tc::tmem_load_wait(v[c & 1]);
                    if (c + 1 < kChunks) tc::tmem_load16(at + column(c + 1), v[(c + 1) & 1]);
                    else {
                        // everything of this buffer is in registers
                        tc::fence_before_sync();
                        __syncwarp();
                        if (lane == 0) {
                            if (kPair) tc::barrier_arrive_first(tc::first_of_pair(taken(turn)));
                            else tc::barrier_arrive(taken(turn));
                        }
                    }
                    add_chunk<kColumns>(acc, c, v[c & 1], Kind::kGated && c >= kChunks / 2 ? scale_u : scale);
                }
                if (++turn == kBuffers) turn = 0;
                if (++stage == kStages) { stage = 0; phase ^= 1; }
            }
            if (!ok) break;
            if (first < width && row0 < rows) {
                // the bias of this warp's results, kMine neighbours to a lane: fetched packet by packet, it cost 3 us a tile
                constexpr int kMine = kOut / 32;
                float bias[kMine], bias_u[kMine];
#pragma unroll
                for (int i = 0; i < kMine; ++i) {
                    const uint32_t c = first + lane * kMine + i;
                    const typename S::elem* p = static_cast<const typename S::elem*>(g.bias) + c;
                    bias[i] = g.bias && c < width ? S::load1(p) : 0.0f;
                    bias_u[i] = Kind::kGated && g.bias && c < width ? S::load1(p + width) : 0.0f;
                }
                // from here on by a copy of the thread's number that is made here, so that no address of this part lives through the steps
                const uint32_t again = fresh(threadIdx.x), place = again & 31;
                unsigned char* boxes = ring + kRingBytes + ((again >> 5) - kFirstResultWarp) * kOutBytes;
                RowPackets packets;
                packets.lane = place;
                packets.rows = min(32, int(rows - row0));
                packets.width = width;
                packets.pitch = width;
                packets.row0 = row0;
                if (out_copies) {
                    // the last tile's boxes have left
                    if (place == 0) tc::stores_read();
                    __syncwarp();
                }
                auto finish = [&](auto kind) {
                    using K = typename decltype(kind)::type;
                    constexpr int kBox = kOut < 64 ? kOut : 64;
#pragma unroll
                    for (int o = 0; o < kOut; o += kBox) {
                        if (first + o >= width) break;
                        packets.stage = reinterpret_cast<uint4*>(boxes + (o ? kStageBytes : 0));
#pragma unroll
                        for (int p = 0; p < kBox / 8; ++p) {
                            float add[8] = {}, add_u[8] = {};
                            if (g.bias)
#pragma unroll
                                for (int e = 0; e < 8; ++e) {
                                    const int c = o + p * 8 + e;
                                    add[e] = __shfl_sync(0xffffffffu, bias[c % kMine], c / kMine);
                                    if (Kind::kGated) add_u[e] = __shfl_sync(0xffffffffu, bias_u[c % kMine], c / kMine);
                                }
                            const uint4 y = finish8<K, S, Kind::kGated>(acc + (o + p * 8) / 2, acc + (Kind::kGated ? kColumns / 4 : 0) + (o + p * 8) / 2, add, add_u);
                            if (out_copies) packets.stage[place * 8 + (p ^ (place & 7))] = y;         // the copies' swizzle
                            else packets.put(p, y);
                        }
                        if (out_copies) {
                            tc::writes_to_async();
                            __syncwarp();
                            if (place == 0) tc::store_box(&map_out, tc::shared_address(packets.stage), int(first + o), int(row0));
                        } else {
                            __syncwarp();
                            if (width % 8 == 0 && (reinterpret_cast<uintptr_t>(g.out) & 15u) == 0) packets.template store<S, kBox / 8>(g.out, first + o, 0);
                            else packets.template store_odd<S, kBox / 8>(g.out, first + o, 0);
                            __syncwarp();
                        }
                    }
                };
                switch (g.act) {
                case kGeluErf:  finish(TypeTag<GeluErf>{}); break;
                case kGeluTanh: finish(TypeTag<GeluTanh>{}); break;
                case kSwish:    finish(TypeTag<Swish>{}); break;
                case kMish:     finish(TypeTag<Mish>{}); break;
                default:        finish(TypeTag<void>{}); break;
                }
            }
        }
        if (out_copies && lane == 0) tc::stores_done();
    } else if (kGather) {
        // ------------------------------------------------ the same by plain loads
        uint32_t stage = 0, phase = 0;
        bool ok = true;
        for (uint32_t t = unit; t < total && ok; t += units) {
            const ScaledAt q = tile_at(t);
            const int thread = threadIdx.x - (kFirstResultWarp + kResultWarps) * 32;
            GatherSource a, b;
            a.pitch = b.pitch = g.in;
            b.second = size_t(g.outs) * g.in;
            a.begin = a.at = static_cast<const unsigned char*>(g.a);
            a.end = a.begin + g.rows * a.pitch;
            a.own = int(q.a0);
            a.own_end = int(rows);
            b.begin = b.at = static_cast<const unsigned char*>(g.b);
            b.end = b.begin + Kind::kPerResult * b.second;
            b.own = int(q.b0);
            b.own_end = int(width);
            a.red_end = b.red_end = int(g.in);
            for (uint32_t block = 0; block < blocks; ++block) {
                a.red = b.red = int(block * kStep);
                GatherPackets<1, false> pa;
                GatherPackets<1, false, Kind::kGated, BN> pb;
                pa.load(a, thread);
                pb.load(b, thread);
                if (!(ok = tc::barrier_wait(done(stage), phase ^ 1, gave_up))) break;
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
