// Low-rank adapters (k14_adapters.cu) on long inputs: windows of 128 rows that hold few adapters, on tensor memory.
//
// A CTA takes 128 consecutive rows and a range of columns.  X and A come by TMA and T = X A^T is accumulated in tensor memory, for every
// adapter of the window over all its rows (a row's own T is picked from its adapter's columns).  T is scaled and split into two fp16 halves
// as in k14_adapters.cu and laid down as the left operand of the second product, which runs over N in steps of 64 columns, once for every
// adapter into an accumulator of its own: what an adapter holds reaches no row of another.  base comes by TMA into a ring of tiles, the
// results are written over it there and leave by TMA, so that no thread addresses global memory and the kernel moves X, base and Y
// once.  Rows are not sorted: prompts bring an adapter's rows together.
//
// Windows with more adapters than tensor memory has columns for are left to k_adapters, which runs behind this kernel over all windows and
// makes the same choice.  Windows without any adapter are copied.
//
// Roles: warp 0 TMA for X, A, then base; warp 1 products; groups of four warps for the results (one per quarter of the tensor memory's
// lanes, the first group also for T), steps of N dealt out in turn so that their chains of latencies overlap; the last warp TMA for B.
// Every wait is bounded; on expiry the CTA raises MUXQ_ERR_TIMEOUT, lets the copies and products of all roles end and returns.
//
// Bound: HBM from some 8192 rows on (16384 x 1280 -> 5120 at rank 64: 384 MB in 72 to 77 us a call, 5.0 to 5.3 TB/s, with the launch of k_adapters
// behind it; this kernel's steps of N run at the rate of HBM, but nothing of them overlaps the first product and T, which took 31 of 125
// thousand cycles), below that the chain window - T - products with few windows for the device.  Taken from 1024 rows on, k_adapters below.  Rows
// alone decide, which suits high ranks and N longer than K and costs the others up to a half until some 2500 rows; us here / k_adapters, four adapters
// in runs, fp16, at 1024, 2048, 3000 rows: 1280 -> 5120 rank 64 17.6 / 21.0, 22.7 / 28.1, 27.4 / 56.6; 768 -> 2304 rank 64 13.9 / 15.3, 15.2 / 17.4,
// 17.6 / 31.5; 1280 -> 5120 rank 16 15.6 / 12.6, 18.9 / 19.3, 23.4 / 38.0; 2560 -> 2560 rank 16 20.8 / 10.6, 22.0 / 14.6, 25.2 / 28.4; 1280 -> 1280
// rank 16 14.0 / 8.8, 14.5 / 9.3, 15.5 / 13.9; fp32 1003 x 1280 -> 5120 rank 32 20.8 / 20.9; 8192 x 768 -> 2304 22.6 / 46, 16384 rows 73 / 179.
// Tried: clusters that divide K among the CTAs of a window and exchange T (the exchange costs 7000 cycles: 2000 rows 18.0 -> 19.6 us,
// 8192 22.8 -> 26.2), eight stages of X instead of four (no change: a stage takes 600 cycles to be issued), three groups of result
// warps (no change).
#include <limits.h>

#include <type_traits>

#include "../../include/muxq.h"
#include "gemm_common.cuh"
#include "k14_adapters.cuh"

namespace muxq {

namespace {

using namespace adapters;

constexpr int kGroups = 2;                // of four result warps; a group takes every kGroups-th step of N
constexpr int kThreads = 32 * (3 + 4 * kGroups), kWarpB = 2 + 4 * kGroups;
constexpr int kUnit = 64;                 // columns of N at a time
constexpr int kBox = 128 * 128;           // bytes of 128 rows x 128 bytes
constexpr int kXRing = 6 * kBox, kMaxX = 6;  // stages of X, 128 x 64, and A, up to 256 rows of 64
constexpr int kTB = 96 * 1024;            // T (32 or 64 KB) and the ring of B
constexpr int kMaxB = 4, kMaxBase = 8;
static_assert(kXRing >= 2 * (kBox + kWindowRanks * 128), "two stages of X and A");
constexpr int kSmem = kTB + 2 * kBox + kXRing + 1024;  // + alignment

// Steps of N that one instruction of the second product covers, so that T, which it reads from shared memory every time, is read less often:
// with one step an instruction the kernel was bound by shared memory (T and B 48 KB of 112 KB a step; 82 us at 16384 x 1280 -> 5120).  As many as
// two accumulators for every adapter have columns for, and two stages of an adapter's B room.
__host__ __device__ constexpr int group_units(int adapters, bool high) { return high || adapters > 2 ? 1 : adapters == 2 ? 2 : 4; }

struct TileParams {
    int M, K, N, slots, max_rank;
    const void *base;
    void *Y;
    int ldbase, ldy;
    const int32_t *row_slot, *rank;
    const float *scale;
    int32_t *dev_status;
    uint32_t spin;
    int skip_chunk;  // -1; a test names a chunk of K whose loads are left out so that a wait runs out
};

__device__ __forceinline__ void mma_f16_elect(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "elect.sync _|q, 0xffffffff;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}\n"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
        : "memory");
}
// fp16 operands, both K-major, fp32 accumulator, 128 rows
__device__ __forceinline__ uint32_t idesc_f16(int n) { return (1u << 4) | ((uint32_t)(n >> 3) << 17) | (8u << 24); }
__device__ __forceinline__ void tma_load_3d_elect(void *dst, const void *map, uint64_t *bar, int c0, int c1, int c2) {
    asm volatile(
        "{\n\t.reg .pred q;\n\t"
        "elect.sync _|q, 0xffffffff;\n\t"
        "@q cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];\n\t}\n"
        ::"r"(smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(map)), "r"(smem_u32(bar)), "r"(c0), "r"(c1), "r"(c2)
        : "memory");
}
__device__ __forceinline__ void mbar_arrive_elect(uint64_t *bar) {
    asm volatile(
        "{\n\t.reg .pred q;\n\t"
        "elect.sync _|q, 0xffffffff;\n\t"
        "@q mbarrier.arrive.shared::cta.b64 _, [%0];\n\t}\n"
        ::"r"(smem_u32(bar))
        : "memory");
}

// Where part i of n begins when they are as even as they come.
__device__ __forceinline__ int part_begin(int total, int i, int n) { return total / n * i + min(i, total % n); }

// A window without adapters: this CTA's columns of base.
template <bool kF32>
__device__ __forceinline__ void copy_window(const TileParams &p, int m0) {
    if (p.base == p.Y) return;
    constexpr int kSize = kF32 ? 4 : 2, kPer = 16 / kSize, kAhead = 4;
    const int words = p.N / kPer, w0 = part_begin(words, blockIdx.y, gridDim.y), n = part_begin(words, blockIdx.y + 1, gridDim.y) - w0;
    const int total = min(128, p.M - m0) * n;
    for (int i = threadIdx.x; i < total; i += kAhead * kThreads) {
        uint4 v[kAhead];
        size_t to[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int j = i + k * kThreads, r = j / n, c = w0 + j - r * n;
            v[k] = make_uint4(0, 0, 0, 0);
            to[k] = ((size_t)(m0 + r) * p.ldy + (size_t)c * kPer) * kSize;
            if (j < total && p.base)
                v[k] = *reinterpret_cast<const uint4 *>(static_cast<const uint8_t *>(p.base) + ((size_t)(m0 + r) * p.ldbase + (size_t)c * kPer) * kSize);
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (i + k * kThreads < total) *reinterpret_cast<uint4 *>(static_cast<uint8_t *>(p.Y) + to[k]) = v[k];
    }
}

template <bool kF32>
__global__ void __launch_bounds__(kThreads, 1)
k_adapter_tiles(const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_b,
                const __grid_constant__ CUtensorMap tm_base, const __grid_constant__ CUtensorMap tm_y, const TileParams p) {
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t x_full[kMaxX], x_empty[kMaxX], b_full[kMaxB], b_even[kMaxB], b_empty[kMaxB], base_full[kMaxBase], base_empty[kMaxBase];
    __shared__ uint64_t t_full, t_ready, acc_full[2], acc_empty[2], drained;
    __shared__ float s_factor[128];
    __shared__ WindowAdapters s_win;
    __shared__ uint32_t s_tmem, s_abort;

    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const int m0 = blockIdx.x * 128;
    if (threadIdx.x == 0) {
        // (the first copy by a map that is not at hand took 3300 cycles to be issued)
        tma_prefetch_desc(&tm_x);
        tma_prefetch_desc(&tm_a);
        tma_prefetch_desc(&tm_b);
        tma_prefetch_desc(&tm_base);
        tma_prefetch_desc(&tm_y);
    }
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // behind the wait: k_adapters may look at the rows at once
    int mine;
    bool bad;
    if (!window_adapters(&s_win, p.row_slot, p.rank, p.slots, p.max_rank, m0, p.M, &mine, &bad)) return;
    if (bad && blockIdx.y == 0) atomicMax(p.dev_status, MUXQ_ERR_INVALID_ARG);
    if (s_win.count == 0) {
        copy_window<kF32>(p, m0);
        return;
    }
    const int d = s_win.count, R8 = p.max_rank, R16 = (R8 + 15) & ~15, R64 = R8 > 64 ? 2 : 1;

    // shared memory: T (upper halves, lower halves) | ring of B | two boxes for base | stages of X and A, later base too
    const uint32_t base_addr = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t *sm = smem_raw + (base_addr - smem_u32(smem_raw));
    const int x_stage = kBox + d * R16 * 128, x_stages = min(kXRing / x_stage, kMaxX);
    const int t_bytes = R64 * 2 * kBox, G = group_units(d, R64 == 2), b_stage = R64 * G * (kBox / 2);
    int b_stages = (kTB - t_bytes) / b_stage;
    if (b_stages > kMaxB) b_stages = kMaxB;
    constexpr int kBaseStage = kF32 ? 2 * kBox : kBox;
    constexpr int kBaseStages = (2 * kBox + kXRing) / kBaseStage;  // 8, fp32 4
    constexpr int kBaseEarly = 2 * kBox / kBaseStage;                          // those that do not lie over X and A
    static_assert(kBaseStages <= kMaxBase && kBaseStages > kGroups, "ring of base (a group gives a tile back with its next one)");
    uint8_t *sm_t = sm, *sm_b = sm + t_bytes, *sm_base = sm + kTB, *sm_x = sm_base + 2 * kBox;

    if (threadIdx.x == 0) {
        for (int i = 0; i < kMaxX; ++i) { mbar_init(&x_full[i], 1); mbar_init(&x_empty[i], 1); }
        for (int i = 0; i < kMaxB; ++i) { mbar_init(&b_full[i], 1); mbar_init(&b_even[i], 1); mbar_init(&b_empty[i], 1); }
        for (int i = 0; i < kMaxBase; ++i) { mbar_init(&base_full[i], 1); mbar_init(&base_empty[i], 4); }
        mbar_init(&t_full, 1);
        mbar_init(&t_ready, 4);
        for (int i = 0; i < 2; ++i) { mbar_init(&acc_full[i], 1); mbar_init(&acc_empty[i], 4 * G); }
        mbar_init(&drained, 1);
        s_abort = 0;
        fence_barrier_init();
    }
    if (warp == 1) {
        tmem_alloc(&s_tmem, 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, s_tmem, 0);
    volatile uint32_t *abort_flag = &s_abort;
    const int chunks = (p.K + 63) >> 6, units = (p.N + kUnit - 1) / kUnit;
    const int u0 = part_begin(units, blockIdx.y, gridDim.y), u1 = part_begin(units, blockIdx.y + 1, gridDim.y);

    if (warp == 0) {
        // ------------------------------------------------------------ X and A, then base
        int issued_x = 0, issued_base = 0;
        bool ok = true;
        auto load_base = [&](int k) {
            const int s = k % kBaseStages;
            if (!mbar_wait_warp(&base_empty[s], ((k / kBaseStages) & 1) ^ 1, abort_flag, p.spin)) return false;
            uint8_t *to = sm_base + s * kBaseStage;
            if (p.base) {
                mbar_expect_tx_elect(&base_full[s], kBaseStage);
                tma_load_2d_elect(to, &tm_base, &base_full[s], (u0 + k) * kUnit, m0);
                if (kF32) tma_load_2d_elect(to + kBox, &tm_base, &base_full[s], (u0 + k) * kUnit + 32, m0);
            } else {
                mbar_arrive_elect(&base_full[s]);
            }
            return true;
        };
        for (; issued_base < kBaseEarly && issued_base < u1 - u0 && ok; ++issued_base) ok = load_base(issued_base);
        for (; issued_x < chunks && ok; ++issued_x) {
            const int s = issued_x % x_stages;
            if (!mbar_wait_warp(&x_empty[s], ((issued_x / x_stages) & 1) ^ 1, abort_flag, p.spin)) { ok = false; break; }
            if (issued_x == p.skip_chunk) continue;
            uint8_t *to = sm_x + s * x_stage;
            mbar_expect_tx_elect(&x_full[s], kBox + d * R8 * 128);
            tma_load_2d_elect(to, &tm_x, &x_full[s], issued_x * 64, m0);
            for (int i = 0; i < d; ++i) tma_load_3d_elect(to + kBox + i * R16 * 128, &tm_a, &x_full[s], issued_x * 64, 0, s_win.slot[i]);
        }
        // the other tiles of base lie over the stages of X and A: free once the first product is done
        if (ok) ok = mbar_wait_warp(&t_full, 0, abort_flag, p.spin);
        for (; issued_base < u1 - u0 && ok; ++issued_base)
            if (!load_base(issued_base)) { ok = false; break; }
        // Every copy that was started lands before the CTA ends, also where this warp was through with all of its own when another one gave up.
        for (int k = issued_x > x_stages ? issued_x - x_stages : 0; k < issued_x; ++k)
            if (k != p.skip_chunk)
                for (uint32_t i = 0; i < kSpinLimit; ++i)
                    if (__all_sync(0xffffffffu, mbar_try_wait(&x_full[k % x_stages], (k / x_stages) & 1))) break;
        for (int k = issued_base > kBaseStages ? issued_base - kBaseStages : 0; k < issued_base; ++k)
            for (uint32_t i = 0; i < kSpinLimit; ++i)
                if (__all_sync(0xffffffffu, mbar_try_wait(&base_full[k % kBaseStages], (k / kBaseStages) & 1))) break;
    } else if (warp == kWarpB) {
        // ------------------------------------------------------------ B, one adapter's for G steps of N at a time
        const int all = (u1 - u0 + G - 1) / G * d;
        int issued = 0;
        bool ok = true;
        // What stands beyond a rank that ends inside a step of 16 is set to zero once it has landed: T has zeros there, but it may be no numbers.
        auto even = [&](int j) {
            const int s = j % b_stages, rows = min(G, u1 - u0 - j / d * G) * kUnit, r = s_win.rank[j % d], end = (r + 15) & ~15;
            if (!mbar_wait_warp(&b_full[s], (j / b_stages) & 1, abort_flag, p.spin)) return false;
            uint8_t *block = sm_b + s * b_stage + (r >> 6) * G * (kBox / 2);
            for (int n = lane; n < rows; n += 32)
                for (int k = r; k < end; ++k)
                    *reinterpret_cast<__half *>(block + n * 128 + (((k & 63) >> 3) ^ (n & 7)) * 16 + (k & 7) * 2) = __float2half_rn(0.0f);
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) mbar_arrive(&b_even[s]);
            return true;
        };
        for (; issued < all && ok; ++issued) {
            const int s = issued % b_stages, u = issued / d * G, n = min(G, u1 - u0 - u);
            if (!mbar_wait_warp(&b_empty[s], ((issued / b_stages) & 1) ^ 1, abort_flag, p.spin)) { ok = false; break; }
            mbar_expect_tx_elect(&b_full[s], R64 * n * (kBox / 2));
            for (int blk = 0; blk < R64; ++blk)
                for (int k = 0; k < n; ++k)
                    tma_load_3d_elect(sm_b + s * b_stage + (blk * G + k) * (kBox / 2), &tm_b, &b_full[s], blk * 64, (u0 + u + k) * kUnit, s_win.slot[issued % d]);
            if (s_win.uneven && issued) ok = even(issued - 1);
        }
        if (ok && s_win.uneven) ok = even(issued - 1);
        for (int k = issued > b_stages ? issued - b_stages : 0; k < issued; ++k)  // (as above)
            for (uint32_t i = 0; i < kSpinLimit; ++i)
                if (__all_sync(0xffffffffu, mbar_try_wait(&b_full[k % b_stages], (k / b_stages) & 1))) break;
    } else if (warp == 1) {
        // ------------------------------------------------------------ products
        // Addresses and descriptors have to be uniform to the compiler, too, or every instruction waits for several moves to uniform registers: they
        // are made of kernel arguments, loop counters and constants, and the number of adapters, which shared memory tells, is one of the latter.
        // All of tensor memory is ours, so it begins at 0.
        const uint32_t sm0 = (smem_u32(smem_raw) + 1023u) & ~1023u;
        auto issue = [&](auto number) {
            constexpr int D = decltype(number)::value;
            const int r16 = (p.max_rank + 15) & ~15, blocks = p.max_rank > 64 ? 2 : 1;
            const int xb = kBox + D * r16 * 128, xs = min(kXRing / xb, kMaxX);
            const int units_g = group_units(D, blocks == 2), bb = blocks * units_g * (kBox / 2), bs = min((kTB - blocks * 2 * kBox) / bb, kMaxB);
            const uint32_t idesc_t = idesc_f16(r16), idesc_y = idesc_f16(units_g * kUnit);
            const uint64_t x_desc = smem_desc_sw128(sm0 + kTB + 2 * kBox);
            for (int c = 0, st = 0, ph = 0; c < chunks; ++c) {
                if (!mbar_wait_warp(&x_full[st], ph, abort_flag, p.spin)) return false;
                tc_fence_after();
                const uint64_t xd = x_desc + (uint64_t)(uint32_t)(st * (xb >> 4));
                const int steps = (p.K - c * 64 + 15) >> 4;  // of 16
#pragma unroll
                for (int i = 0; i < D; ++i)
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (k < steps) mma_f16_elect(i * r16, xd + 2 * k, xd + (uint64_t)(uint32_t)((kBox >> 4) + i * r16 * 8 + 2 * k), idesc_t, k ? 1u : c ? 1u : 0u);
                mma_commit_elect(&x_empty[st]);
                if (++st == xs) { st = 0; ph ^= 1; }
            }
            mma_commit_elect(&t_full);
            if (!mbar_wait_warp(&t_ready, 0, abort_flag, p.spin)) return false;
            tc_fence_after();
            const bool uneven = s_win.uneven != 0;
            uint32_t packed = 0;  // steps of 16 ranks of every adapter
#pragma unroll
            for (int i = 0; i < D; ++i) packed |= (uint32_t)((s_win.rank[i] + 15) >> 4) << (8 * i);
            const uint64_t t_desc = smem_desc_sw128(sm0), b_desc = smem_desc_sw128(sm0 + blocks * 2 * kBox);
            const int count = (u1 - u0 + units_g - 1) / units_g;
            for (int u = 0, st = 0, ph = 0, buf = 0, bph = 1; u < count; ++u) {
                if (!mbar_wait_warp(&acc_empty[buf], bph, abort_flag, p.spin)) return false;
                tc_fence_after();
                auto products = [&](auto blocks_c, int i) {
                    constexpr int kB = decltype(blocks_c)::value, kG = group_units(D, kB == 2);  // blocks of 64 ranks
                    const int steps = packed >> (8 * i) & 0xff;
                    const uint64_t bd = b_desc + (uint64_t)(uint32_t)(st * (bb >> 4));
#pragma unroll
                    for (int half = 0; half < 2; ++half)
#pragma unroll
                        for (int k = 0; k < 4 * kB; ++k)
                            if (k < steps)
                                mma_f16_elect(buf * 256 + i * kG * kUnit, t_desc + (uint64_t)((half * kB + (k >> 2)) * (kBox >> 4) + (k & 3) * 2),
                                              bd + (uint64_t)((k >> 2) * kG * (kBox >> 5) + (k & 3) * 2), idesc_y, half || k ? 1u : 0u);
                };
#pragma unroll
                for (int i = 0; i < D; ++i) {
                    if (!mbar_wait_warp(uneven ? &b_even[st] : &b_full[st], ph, abort_flag, p.spin)) return false;
                    tc_fence_after();
                    if (blocks == 1) products(std::integral_constant<int, 1>{}, i);
                    else products(std::integral_constant<int, 2>{}, i);
                    mma_commit_elect(&b_empty[st]);
                    if (++st == bs) { st = 0; ph ^= 1; }
                }
                mma_commit_elect(&acc_full[buf]);
                if (++buf == 2) { buf = 0; bph ^= 1; }
            }
            return true;
        };
        switch (d) {
            case 1: issue(std::integral_constant<int, 1>{}); break;
            case 2: issue(std::integral_constant<int, 2>{}); break;
            case 3: issue(std::integral_constant<int, 3>{}); break;
            default: issue(std::integral_constant<int, 4>{}); break;
        }
        mma_commit_elect(&drained);  // products that are on their way end before their memory is given back
        for (uint32_t i = 0; i < kSpinLimit; ++i)
            if (__all_sync(0xffffffffu, mbar_try_wait(&drained, 0))) break;
    } else {
        // ------------------------------------------------------------ T, then the results
        const int quad = warp & 3, group = (warp - 2) >> 2, row = quad * 32 + lane;
        const int own = s_win.index[row];
        uint32_t present = 0;  // adapters among this warp's rows
        for (int i = 0; i < d; ++i) present |= __any_sync(0xffffffffu, own == i) ? 1u << i : 0u;
        const uint32_t taddr = tmem + ((uint32_t)(quad * 32) << 16);
        bool ok = true;
        if (group == 0) {
            ok = mbar_wait_warp(&t_full, 0, abort_flag, p.spin);
            if (ok) {
                tc_fence_after();
                const int r = own >= 0 ? s_win.rank[own] : 0;
                float most = 0.0f;
                for (int i = 0; i < d; ++i) {
                    if (!(present >> i & 1)) continue;
                    for (int c = 0; c < R16; c += 16) {
                        uint32_t v[16];
                        tmem_ld_32x16(taddr + i * R16 + c, v);
                        tmem_ld_wait();
#pragma unroll
                        for (int j = 0; j < 16; ++j)
                            if (own == i && c + j < r) most = fmaxf(most, fabsf(__uint_as_float(v[j])));
                    }
                }
                float up, down;
                row_factors(most, &up, &down);
                s_factor[row] = own >= 0 ? (p.scale ? p.scale[s_win.slot[own]] : 1.0f) * down : 0.0f;
                for (int i = 0; i < d; ++i) {
                    if (!(present >> i & 1)) continue;
                    for (int c = 0; c < R16; c += 16) {
                        uint32_t v[16];
                        tmem_ld_32x16(taddr + i * R16 + c, v);
                        tmem_ld_wait();
                        alignas(16) __half hi[16], lo[16];
#pragma unroll
                        for (int j = 0; j < 16; ++j) split(c + j < r ? __uint_as_float(v[j]) * up : 0.0f, &hi[j], &lo[j]);
                        if (own == i) {
                            uint8_t *to = sm_t + (c >> 6) * kBox + row * 128;
#pragma unroll
                            for (int k = 0; k < 2; ++k) {
                                const int at = ((((c & 63) >> 3) + k) ^ (row & 7)) * 16;
                                *reinterpret_cast<uint4 *>(to + at) = *reinterpret_cast<const uint4 *>(hi + 8 * k);
                                *reinterpret_cast<uint4 *>(to + R64 * kBox + at) = *reinterpret_cast<const uint4 *>(lo + 8 * k);
                            }
                        }
                    }
                }
                tc_fence_before();
                fence_proxy_async();
                __syncwarp();
                if (lane == 0) mbar_arrive(&t_ready);
            }
        }
        if (ok) ok = mbar_wait_warp(&t_ready, 0, abort_flag, p.spin);
        const float f = ok ? s_factor[row] : 0.0f;
        const int first = present ? __ffs(present) - 1 : 0;
        int last = -1;  // tile of base whose store may still be reading it
        for (int u = group; u < u1 - u0 && ok; u += kGroups) {
            const int s = u % kBaseStages, step = u / G, buf = step & 1;
            if (!mbar_wait_warp(&acc_full[buf], (step >> 1) & 1, abort_flag, p.spin)) { ok = false; break; }
            tc_fence_after();
            uint32_t v[64];
            const uint32_t from = taddr + buf * 256 + (u - step * G) * kUnit;
            tmem_ld_32x32(from + first * G * kUnit, *reinterpret_cast<uint32_t(*)[32]>(v));
            tmem_ld_32x32(from + first * G * kUnit + 32, *reinterpret_cast<uint32_t(*)[32]>(v + 32));
            tmem_ld_wait();
            for (uint32_t more = present & (present - 1); more; more &= more - 1) {  // another adapter among these rows
                const int i = __ffs(more) - 1;
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    uint32_t w[16];
                    tmem_ld_32x16(from + i * G * kUnit + 16 * h, w);
                    tmem_ld_wait();
#pragma unroll
                    for (int j = 0; j < 16; ++j) v[16 * h + j] = own == i ? w[j] : v[16 * h + j];
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&acc_empty[buf]);
            if (!mbar_wait_warp(&base_full[s], (u / kBaseStages) & 1, abort_flag, p.spin)) { ok = false; break; }
            uint8_t *tile = sm_base + s * kBaseStage, *at = tile + row * 128;
            if (own < 0) {  // base as it is
                if (!p.base)
                    for (int c = 0; c < kBaseStage / kBox * 8; ++c) *reinterpret_cast<uint4 *>(at + (c >> 3) * kBox + (c & 7) * 16) = make_uint4(0, 0, 0, 0);
            } else if (kF32) {
#pragma unroll
                for (int c = 0; c < 16; ++c) {
                    float4 *q = reinterpret_cast<float4 *>(at + (c >> 3) * kBox + ((c & 7) ^ (row & 7)) * 16);
                    const float4 b = p.base ? *q : make_float4(0.f, 0.f, 0.f, 0.f);
                    *q = make_float4(__fmaf_rn(f, __uint_as_float(v[4 * c]), b.x), __fmaf_rn(f, __uint_as_float(v[4 * c + 1]), b.y),
                                     __fmaf_rn(f, __uint_as_float(v[4 * c + 2]), b.z), __fmaf_rn(f, __uint_as_float(v[4 * c + 3]), b.w));
                }
            } else {
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    uint4 *q = reinterpret_cast<uint4 *>(at + (c ^ (row & 7)) * 16);
                    uint4 b = p.base ? *q : make_uint4(0, 0, 0, 0);
                    __half2 *h = reinterpret_cast<__half2 *>(&b);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float2 x = __half22float2(h[j]);
                        h[j] = __floats2half2_rn(__fmaf_rn(f, __uint_as_float(v[8 * c + 2 * j]), x.x), __fmaf_rn(f, __uint_as_float(v[8 * c + 2 * j + 1]), x.y));
                    }
                    *q = b;
                }
            }
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) {  // this warp's 32 rows
                const int col = (u0 + u) * kUnit, r0 = m0 + quad * 32;
                if (r0 < p.M) {
                    tma_store_2d(&tm_y, tile + quad * 4096, col, r0);
                    if (kF32 && col + 32 < p.N) tma_store_2d(&tm_y, tile + kBox + quad * 4096, col + 32, r0);
                }
                tma_store_commit();
                tma_store_wait_read<1>();  // the tile before this one may be loaded over
                if (last >= 0) mbar_arrive(&base_empty[last]);
            }
            last = s;
            __syncwarp();
        }
        if (lane == 0) {
            tma_store_wait_read<0>();
            if (ok && last >= 0) mbar_arrive(&base_empty[last]);
        }
    }
    // ---------------------------------------------------------------- teardown
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        __syncwarp();
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
    if (threadIdx.x == 0 && s_abort) atomicMax(p.dev_status, MUXQ_ERR_TIMEOUT);
}

// fp16 or fp32 matrices and stacks of matrices, boxes 128 bytes wide, 128-byte swizzle; what lies outside reads as zero
bool make_map(CUtensorMap *map, const void *p, bool f32, int dims, const uint64_t (&size)[3], const uint64_t (&pitch)[2], int box_rows) {
    gemm::EncodeTiledFn fn = gemm::get_encode_fn();
    if (!fn) return false;
    const uint64_t esz = f32 ? 4 : 2;
    cuuint64_t d[3] = {size[0], size[1], size[2]}, st[2] = {pitch[0] * esz, pitch[1] * esz};
    cuuint32_t box[3] = {(cuuint32_t)(128 / esz), (cuuint32_t)box_rows, 1}, one[3] = {1, 1, 1};
    return fn(map, f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, dims, const_cast<void *>(p), d, st, box, one,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <bool kF32>
cudaError_t launch_form(const AdapterArgs &a, const CUtensorMap (&m)[5], const TileParams &p, int parts, cudaStream_t s) {
    static PerDevice<int> done;
    const int dev = current_device();
    if (dev < 0) return cudaErrorInvalidDevice;
    {
        std::lock_guard<std::mutex> lock(device_mutex());
        if (!done.have[dev]) {
            const cudaError_t e = cudaFuncSetAttribute(reinterpret_cast<const void *>(k_adapter_tiles<kF32>), cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
            if (e != cudaSuccess) return e;
            done.have[dev] = true;
        }
    }
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(((long long)a.M + 127) / 128), parts);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = kSmem;
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, k_adapter_tiles<kF32>, m[0], m[1], m[2], m[3], m[4], p);
}

constexpr int kMinRows = 1024;

}  // namespace

bool launch_adapter_tiles(const AdapterArgs &a, cudaStream_t s, cudaError_t *e) {
    const int sms = num_sms();
    if (a.M < kMinRows || sms < 1) return false;
    const int64_t far = (int64_t)1 << 38;  // elements; a map's strides end at 2^40 bytes
    if (a.stride_a > far || a.stride_b > far) return false;
    CUtensorMap m[5];
    const bool f32 = a.out_f32;
    const uint64_t M = a.M, K = a.K, N = a.N, R = a.max_rank, S = a.slots;
    const uint64_t sa = S > 1 ? (uint64_t)a.stride_a : R * a.lda, sb = S > 1 ? (uint64_t)a.stride_b : N * a.ldb;
    if (!make_map(&m[0], a.X, false, 2, {K, M, 1}, {(uint64_t)a.ldx, 0}, 128) || !make_map(&m[1], a.A, false, 3, {K, R, S}, {(uint64_t)a.lda, sa}, a.max_rank) ||
        !make_map(&m[2], a.B, false, 3, {R, N, S}, {(uint64_t)a.ldb, sb}, kUnit) ||
        !make_map(&m[3], a.base ? a.base : a.Y, f32, 2, {N, M, 1}, {(uint64_t)(a.base ? a.ldbase : a.ldy), 0}, 128) ||
        !make_map(&m[4], a.Y, f32, 2, {N, M, 1}, {(uint64_t)a.ldy, 0}, 32))
        return false;
    TileParams p{};
    p.M = a.M; p.K = a.K; p.N = a.N; p.slots = a.slots; p.max_rank = a.max_rank;
    p.row_slot = a.row_slot; p.rank = a.rank; p.scale = a.scale;
    p.base = a.base; p.Y = a.Y; p.ldbase = a.ldbase; p.ldy = a.ldy;
    p.dev_status = a.dev_status;
    p.spin = test_hooks().spin_limit ? test_hooks().spin_limit : kSpinLimit;
    p.skip_chunk = test_hooks().gemm_skip_kb - 1;
    // CTAs that share a window's columns: the fewest cycles of the fullest SM, each CTA doing all of the first product (cycles by the kernel's own
    // clock).  More of them than the device holds at once only where that is clearly less: 10525 rows, 1448 -> 3880 at rank 128 in fp32 107 -> 99 us,
    // 10000 rows, 1280 -> 3840, 51.6 -> 50.3, but 12000 rows, 768 -> 2560, 38.1 -> 39.4 where the estimate gained 2 %.
    const int units = (a.N + kUnit - 1) / kUnit, chunks = (a.K + 63) / 64;
    const long long tiles = ((long long)a.M + 127) / 128;
    int parts = 1;
    double best = 0.0;
    for (int n = 1; n <= units && (n == 1 || tiles * n <= 4 * sms); ++n) {
        const double cost = (double)((tiles * n + sms - 1) / sms) * (5000.0 + 700.0 * chunks + (f32 ? 2000.0 : 1200.0) * ((units + n - 1) / n));
        if (n > 1 && cost >= (tiles * n > sms ? 0.95 : 1.0) * best) continue;
        best = cost;
        parts = n;
    }
    *e = f32 ? launch_form<true>(a, m, p, parts, s) : launch_form<false>(a, m, p, parts, s);
    return true;
}

}  // namespace muxq
