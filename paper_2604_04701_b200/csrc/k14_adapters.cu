// Low-rank adapters of many requests beside a shared projection:
//   Y[m] = base[m] + s_a * (X[m] A_a^T) B_a^T,   a = slot[m]
// in one launch.  A cluster of CTAs takes a window of consecutive token rows.  It sorts them by adapter, so that rows of one adapter
// share m16 tiles of matrix instructions wherever in the window they stand; its CTAs divide K between them for T = X A^T, exchange
// their parts of T through distributed shared memory, and divide N for T B^T.
//
// T is held in fp32.  For the second product every row of T is scaled by a power of two (exact; undone in fp32 afterwards) and split into two
// fp16 numbers whose sum has 22 bits of it: one fp16 number alone would put an error of 2^-11 on an fp32 result, and rows
// of large activations would leave its range.
//
// The matrix instructions are the ones that read registers (m16n8k16): the operator is bound by latencies and by memory here, and operands
// whose order of k may be chosen freely go from global memory to registers in whole 16-byte words without a detour; n is permuted so that a
// thread ends up with eight neighbouring results.  Long inputs go to k_adapter_tiles first (k15_adapter_tiles.cu).
//
// Bound: one chain of latencies at decode steps -- row_slot, then X and A, the parts of T through the cluster, T B^T -- of about 6200 cycles
// behind the wait for the launch before (1 x 768 -> 768 rank 8 in a row of calls 3.9 us, 16 x 1280 -> 3840 with 16 adapters 5.4); what shaped it, us of the first:
// 64-bit divisions for a CTA's share of K and N 4.8 -> 4.1, parts of T pushed by stores instead of fetched behind the barrier and rows
// ordered by one warp 5.9 -> 4.8.  Between, memory: 1003 x 1280 -> 5120 rank 32 20.6 us, its columns of N at 4.8 TB/s.
#include "../../include/muxq.h"
#include "k14_adapters.cuh"

namespace muxq {

namespace {

using namespace adapters;

constexpr int kT = 256, kWarps = kT / 32;
constexpr int kMostRows = 32;     // of a window: a warp puts them in order
constexpr int kSmemMost = 220 * 1024;

__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void st_cluster_f4(uint32_t addr, const float4 &v) {
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}

// Rows of T parts (fp32) and of T itself (per four ranks: four upper halves, four lower halves); the pitches keep the eight rows of
// a fragment on different banks.
template <int NR> __host__ __device__ constexpr int part_pitch() { return NR * 8 + 8; }                              // floats
template <int NR> __host__ __device__ constexpr int t_pitch() { return (NR * 32 / 64 | 1) * 64; }                    // bytes
template <int NR> __host__ __device__ constexpr int part_rows(int W) { return W * kWarps < 128 ? W * kWarps : 128; }  // slices of K times rows (W <= 128)
template <int NR> __host__ __device__ constexpr size_t smem_bytes(int W, int C) {  // parts of all CTAs, then this one's own, which T replaces
    const size_t own = (size_t)part_rows<NR>(W) * part_pitch<NR>() * 4, t = (size_t)W * t_pitch<NR>();
    return (size_t)C * W * part_pitch<NR>() * 4 + (own > t ? own : t);
}

// eight neighbouring results
__device__ __forceinline__ void add_store(__half *y, const uint4 &b, const float (&v)[8], float f) {
    const __half2 *h = reinterpret_cast<const __half2 *>(&b);
    uint4 o;
    __half2 *q = reinterpret_cast<__half2 *>(&o);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 c = __half22float2(h[i]);
        q[i] = __floats2half2_rn(__fmaf_rn(f, v[2 * i], c.x), __fmaf_rn(f, v[2 * i + 1], c.y));
    }
    *reinterpret_cast<uint4 *>(y) = o;
}
struct Eight32 { float4 a, b; };
__device__ __forceinline__ void add_store(float *y, const Eight32 &b, const float (&v)[8], float f) {
    float4 *o = reinterpret_cast<float4 *>(y);
    o[0] = make_float4(__fmaf_rn(f, v[0], b.a.x), __fmaf_rn(f, v[1], b.a.y), __fmaf_rn(f, v[2], b.a.z), __fmaf_rn(f, v[3], b.a.w));
    o[1] = make_float4(__fmaf_rn(f, v[4], b.b.x), __fmaf_rn(f, v[5], b.b.y), __fmaf_rn(f, v[6], b.b.z), __fmaf_rn(f, v[7], b.b.w));
}
// ranks of a word from `left` on are set to zero
__device__ __forceinline__ uint32_t mask_pair(uint32_t v, int left) { return left >= 2 ? v : left == 1 ? v & 0xffffu : 0u; }
__device__ __forceinline__ void mask_beyond(uint2 &w, int left) {
    w.x = mask_pair(w.x, left);
    w.y = mask_pair(w.y, left - 2);
}
__device__ __forceinline__ void mask_beyond(uint4 &w, int left) {
    w.x = mask_pair(w.x, left);
    w.y = mask_pair(w.y, left - 2);
    w.z = mask_pair(w.z, left - 4);
    w.w = mask_pair(w.w, left - 6);
}
template <bool wide> struct BWordOf { using type = uint4; };
template <> struct BWordOf<false> { using type = uint2; };
template <typename T> struct EightOf;
template <> struct EightOf<__half> { using type = uint4; };
template <> struct EightOf<float> { using type = Eight32; };

template <int kRows>
struct Tiles {  // a window's rows in order of their adapters
    int row[kRows];      // by position: row within the window
    int slot[kRows];     // by position; rows without an adapter come last
    int rank[kRows];     // by position: its adapter's rank, 0, which adds nothing, where it is out of range
    float scale[kRows], factor[kRows]; // by position: its adapter's scale; what T B^T is multiplied by
    int pos[kRows], count[kRows];  // by tile: first position, rows (up to 16)
    int tiles, active;   // positions with an adapter
};

// Puts the rows of a window in order: one adapter's behind one another, tiles of up to 16 of them.  Called by a whole warp, lane = row.
__device__ __forceinline__ void order_rows(Tiles<kMostRows> *s, int key, int rows) {
    const int lane = threadIdx.x & 31;
    const uint32_t valid = rows == 32 ? 0xffffffffu : (1u << rows) - 1u, below = (1u << lane) - 1u;
    const uint32_t peers = __match_any_sync(0xffffffffu, key) & valid;
    const bool with = key != INT_MAX;
    const int same = __popc(peers & below), of_key = __popc(peers);
    // in the order of the adapters' first rows: positions and tiles before each of them, in one sum
    const uint32_t mine = with && !same ? (uint32_t)of_key | (uint32_t)((of_key + 15) >> 4) << 16 : 0u;
    uint32_t sum = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t v = __shfl_up_sync(0xffffffffu, sum, o);
        if (lane >= o) sum += v;
    }
    const uint32_t total = __shfl_sync(0xffffffffu, sum, 31), before = __shfl_sync(0xffffffffu, sum - mine, peers ? __ffs(peers) - 1 : 0);
    const int active = total & 0xffff;
    const uint32_t without = __ballot_sync(0xffffffffu, !with) & valid;
    if (lane < rows) {
        const int at = with ? (int)(before & 0xffff) + same : active + __popc(without & below);
        s->row[at] = lane;
        s->slot[at] = with ? key : -1;
        if (with && same % 16 == 0) {
            const int i = (int)(before >> 16) + same / 16;
            s->pos[i] = at;
            s->count[i] = min(16, of_key - same);
        }
    }
    if (lane == 0) {
        s->tiles = total >> 16;
        s->active = active;
    }
}

// The same for 128 rows, by a whole CTA: every row counts those that come before it.
__device__ __forceinline__ void order_rows(Tiles<kWindow> *s, int key, int rows) {
    __shared__ int keys[kWindow];
    __shared__ bool start[kWindow];
    const int tid = threadIdx.x;
    if (tid < rows) keys[tid] = key;
    const int active = __syncthreads_count(key != INT_MAX);
    int at = 0, same = 0, of_key = 0;
    if (tid < rows) {
        for (int j = 0; j < rows; ++j) {
            const int k = keys[j];
            at += k < key || (k == key && j < tid);
            same += k == key && j < tid;
            of_key += k == key;
        }
        s->row[at] = tid;
        s->slot[at] = key == INT_MAX ? -1 : key;
    }
    const bool first = key != INT_MAX && same % 16 == 0;
    if (tid < rows) start[tid] = first;
    const int tiles = __syncthreads_count(first);
    if (first) {
        int i = same / 16;
        for (int j = 0; j < rows; ++j) i += start[j] && keys[j] < key;
        s->pos[i] = at;
        s->count[i] = min(16, of_key - same);
    }
    if (tid == 0) {
        s->tiles = tiles;
        s->active = active;
    }
}

// kBehind: windows of 128 rows that k_adapter_tiles has left (k15_adapter_tiles.cu).  Larger windows have more rows of an adapter to share its
// A and B: 12000 rows of 16 adapters in any order, 1280 -> 2560, rank 64: 560 us with windows of 32 rows, 321 with these.
template <int NR, typename TO, bool kBehind>
__global__ void __launch_bounds__(kT, NR > 8 ? 1 : 2) k_adapters(const AdapterArgs a, int W, int log_c) {
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ Tiles<kBehind ? kWindow : kMostRows> s;
    constexpr int kPP = part_pitch<NR>(), kTP = t_pitch<NR>();
    // A lane of the second product holds eight neighbouring ranks of T and B (two instructions' worth), four where ranks end at 16
    constexpr bool kWide = NR >= 4;
    constexpr int kLane = kWide ? 8 : 4;
    using Eight = typename EightOf<TO>::type;
    using BWord = typename BWordOf<kWide>::type;
    const int C = 1 << log_c;
    float *all = reinterpret_cast<float *>(smem), *part = all + (size_t)C * W * kPP;
    uint8_t *tsm = reinterpret_cast<uint8_t *>(part);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    const int cta = C > 1 ? (int)cluster_ctarank() : 0;
    const int m0 = (int)(blockIdx.x >> log_c) * W, rows = min(W, a.M - m0);
    if constexpr (kBehind) {
        // k_adapter_tiles lets this kernel start behind its own wait, so what both read is there.  It has done the 128 rows that these belong to,
        // or does not touch them; either way this kernel must not end before that one has.
        __shared__ WindowAdapters s_win;
        int mine;
        bool bad;
        asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
        if (window_adapters(&s_win, a.row_slot, a.rank, a.slots, a.max_rank, m0 / kWindow * kWindow, a.M, &mine, &bad)) {
            asm volatile("griddepcontrol.wait;" ::: "memory");
            return;
        }
    } else {
        asm volatile("griddepcontrol.wait;" ::: "memory");
        asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // behind the wait: a layer kernel may read its W_q at once
    }

    if (C > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");  // waited for before anything is sent

    // ---- rows in order of their adapters
    if (kBehind || warp == 0) {
        int key = INT_MAX;
        if (tid < rows) {
            const int slot = a.row_slot[m0 + tid];
            if (slot >= 0 && slot < a.slots) key = slot;
            else if (slot != -1 && cta == 0) atomicMax(a.dev_status, MUXQ_ERR_INVALID_ARG);
        }
        order_rows(&s, key, rows);
    }
    __syncthreads();
    const int tiles = s.tiles, active = s.active;
    // ranks and scales are on their way beside the first operands
    int my_rank = 0;
    float my_scale = 1.0f;
    if (tid < active) {
        const int slot = s.slot[tid];
        my_rank = a.rank ? a.rank[slot] : a.max_rank;
        if (a.scale) my_scale = a.scale[slot];
    }

    // ---- T = X A^T: this CTA's part of K.  With fewer tiles than warps the warps divide it further.
    int lanes_t = 1;  // warps side by side on different tiles: tiles rounded up to a power of two, at most all
    while (lanes_t < kWarps && lanes_t < tiles) lanes_t *= 2;
    const int k_chunks = (a.K + 31) >> 5, c0 = k_chunks * cta >> log_c, c1 = k_chunks * (cta + 1) >> log_c;
    const int slices = max(1, min(kWarps / lanes_t, c1 - c0)), wt = warp & (lanes_t - 1), wk = warp / lanes_t;
    if (wk < slices) {
        for (int i = wt; i < tiles; i += lanes_t) {
            const int p0 = s.pos[i], n = s.count[i];
            float acc[NR][4];
#pragma unroll
            for (int j = 0; j < NR; ++j) acc[j][0] = acc[j][1] = acc[j][2] = acc[j][3] = 0.0f;
            const bool in0 = g < n, in1 = g + 8 < n;
            const __half *x0 = a.X + (size_t)(m0 + s.row[in0 ? p0 + g : p0]) * a.ldx + 8 * t;
            const __half *x1 = a.X + (size_t)(m0 + s.row[in1 ? p0 + g + 8 : p0]) * a.ldx + 8 * t;
            const __half *A = a.A + (size_t)s.slot[p0] * a.stride_a + (size_t)g * a.lda + 8 * t;
            const uint4 z = make_uint4(0, 0, 0, 0);
            constexpr int kAhead = 2;  // chunks of X that are on their way while as many are worked on
            uint4 u[kAhead], v[kAhead];
            auto load_x = [&](int c) {
#pragma unroll
                for (int d = 0; d < kAhead; ++d) {
                    const int cc = c + d * slices;
                    const bool in = cc < c1 && cc * 32 + 8 * t < a.K;
                    u[d] = in && in0 ? *reinterpret_cast<const uint4 *>(x0 + cc * 32) : z;
                    v[d] = in && in1 ? *reinterpret_cast<const uint4 *>(x1 + cc * 32) : z;
                }
            };
            load_x(c0 + wk);
            // Rows of A beyond the rank are in memory and their products are not used: where there are at most 16, nothing waits for the
            // rank; beyond that what need not be read is worth the wait.
            const int r = NR <= 2 ? a.max_rank : min(a.rank ? a.rank[s.slot[p0]] : a.max_rank, a.max_rank);
            for (int c = c0 + wk; c < c1; c += kAhead * slices) {
                uint4 xu[kAhead], xv[kAhead];
#pragma unroll
                for (int d = 0; d < kAhead; ++d) {
                    xu[d] = u[d];
                    xv[d] = v[d];
                }
                load_x(c + kAhead * slices);
                constexpr int kA = NR <= 4 ? kAhead : 1;  // chunks whose A is on its way at once
#pragma unroll
                for (int d = 0; d < kAhead; d += kA) {
                    if (kA == 1 && c + d * slices >= c1) break;
                    uint4 w[kA][NR];
#pragma unroll
                    for (int e = 0; e < kA; ++e) {
                        const int cc = c + (d + e) * slices;
                        const bool in = cc < c1 && cc * 32 + 8 * t < a.K;
#pragma unroll
                        for (int j = 0; j < NR; ++j) w[e][j] = in && j * 8 < r ? *reinterpret_cast<const uint4 *>(A + (size_t)j * 8 * a.lda + cc * 32) : z;
                    }
#pragma unroll
                    for (int e = 0; e < kA; ++e)
#pragma unroll
                        for (int j = 0; j < NR; ++j) {
                            if (j * 8 < r) {
                                mma16816(acc[j], xu[d + e].x, xv[d + e].x, xu[d + e].y, xv[d + e].y, w[e][j].x, w[e][j].y);
                                mma16816(acc[j], xu[d + e].z, xv[d + e].z, xu[d + e].w, xv[d + e].w, w[e][j].z, w[e][j].w);
                            }
                        }
                }
            }
            float *to = part + (size_t)(wk * active + p0) * kPP + 2 * t;
#pragma unroll
            for (int j = 0; j < NR; ++j) {
                if (j * 8 < r) {
                    if (in0) *reinterpret_cast<float2 *>(to + g * kPP + j * 8) = make_float2(acc[j][0], acc[j][1]);
                    if (in1) *reinterpret_cast<float2 *>(to + (g + 8) * kPP + j * 8) = make_float2(acc[j][2], acc[j][3]);
                }
            }
        }
    }
    if (tid < active) {
        const bool bad = my_rank < 0 || my_rank > a.max_rank;
        if (bad && cta == 0) atomicMax(a.dev_status, MUXQ_ERR_INVALID_ARG);
        s.rank[tid] = bad ? 0 : my_rank;
        s.scale[tid] = my_scale;
    }
    __syncthreads();

    // ---- what the second product reads beside T: on its way before T is there
    const int chunks = (a.N + 31) >> 5, q0 = chunks * cta >> log_c, q1 = chunks * (cta + 1) >> log_c;
    const int rounds = q1 - q0 > warp ? (q1 - q0 - warp + kWarps - 1) / kWarps : 0;  // this warp's steps of 32 columns
    const TO *base = static_cast<const TO *>(a.base);
    TO *Y = static_cast<TO *>(a.Y);
    const Eight none{};
    BWord bw[kWide ? NR / 4 : 1][4];
    int b_rank = 0;  // of the adapter whose B this is
    Eight next0 = none, next1 = none;
    // B of the next tile or the next columns, where there are registers for it
    constexpr bool kAheadB = NR <= 4;
    BWord bn[kAheadB ? (kWide ? NR / 4 : 1) : 1][kAheadB ? 4 : 1];
    auto load_b = [&](auto &to, int i, int q) {
        const int p0 = s.pos[i], r = s.rank[p0];
        const __half *B = a.B + (size_t)s.slot[p0] * a.stride_b + kLane * t;
#pragma unroll
        for (int k = 0; k < (kWide ? NR / 4 : 1); ++k) {
            const int k0 = 4 * kLane * k + kLane * t;  // this lane's first rank
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int col = q * 32 + (g >> 1) * 8 + 2 * j + (g & 1);
                BWord w{};
                if (col < a.N && k0 < (NR <= 2 ? a.max_rank : r)) w = *reinterpret_cast<const BWord *>(B + (size_t)col * a.ldb + 4 * kLane * k);
                to[k][j] = w;
            }
        }
    };
    auto mask_b = [&]() {  // ranks beyond the adapter's own are not looked at
        if (NR <= 2 ? b_rank == a.max_rank : b_rank % kLane == 0) return;
#pragma unroll
        for (int k = 0; k < (kWide ? NR / 4 : 1); ++k) {
            const int k0 = 4 * kLane * k + kLane * t;
            if (k0 + kLane > b_rank)
#pragma unroll
                for (int j = 0; j < 4; ++j) mask_beyond(bw[k][j], b_rank - k0);
        }
    };
    auto load_base = [&](int i, int q) {
        const int p0 = s.pos[i], n = s.count[i], n0 = q * 32 + 8 * t;
        const bool in = base && n0 < a.N;
        next0 = in && g < n ? *reinterpret_cast<const Eight *>(base + (size_t)(m0 + s.row[p0 + g]) * a.ldbase + n0) : none;
        next1 = in && g + 8 < n ? *reinterpret_cast<const Eight *>(base + (size_t)(m0 + s.row[p0 + g + 8]) * a.ldbase + n0) : none;
    };
    if (rounds && tiles) {
        load_b(bw, 0, q0 + warp);
        load_base(0, q0 + warp);
    }
    // ---- this CTA's part of T to every CTA of the cluster
    if (C > 1) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");  // they have all started
    for (int i = tid; i < active * NR * 2; i += kT) {
        const int p = i / (NR * 2), r = (i - p * (NR * 2)) * 4;
        float4 v = *reinterpret_cast<const float4 *>(part + p * kPP + r);
        for (int k = 1; k < slices; ++k) {
            const float4 w = *reinterpret_cast<const float4 *>(part + (k * active + p) * kPP + r);
            v = make_float4(v.x + w.x, v.y + w.y, v.z + w.z, v.w + w.w);
        }
        float *to = all + (size_t)(cta * W + p) * kPP + r;
        if (C == 1) {
            *reinterpret_cast<float4 *>(to) = v;
        } else {
            const uint32_t at = smem_u32(to);
#pragma unroll 8
            for (int c = 0; c < C; ++c) st_cluster_f4(map_to_cta(at, c), v);
        }
    }
    if (C > 1) cluster_sync_all();
    else __syncthreads();

    // ---- the whole of T, scaled and split, where this CTA's own parts were
    for (int p = warp; p < active; p += kWarps) {
        constexpr int kPer = (NR * 8 + 31) / 32;
        const int r = s.rank[p];
        float v[kPer], most = 0.0f;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int j = lane + 32 * i;
            v[i] = 0.0f;
            if (j < r) {
#pragma unroll 8
                for (int c = 0; c < C; ++c) v[i] += all[(size_t)(c * W + p) * kPP + j];
            }
            most = fmaxf(most, fabsf(v[i]));
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
        float up, down;
        row_factors(most, &up, &down);
        uint8_t *to = tsm + p * kTP;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int j = lane + 32 * i;
            if (j < NR * 8) {
                __half hi, lo;
                split(v[i] * up, &hi, &lo);
                const int at = kWide ? j * 2 : (j >> 2) * 16 + (j & 3) * 2;
                *reinterpret_cast<__half *>(to + at) = hi;
                *reinterpret_cast<__half *>(to + at + (kWide ? NR * 16 : 8)) = lo;
            }
        }
        if (lane == 0) s.factor[p] = r ? s.scale[p] * down : -0.0f;  // (-0 x 0 leaves every base as it is, -0 too)
    }
    __syncthreads();

    // ---- Y = base + T B^T: this CTA's part of N.  A warp takes 32 columns through all tiles: B stays in registers from a tile to the
    // next of the same adapter, base comes one tile ahead.
    for (int i = 0, q = q0 + warp, fresh = 1, left = rounds * tiles; left > 0; --left) {
        const int p0 = s.pos[i], n = s.count[i];
        if (fresh) {
            b_rank = s.rank[p0];
            mask_b();
        }
        [[maybe_unused]] const int r = b_rank;
        const Eight b0 = next0, b1 = next1;
        const int next_i = i + 1 < tiles ? i + 1 : 0, next_q = next_i ? q : q + kWarps;
        fresh = left > 1 && (next_i == 0 || s.slot[s.pos[next_i]] != s.slot[p0]);
        if (left > 1) load_base(next_i, next_q);
        if constexpr (kAheadB) {
            if (fresh) load_b(bn, next_i, next_q);
        }
        const int n0 = q * 32 + 8 * t;
        float acc[4][4];
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[j][0] = acc[j][1] = acc[j][2] = acc[j][3] = 0.0f;
        const int g0 = p0 + (g < n ? g : 0), g1 = p0 + (g + 8 < n ? g + 8 : 0);
        const uint8_t *t0 = tsm + g0 * kTP + t * 16, *t1 = tsm + g1 * kTP + t * 16;
        if constexpr (kWide) {
#pragma unroll
            for (int k = 0; k < NR / 4; ++k) {
                if (k * 32 < r) {
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const uint4 u = *reinterpret_cast<const uint4 *>(t0 + half * (NR * 16) + k * 64);
                        const uint4 v = *reinterpret_cast<const uint4 *>(t1 + half * (NR * 16) + k * 64);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            mma16816(acc[j], u.x, v.x, u.y, v.y, bw[k][j].x, bw[k][j].y);
                            mma16816(acc[j], u.z, v.z, u.w, v.w, bw[k][j].z, bw[k][j].w);
                        }
                    }
                }
            }
        } else {
            const uint4 u = *reinterpret_cast<const uint4 *>(t0), v = *reinterpret_cast<const uint4 *>(t1);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                mma16816(acc[j], u.x, v.x, u.y, v.y, bw[0][j].x, bw[0][j].y);
                mma16816(acc[j], u.z, v.z, u.w, v.w, bw[0][j].x, bw[0][j].y);
            }
        }
        const float o0[8] = {acc[0][0], acc[0][1], acc[1][0], acc[1][1], acc[2][0], acc[2][1], acc[3][0], acc[3][1]};
        const float o1[8] = {acc[0][2], acc[0][3], acc[1][2], acc[1][3], acc[2][2], acc[2][3], acc[3][2], acc[3][3]};
        if (n0 < a.N && g < n) add_store(Y + (size_t)(m0 + s.row[g0]) * a.ldy + n0, b0, o0, s.factor[g0]);
        if (n0 < a.N && g + 8 < n) add_store(Y + (size_t)(m0 + s.row[g1]) * a.ldy + n0, b1, o1, s.factor[g1]);
        if (fresh) {
            if constexpr (kAheadB) {
#pragma unroll
                for (int k = 0; k < (kWide ? NR / 4 : 1); ++k)
#pragma unroll
                    for (int j = 0; j < 4; ++j) bw[k][j] = bn[k][j];
            } else {
                load_b(bw, next_i, next_q);
            }
        }
        i = next_i;
        q = next_q;
    }
    // ---- rows without an adapter
    if (base != Y) {
        const int first = q0 * 4, last = min(q1 * 4, a.N >> 3);  // in eights of columns
        for (int p = active + warp; p < rows; p += kWarps) {
            const size_t r = m0 + s.row[p];
            for (int c = first + lane; c < last; c += 32)
                *reinterpret_cast<Eight *>(Y + r * a.ldy + c * 8) = base ? *reinterpret_cast<const Eight *>(base + r * a.ldbase + c * 8) : none;
        }
    }
    if constexpr (kBehind) asm volatile("griddepcontrol.wait;" ::: "memory");
}

static_assert(smem_bytes<2>(32, 8) <= kSmemMost && smem_bytes<4>(32, 8) <= kSmemMost && smem_bytes<8>(32, 8) <= kSmemMost && smem_bytes<16>(16, 8) <= kSmemMost &&
                  smem_bytes<16>(32, 4) <= kSmemMost && smem_bytes<16>(kWindow, 1) <= kSmemMost, "shared memory");

template <int NR, typename TO, bool kBehind>
cudaError_t launch_form(const AdapterArgs &a, int sms, cudaStream_t s) {
    static PerDevice<int> done;
    const int dev = current_device();
    if (dev < 0) return cudaErrorInvalidDevice;
    {
        std::lock_guard<std::mutex> lock(device_mutex());
        if (!done.have[dev]) {
            const cudaError_t e = cudaFuncSetAttribute(reinterpret_cast<const void *>(k_adapters<NR, TO, kBehind>),
                                                       cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemMost);
            if (e != cudaSuccess) return e;
            done.have[dev] = true;
        }
    }
    // Up to two CTAs for every SM: clusters of 8 as long as windows of up to 32 rows make few enough of them, then smaller ones.  An SM holds
    // two up to rank 64; above, it holds one (registers; from windows of 16 rows shared memory too), and more CTAs than SMs run one behind the other.
    // Behind k_adapter_tiles windows of 128 rows, of 64 or 32 where those would leave SMs idle.
    const auto windows = [&](int rows) { return ((long long)a.M + rows - 1) / rows; };
    const auto largest = [&](int rows) {  // cluster
        int l = 3;
        while (l && (windows(rows) << l > 2 * sms || smem_bytes<NR>(rows, 1 << l) > kSmemMost)) --l;
        return l;
    };
    int W = kBehind ? kWindow : 1;
    while (!kBehind && W < kMostRows && windows(W) * 8 > 2 * sms) W *= 2;
    while (kBehind && W > kMostRows && windows(W) << largest(W) < sms) W /= 2;
    const int log_c = largest(W);
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(windows(W) << log_c));
    cfg.blockDim = dim3(kT);
    cfg.dynamicSmemBytes = smem_bytes<NR>(W, 1 << log_c);
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 1 << log_c; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = log_c ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, k_adapters<NR, TO, kBehind>, a, W, log_c);
}

template <typename TO, bool kBehind>
cudaError_t launch_type(const AdapterArgs &a, int sms, cudaStream_t s) {
    if (a.max_rank <= 16) return launch_form<2, TO, kBehind>(a, sms, s);
    if (a.max_rank <= 32) return launch_form<4, TO, kBehind>(a, sms, s);
    if (a.max_rank <= 64) return launch_form<8, TO, kBehind>(a, sms, s);
    return launch_form<16, TO, kBehind>(a, sms, s);
}

}  // namespace

cudaError_t launch_adapters(const AdapterArgs &a, cudaStream_t s) {
    const int sms = num_sms();
    if (sms < 1) return cudaErrorInvalidDevice;
    cudaError_t e = cudaSuccess;
    const bool behind = launch_adapter_tiles(a, s, &e);
    if (e != cudaSuccess) return e;
    if (a.out_f32) return behind ? launch_type<float, true>(a, sms, s) : launch_type<float, false>(a, sms, s);
    return behind ? launch_type<__half, true>(a, sms, s) : launch_type<__half, false>(a, sms, s);
}

}  // namespace muxq
