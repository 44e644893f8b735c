// What stands between two projections of a transformer block, in one pass:
//   h = R + alpha * g (.) post(Y),   x = pre(h)
// with post and pre a layer norm, a root-mean-square norm or nothing; x is the fp16 input of the next muxq_linear.
//
// A token row is held in the registers of a group of threads from its load to its stores, so R and Y are read once and H and X
// written once.  The mean is taken first and the squares of the differences from it second, both from the registers: no
// cancellation of large sums.  All of it is fp32; H and X are rounded once each (x from h as it is before its own rounding: the
// fp16 form of the stream costs no accuracy of x).
//
// Bound: HBM on long inputs (16384 x 1280, fp32 stream, fp16 Y and gate by rows: 48 us for 294 MB, 6.1 TB/s; 32768 x 768 in fp16 35 us, 5.7),
// where what counts is that an SM has enough rows under way and that few instructions are spent on each (packed arithmetic on pairs, no
// divisions, channels addressed from one counter: 87 -> 48 us); by the launch at decode steps (1.7 us in a row of calls).  Tried: CTAs that
// stay and copy rows ahead into shared memory asynchronously (80 to 140 us: too few warps for the arithmetic); a named barrier for each row
// of several warps (a kernel that names barriers by number is given all 16 of a CTA, so four CTAs fill an SM).
#include "../../include/muxq.h"
#include "kernels.h"

namespace muxq {

namespace {

constexpr int kMaxThreads = 512;  // of a row
constexpr int kMostUnits = 10;    // of four channels, per thread
constexpr int kGateUnits = 6;     // up to here it fetches a gate by rows together with its row
constexpr int kEarlyUnits = 3;    // up to here the vectors too

struct RowSum {  // sums over the threads of a row; every call has a place of its own in shared memory, so one barrier is enough
    float *red;      // [4][16]
    int warps, warp, lane, at;
    __device__ __forceinline__ float operator()(float v) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        if (warps == 1) return v;
        float *to = red + 16 * at++;
        if (lane == 0) to[warp] = v;
        __syncthreads();
        float s = 0.0f;
        for (int w = 0; w < warps; ++w) s += to[w];
        return s;
    }
};

template <typename T> struct RawOf;
template <> struct RawOf<__half> { using type = uint2; };
template <> struct RawOf<float> { using type = uint4; };

// (plain loads: the kernel may have started before the one that stores these values had ended)
template <typename T>
__device__ __forceinline__ typename RawOf<T>::type load4(const T *p) {
    return *reinterpret_cast<const typename RawOf<T>::type *>(p);
}
struct Four {  // four neighbouring channels as two pairs: the packed instructions on pairs halve what there is to issue
    float2 a, b;
};
__device__ __forceinline__ Four four(const uint2 &v) {
    return Four{__half22float2(*reinterpret_cast<const __half2 *>(&v.x)), __half22float2(*reinterpret_cast<const __half2 *>(&v.y))};
}
__device__ __forceinline__ Four four(const uint4 &v) {
    return Four{make_float2(__uint_as_float(v.x), __uint_as_float(v.y)), make_float2(__uint_as_float(v.z), __uint_as_float(v.w))};
}
__device__ __forceinline__ Four four(float x) { return Four{make_float2(x, x), make_float2(x, x)}; }
__device__ __forceinline__ Four load_vec(const float *p) { return four(load4(p)); }
__device__ __forceinline__ Four operator*(const Four &x, const Four &y) { return Four{__fmul2_rn(x.a, y.a), __fmul2_rn(x.b, y.b)}; }
__device__ __forceinline__ Four operator+(const Four &x, const Four &y) { return Four{__fadd2_rn(x.a, y.a), __fadd2_rn(x.b, y.b)}; }
__device__ __forceinline__ Four fma4(const Four &x, const Four &y, const Four &z) { return Four{__ffma2_rn(x.a, y.a, z.a), __ffma2_rn(x.b, y.b, z.b)}; }
__device__ __forceinline__ void store4(__half *p, const Four &v) {
    const __half2 a = __float22half2_rn(v.a), b = __float22half2_rn(v.b);
    *reinterpret_cast<uint2 *>(p) = make_uint2(*reinterpret_cast<const uint32_t *>(&a), *reinterpret_cast<const uint32_t *>(&b));
}
__device__ __forceinline__ void store4(float *p, const Four &v) { *reinterpret_cast<float4 *>(p) = make_float4(v.a.x, v.a.y, v.b.x, v.b.y); }

// The differences from the row's mean where the norm wants them, and the factor that norms them.  A unit beyond the row (only a thread's last
// can be one) holds zeros and keeps them.
template <int V>
__device__ __forceinline__ Four normalize(Four (&v)[V], const NormSpec &n, float inv_d, bool last_in, RowSum &sum) {
    if (n.kind == MUXQ_NORM_LAYER) {
        Four s = v[0];
#pragma unroll
        for (int i = 1; i < V; ++i) s = s + v[i];
        const Four minus = four(-(sum((s.a.x + s.a.y) + (s.b.x + s.b.y)) * inv_d));
#pragma unroll
        for (int i = 0; i < V - 1; ++i) v[i] = v[i] + minus;
        if (last_in) v[V - 1] = v[V - 1] + minus;
    }
    Four q = v[0] * v[0];
#pragma unroll
    for (int i = 1; i < V; ++i) q = fma4(v[i], v[i], q);
    // D squares of finite values may add up to more than fp32 holds.  The shares of the threads are therefore added 2^-8 times as large: up to 1e18 the
    // sum is then at most 16384 x 1e36 / 256, and a share (40 squares, of up to 2e18 where the mean is at one end) fits as it is.  Nothing is rounded
    // by it but shares below 2^-118, which moves the mean square by less than 2^-144.
    const float mean = __fmaf_rn(sum(((q.a.x + q.a.y) + (q.b.x + q.b.y)) * 0x1p-8f), inv_d * 0x1p8f, n.eps);
    return four(rsqrtf(mean));  // (off by 2 units at most)
}

// v <- v r weight + bias; the vectors come from memory where they have not been fetched ahead
template <int V>
__device__ __forceinline__ void scale_shift(Four (&v)[V], const Four &r, const float *weight, const float *bias, uint32_t c, uint32_t step, bool last_in) {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = v[i] * r;
    if (weight) {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < V - 1 || last_in) v[i] = v[i] * load_vec(weight + (c + i * step));
    }
    if (bias) {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < V - 1 || last_in) v[i] = v[i] + load_vec(bias + (c + i * step));
    }
}
template <int V>
__device__ __forceinline__ void scale_shift(Four (&v)[V], const Four &r, const Four (&weight)[V], const Four (&bias)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = fma4(v[i] * r, weight[i], bias[i]);
}
template <int V>
__device__ __forceinline__ void fetch(Four (&to)[V], const float *p, float none, uint32_t c, uint32_t step, bool last_in) {
#pragma unroll
    for (int i = 0; i < V; ++i) to[i] = p && (i < V - 1 || last_in) ? load_vec(p + (c + i * step)) : four(none);
}

template <int V, typename TR, typename TY>
__global__ void __maxnreg__(V > 6 ? 128 : sizeof(TR) == 4 ? 112 : 96) k_residual_norm(const ResidualNormArgs a) {
    __shared__ float s_red[4][16];
    const int t = threadIdx.x, T = blockDim.x;
    const int m = blockIdx.x * blockDim.y + threadIdx.y;
    if (m >= a.M) return;  // (a row of several warps has its CTA to itself)
    RowSum sum{&s_red[0][0], T >> 5, t >> 5, t & 31, 0};
    // this thread's channels: four from c on, then every `step` further; all but the last four are within the row
    const uint32_t c = 4 * t, step = 4 * T;
    const bool last_in = c + (V - 1) * step < (uint32_t)a.D;
    const size_t row = m;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // behind the wait: a layer kernel may read its W_q at once
    using RawR = typename RawOf<TR>::type;
    using RawY = typename RawOf<TY>::type;
    RawR r[V];
    RawY yr[V];
    if (a.R) {
        const TR *R = static_cast<const TR *>(a.R) + row * a.ldr;
#pragma unroll
        for (int i = 0; i < V; ++i) r[i] = i < V - 1 || last_in ? load4(R + (c + i * step)) : RawR{};
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) r[i] = RawR{};
    }
    if (a.Y) {
        const TY *Y = static_cast<const TY *>(a.Y) + row * a.ldy;
#pragma unroll
        for (int i = 0; i < V; ++i) yr[i] = i < V - 1 || last_in ? load4(Y + (c + i * step)) : RawY{};
    }
    // A gate by rows is as many bytes as Y, and on its way with the row, as it stands in memory.
    constexpr bool kGateAhead = V <= kGateUnits;
    const float *gate32 = static_cast<const float *>(a.gate);
    const __half *gate16 = static_cast<const __half *>(a.gate);
    if (a.gate && a.gate_group) {
        const size_t at = (size_t)(a.gate_group == 1 ? (uint32_t)row : (uint32_t)row / (uint32_t)a.gate_group) * a.ldg;
        gate32 += at;
        gate16 += at;
    }
    uint4 gr[kGateAhead ? V : 1];
    if (kGateAhead && a.gate) {
        if (a.gate_f32) {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (i < V - 1 || last_in) gr[kGateAhead ? i : 0] = load4(gate32 + (c + i * step));
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (i < V - 1 || last_in) {
                    const uint2 v = load4(gate16 + (c + i * step));
                    gr[kGateAhead ? i : 0].x = v.x;
                    gr[kGateAhead ? i : 0].y = v.y;
                }
        }
    }
    constexpr bool kEarly = V <= kEarlyUnits;
    Four wp[kEarly ? V : 1], bp[kEarly ? V : 1], wn[kEarly ? V : 1], bn[kEarly ? V : 1];
    if constexpr (kEarly) {
        fetch(wp, a.post.weight, 1.0f, c, step, last_in);
        fetch(bp, a.post.bias, 0.0f, c, step, last_in);
        fetch(wn, a.pre.weight, 1.0f, c, step, last_in);
        fetch(bn, a.pre.bias, 0.0f, c, step, last_in);
    }
    Four h[V];
    if (a.Y) {
#pragma unroll
        for (int i = 0; i < V; ++i) h[i] = four(yr[i]);
        if (a.post.kind != MUXQ_NORM_NONE) {
            const Four by = normalize(h, a.post, a.inv_d, last_in, sum);
            if constexpr (kEarly) scale_shift(h, by, wp, bp);
            else scale_shift(h, by, a.post.weight, a.post.bias, c, step, last_in);
        }
        if (a.gate) {
            if (a.gate_f32) {
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (i < V - 1 || last_in) h[i] = h[i] * (kGateAhead ? four(gr[kGateAhead ? i : 0]) : four(load4(gate32 + (c + i * step))));
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (i < V - 1 || last_in)
                        h[i] = h[i] * (kGateAhead ? four(make_uint2(gr[kGateAhead ? i : 0].x, gr[kGateAhead ? i : 0].y)) : four(load4(gate16 + (c + i * step))));
            }
        }
        const Four alpha = four(a.alpha);
#pragma unroll
        for (int i = 0; i < V; ++i) h[i] = fma4(alpha, h[i], four(r[i]));
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) h[i] = four(r[i]);
    }
    if (a.H) {
        TR *H = static_cast<TR *>(a.H) + row * a.ldh;
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < V - 1 || last_in) store4(H + (c + i * step), h[i]);
    }
    if (!a.X) return;
    if (a.pre.kind != MUXQ_NORM_NONE) {
        const Four by = normalize(h, a.pre, a.inv_d, last_in, sum);
        if constexpr (kEarly) scale_shift(h, by, wn, bn);
        else scale_shift(h, by, a.pre.weight, a.pre.bias, c, step, last_in);
    }
    __half *X = a.X + row * a.ldx;
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (i < V - 1 || last_in) store4(X + (c + i * step), h[i]);
}

template <int V, typename TR, typename TY>
cudaError_t launch_form(const ResidualNormArgs &a, int T, int rows, cudaStream_t s) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(((long long)a.M + rows - 1) / rows));
    cfg.blockDim = dim3(T, rows);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, k_residual_norm<V, TR, TY>, a);
}

template <typename TR, typename TY>
cudaError_t launch_types(const ResidualNormArgs &a, int V, int T, int rows, cudaStream_t s) {
    switch (V) {
        case 1: return launch_form<1, TR, TY>(a, T, rows, s);
        case 2: return launch_form<2, TR, TY>(a, T, rows, s);
        case 3: return launch_form<3, TR, TY>(a, T, rows, s);
        case 4: return launch_form<4, TR, TY>(a, T, rows, s);
        case 5: return launch_form<5, TR, TY>(a, T, rows, s);
        case 6: return launch_form<6, TR, TY>(a, T, rows, s);
        case 7: return launch_form<7, TR, TY>(a, T, rows, s);
        case 8: return launch_form<8, TR, TY>(a, T, rows, s);
        case 9: return launch_form<9, TR, TY>(a, T, rows, s);
        default: return launch_form<kMostUnits, TR, TY>(a, T, rows, s);
    }
}

}  // namespace

cudaError_t launch_residual_norm(const ResidualNormArgs &a, cudaStream_t s) {
    const int units = a.D >> 2, sms = num_sms();
    if (sms < 1) return cudaErrorInvalidDevice;
    // Few rows: as many threads as leave a unit or two to each.  Many: as few as can hold a row in their registers, one warp as long as it can;
    // an SM then holds enough rows that one's loads go on under another's sums (us, one warp / two / four: 8192 x 768 11.6 / 15.6 / 24.1,
    // 16384 x 1280 with a gate by rows 47.9 / 51.2 / 66.7; two / four: 2000 x 2560 12.7 / 12.8; 300 x 1280 3.2 / 3.2 / 2.9).
    const bool few = (long long)a.M <= 4 * sms;
    int T = few ? ((units + 1) / 2 + 31) / 32 * 32 : 32;
    while (!few && T * kMostUnits < units) T *= 2;
    if (T > kMaxThreads) T = kMaxThreads;
    const int V = (units + T - 1) / T;
    const int rows = T == 32 ? 2 : 1;
    if (a.res_f32) return a.y_f32 ? launch_types<float, float>(a, V, T, rows, s) : launch_types<float, __half>(a, V, T, rows, s);
    return a.y_f32 ? launch_types<__half, float>(a, V, T, rows, s) : launch_types<__half, __half>(a, V, T, rows, s);
}

}  // namespace muxq
