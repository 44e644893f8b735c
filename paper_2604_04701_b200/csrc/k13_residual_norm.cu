// What stands between two projections of a transformer block, in one pass:
//   h = R + alpha * g (.) post(Y),   x = pre(h)
// with post and pre a layer norm, a root-mean-square norm or nothing; x is the fp16 input of the next muxq_linear.
//
// A token row is held in the registers of a group of threads from its load to its stores, so R and Y are read once and H and X
// written once.  The mean is taken first and the squares of the differences from it second, both from the registers: no
// cancellation of large sums.  All of it is fp32; H and X are rounded once each (x from h as it is before its own rounding: the
// fp16 form of the stream costs no accuracy of x).
#include "../../include/muxq.h"
#include "kernels.h"

namespace muxq {

namespace {

constexpr int kMaxThreads = 512;  // of a row
constexpr int kMostUnits = 10;    // of four channels, per thread
constexpr int kEarlyUnits = 3;    // up to here a thread fetches vectors and gate together with its row

struct RowSum {  // sums over the threads of a row; every call has a place of its own in shared memory, so one barrier is enough
    float *red;      // [4][16] of this row
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
__device__ __forceinline__ float4 floats(const uint2 &v) {
    const float2 a = __half22float2(*reinterpret_cast<const __half2 *>(&v.x)), b = __half22float2(*reinterpret_cast<const __half2 *>(&v.y));
    return make_float4(a.x, a.y, b.x, b.y);
}
__device__ __forceinline__ float4 floats(const uint4 &v) {
    return make_float4(__uint_as_float(v.x), __uint_as_float(v.y), __uint_as_float(v.z), __uint_as_float(v.w));
}
__device__ __forceinline__ void store4(__half *p, const float4 &v) {
    const __half2 a = __floats2half2_rn(v.x, v.y), b = __floats2half2_rn(v.z, v.w);
    *reinterpret_cast<uint2 *>(p) = make_uint2(*reinterpret_cast<const uint32_t *>(&a), *reinterpret_cast<const uint32_t *>(&b));
}
__device__ __forceinline__ void store4(float *p, const float4 &v) { *reinterpret_cast<float4 *>(p) = v; }

// v <- norm of the row v, without weight and bias.  Units beyond the row hold zeros and keep them.
template <int V>
__device__ __forceinline__ void normalize(float4 (&v)[V], const NormSpec &n, int D, int units, int T, int t, RowSum &sum) {
    const float inv_d = __fdiv_rn(1.0f, (float)D);
    if (n.kind == MUXQ_NORM_LAYER) {
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < V; ++i) s += (v[i].x + v[i].y) + (v[i].z + v[i].w);
        const float mu = sum(s) * inv_d;
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (t + i * T < units) { v[i].x -= mu; v[i].y -= mu; v[i].z -= mu; v[i].w -= mu; }
    }
    float q = 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i)
        q += __fmaf_rn(v[i].x, v[i].x, v[i].y * v[i].y) + __fmaf_rn(v[i].z, v[i].z, v[i].w * v[i].w);
    const float r = __fdiv_rn(1.0f, __fsqrt_rn(__fmaf_rn(sum(q), inv_d, n.eps)));
#pragma unroll
    for (int i = 0; i < V; ++i) { v[i].x *= r; v[i].y *= r; v[i].z *= r; v[i].w *= r; }
}

__device__ __forceinline__ void scale_shift(float4 &v, const float4 &w, const float4 &b) {
    v.x = __fmaf_rn(v.x, w.x, b.x); v.y = __fmaf_rn(v.y, w.y, b.y); v.z = __fmaf_rn(v.z, w.z, b.z); v.w = __fmaf_rn(v.w, w.w, b.w);
}

template <int V, typename TR, typename TY>
__global__ void __launch_bounds__(kMaxThreads) k_residual_norm(const ResidualNormArgs a, int T) {
    __shared__ float s_red[kMaxThreads / 32][4][16];
    const int sub = threadIdx.x / T, t = threadIdx.x - sub * T;
    const int rows = blockDim.x / T, units = a.D >> 2;
    const int m = blockIdx.x * rows + sub;
    const bool have = m < a.M;  // (rows behind the last one go along to the barriers)
    RowSum sum{&s_red[sub][0][0], T >> 5, t >> 5, t & 31, 0};
    const float4 zero = make_float4(0.f, 0.f, 0.f, 0.f), one = make_float4(1.f, 1.f, 1.f, 1.f);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // behind the wait: a layer kernel may read its W_q at once
    const TR *R = static_cast<const TR *>(a.R) + (size_t)m * a.ldr;
    const TY *Y = static_cast<const TY *>(a.Y) + (size_t)m * a.ldy;
    const size_t grow = a.gate_group ? (size_t)(m / a.gate_group) * a.ldg : 0;
    auto vec = [&](const float *p, int i, const float4 &none) {
        return p && t + i * T < units ? *reinterpret_cast<const float4 *>(p + 4 * (t + i * T)) : none;
    };
    auto gate = [&](int i) {
        if (!a.gate || t + i * T >= units || !have) return one;
        const size_t at = grow + 4 * (t + i * T);
        return a.gate_f32 ? floats(load4(static_cast<const float *>(a.gate) + at)) : floats(load4(static_cast<const __half *>(a.gate) + at));
    };
    typename RawOf<TR>::type r[V];
    typename RawOf<TY>::type yr[V];
    const typename RawOf<TR>::type rz{};
    const typename RawOf<TY>::type yz{};
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const bool in = have && t + i * T < units;
        r[i] = in && a.R ? load4(R + 4 * (t + i * T)) : rz;
        yr[i] = in && a.Y ? load4(Y + 4 * (t + i * T)) : yz;
    }
    constexpr bool kEarly = V <= kEarlyUnits;
    float4 wp[kEarly ? V : 1], bp[kEarly ? V : 1], gt[kEarly ? V : 1], wn[kEarly ? V : 1], bn[kEarly ? V : 1];
    if constexpr (kEarly) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            wp[i] = vec(a.post.weight, i, one); bp[i] = vec(a.post.bias, i, zero);
            gt[i] = gate(i);
            wn[i] = vec(a.pre.weight, i, one); bn[i] = vec(a.pre.bias, i, zero);
        }
    }
    float4 h[V];
    if (a.Y) {
        float4 y[V];
#pragma unroll
        for (int i = 0; i < V; ++i) y[i] = floats(yr[i]);
        if (a.post.kind != MUXQ_NORM_NONE) {
            normalize(y, a.post, a.D, units, T, t, sum);
#pragma unroll
            for (int i = 0; i < V; ++i)
                scale_shift(y[i], kEarly ? wp[kEarly ? i : 0] : vec(a.post.weight, i, one), kEarly ? bp[kEarly ? i : 0] : vec(a.post.bias, i, zero));
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float4 g = kEarly ? gt[kEarly ? i : 0] : gate(i), f = floats(r[i]);
            h[i].x = __fmaf_rn(a.alpha, y[i].x * g.x, f.x);
            h[i].y = __fmaf_rn(a.alpha, y[i].y * g.y, f.y);
            h[i].z = __fmaf_rn(a.alpha, y[i].z * g.z, f.z);
            h[i].w = __fmaf_rn(a.alpha, y[i].w * g.w, f.w);
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) h[i] = floats(r[i]);
    }
    if (a.H && have) {
        TR *H = static_cast<TR *>(a.H) + (size_t)m * a.ldh;
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (t + i * T < units) store4(H + 4 * (t + i * T), h[i]);
    }
    if (!a.X) return;
    if (a.pre.kind != MUXQ_NORM_NONE) {
        normalize(h, a.pre, a.D, units, T, t, sum);
#pragma unroll
        for (int i = 0; i < V; ++i)
            scale_shift(h[i], kEarly ? wn[kEarly ? i : 0] : vec(a.pre.weight, i, one), kEarly ? bn[kEarly ? i : 0] : vec(a.pre.bias, i, zero));
    }
    if (!have) return;
    __half *X = a.X + (size_t)m * a.ldx;
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (t + i * T < units) store4(X + 4 * (t + i * T), h[i]);
}

template <int V, typename TR, typename TY>
cudaError_t launch_form(const ResidualNormArgs &a, int T, int rows, cudaStream_t s) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(((long long)a.M + rows - 1) / rows));
    cfg.blockDim = dim3(T * rows);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, k_residual_norm<V, TR, TY>, a, T);
}

template <typename TR, typename TY>
cudaError_t launch_types(const ResidualNormArgs &a, int V, int T, int rows, cudaStream_t s) {
    switch (V) {
        case 1: return launch_form<1, TR, TY>(a, T, rows, s);
        case 2: return launch_form<2, TR, TY>(a, T, rows, s);
        case 3: return launch_form<3, TR, TY>(a, T, rows, s);
        case 4: return launch_form<4, TR, TY>(a, T, rows, s);
        case 5: case 6: return launch_form<6, TR, TY>(a, T, rows, s);
        case 7: case 8: return launch_form<8, TR, TY>(a, T, rows, s);
        default: return launch_form<kMostUnits, TR, TY>(a, T, rows, s);
    }
}

}  // namespace

cudaError_t launch_residual_norm(const ResidualNormArgs &a, cudaStream_t s) {
    const int units = a.D >> 2, sms = num_sms();
    if (sms < 1) return cudaErrorInvalidDevice;
    // few rows: as many threads as leave a unit or two to each; many: as few as can hold a row
    int T;
    if ((long long)a.M <= 4 * sms) T = ((units + 1) / 2 + 31) / 32 * 32;
    else T = ((units + kMostUnits - 1) / kMostUnits + 31) / 32 * 32;
    if (T > kMaxThreads) T = kMaxThreads;
    const int V = (units + T - 1) / T;
    int rows = (long long)a.M <= 4 * sms ? 1 : 256 / T;
    if (rows < 1) rows = 1;
    if (a.res_f32) return a.y_f32 ? launch_types<float, float>(a, V, T, rows, s) : launch_types<float, __half>(a, V, T, rows, s);
    return a.y_f32 ? launch_types<__half, float>(a, V, T, rows, s) : launch_types<__half, __half>(a, V, T, rows, s);
}

}  // namespace muxq
