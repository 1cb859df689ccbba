// halo_norm_glue: the residual between two blocks with a norm behind the one and a norm in front of the other,
//     h_out = h + res_scale * gate * rms_norm(y) * w_post,   x_out = cast(rms_norm(h_out) * w_pre).
// HBM-bound: h, y and the gate are read once, h_out and x_out written once; a row stays in registers between its two
// sums of squares.  A thread holds IT units of 8 elements, a row ceil(d / 8 / IT) threads; h, y and gate are all
// requested before the first sum, so that a row waits for memory once.  8191 rows of 5120 (587 MB) 91 us = 6.4 TB/s, one
// row of 4096 3.2 us, the launch.
#include <math.h>

#include "common.cuh"

namespace halo {
namespace {

struct GlueArgs {
    int d, n_tok;
    float eps, res_scale;
    long long gate_stride;
    const float* h;
    const void* y;
    const void* w_post;
    const void* gate;
    const void* w_pre;
    float* h_out;
    void* x_out;
};

template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&f)[8]) {
    if constexpr (sizeof(T) == 4) {
        const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
        f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
        f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
    } else {
        const uint4 w = *reinterpret_cast<const uint4*>(p);
        Elem<__nv_bfloat16>::widen(w, f);
    }
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&f)[8]) {
    if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
        *reinterpret_cast<float4*>(p + 4) = make_float4(f[4], f[5], f[6], f[7]);
    } else {
        __nv_bfloat162 v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
        *reinterpret_cast<uint4*>(p) =
            make_uint4(*reinterpret_cast<uint32_t*>(&v[0]), *reinterpret_cast<uint32_t*>(&v[1]),
                       *reinterpret_cast<uint32_t*>(&v[2]), *reinterpret_cast<uint32_t*>(&v[3]));
    }
}

// sum over the threads of a row (LANES of a warp, or, 0, the whole thread block); the same value in each of them
template <int LANES>
__device__ __forceinline__ float row_sum(float v, float* sh /*[32]*/) {
#pragma unroll
    for (int o = (LANES ? LANES : 32) / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if constexpr (LANES == 0) {
        const int lane = threadIdx.x & 31;
        if (lane == 0) sh[threadIdx.x >> 5] = v;
        __syncthreads();
        v = lane < static_cast<int>(blockDim.x >> 5) ? sh[lane] : 0.0f;
        v = warp_sum(v);
    }
    return v;
}

// 8 elements as they lie in memory
template <typename T> struct Raw { uint4 w[sizeof(T) / 2]; };
template <typename T>
__device__ __forceinline__ Raw<T> fetch8(const T* p) {
    Raw<T> r;
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i) r.w[i] = *(reinterpret_cast<const uint4*>(p) + i);
    return r;
}
template <typename T>
__device__ __forceinline__ void widen8(const Raw<T>& r, float (&f)[8]) {
    if constexpr (sizeof(T) == 4) {
        f[0] = __uint_as_float(r.w[0].x); f[1] = __uint_as_float(r.w[0].y);
        f[2] = __uint_as_float(r.w[0].z); f[3] = __uint_as_float(r.w[0].w);
        f[4] = __uint_as_float(r.w[1].x); f[5] = __uint_as_float(r.w[1].y);
        f[6] = __uint_as_float(r.w[1].z); f[7] = __uint_as_float(r.w[1].w);
    } else {
        Elem<__nv_bfloat16>::widen(r.w[0], f);
    }
}

constexpr int kRowThreads = 128;   // of a thread block where a row is a warp or less

template <typename TY, typename T, int IT, int LANES>
__global__ void __launch_bounds__(LANES ? kRowThreads : 1024)
norm_glue_kernel(const __grid_constant__ GlueArgs a) {
    __shared__ float sh[2][32];
    constexpr int kPart = LANES ? LANES : 32;
    const int t = LANES ? threadIdx.x % kPart : threadIdx.x, n = LANES ? LANES : blockDim.x;
    const long long mine = LANES ? static_cast<long long>(blockIdx.x) * (kRowThreads / kPart) + threadIdx.x / kPart : blockIdx.x;
    chain_wait();
    const long long row = LANES && mine >= a.n_tok ? a.n_tok - 1 : mine;   // behind the last row: its sums once more, no output
    const bool live = row == mine;
    const long long base = row * a.d;
    const int units = a.d / 8;
    float h[IT][8];
    Raw<TY> y[IT];
    Raw<T> g[IT];
#pragma unroll
    for (int i = 0; i < IT; ++i) {
        const int u = t + i * n;
        if (u < units) {
            load8(a.h + base + u * 8, h[i]);
            if (a.y) y[i] = fetch8(static_cast<const TY*>(a.y) + base + u * 8);
            if (a.gate) g[i] = fetch8(static_cast<const T*>(a.gate) + row * a.gate_stride + u * 8);
        }
    }
    if (a.y) {
        float f = a.res_scale;
        if (a.w_post) {
            float ss = 0.0f;
#pragma unroll
            for (int i = 0; i < IT; ++i) {
                if (t + i * n >= units) continue;
                float v[8];
                widen8(y[i], v);
#pragma unroll
                for (int e = 0; e < 8; ++e) ss = fmaf(v[e], v[e], ss);
            }
            ss = row_sum<LANES>(ss, sh[0]);
            f = rsqrtf(ss / static_cast<float>(a.d) + a.eps);
        }
#pragma unroll
        for (int i = 0; i < IT; ++i) {
            const int u = t + i * n;
            if (u >= units) continue;
            float v[8], w[8];
            widen8(y[i], v);
            if (a.w_post) {
                load8(static_cast<const T*>(a.w_post) + u * 8, w);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = v[e] * f * w[e] * a.res_scale;
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] *= f;
            }
            if (a.gate) {
                widen8(g[i], w);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] *= w[e];
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) h[i][e] += v[e];
        }
    }
    float ss = 0.0f;
#pragma unroll
    for (int i = 0; i < IT; ++i) {
        if (t + i * n >= units) continue;
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = fmaf(h[i][e], h[i][e], ss);
    }
    ss = row_sum<LANES>(ss, sh[1]);
    const float f = rsqrtf(ss / static_cast<float>(a.d) + a.eps);
#pragma unroll
    for (int i = 0; i < IT; ++i) {
        const int u = t + i * n;
        if (u >= units || !live) continue;
        store8(a.h_out + base + u * 8, h[i]);
        float w[8];
        if (a.w_pre) {
            load8(static_cast<const T*>(a.w_pre) + u * 8, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) h[i][e] = h[i][e] * f * w[e];
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) h[i][e] *= f;
        }
        store8(static_cast<T*>(a.x_out) + base + u * 8, h[i]);
    }
}

template <typename TY, typename T, int IT, int LANES>
halo_status go(const GlueArgs& a, int threads, cudaStream_t st) {
    constexpr int kPart = LANES ? LANES : 32;
    const int rows = LANES ? kRowThreads / kPart : 1;   // per thread block
    return launch_chained(norm_glue_kernel<TY, T, IT, LANES>, (a.n_tok - 1) / rows + 1, LANES ? kRowThreads : threads, 0, st, a);
}
template <typename TY, typename T>
halo_status launch(const GlueArgs& a, cudaStream_t st) {
    const int units = a.d / 8;
    const auto threads = [&](int it) { return (units + 32 * it - 1) / (32 * it) * 32; };
    // Many rows: two units per thread (8191 rows of 5120, us: two 91, three 93, four 102, five
    // 105: more units per thread leave fewer rows in flight per SM).  Few rows: one unit per thread while a thread block
    // can hold the row, the shortest time for a row.
    // Short rows: a part of a warp each (100000 rows of 64, us: 31 with a warp per row, 15; of 128: 34 and 29).
    const bool many = a.n_tok >= 2 * kSmCount;
    if (units <= 8) return go<TY, T, 1, 8>(a, 0, st);
    if (units <= 16) return go<TY, T, 1, 16>(a, 0, st);
    if (units <= 32) return go<TY, T, 1, 32>(a, 0, st);
    if (many && units <= 64) return go<TY, T, 2, 32>(a, 0, st);
    if (many || units > 1024) return go<TY, T, 2, 0>(a, threads(2), st);
    return go<TY, T, 1, 0>(a, threads(1), st);
}

}  // namespace
}  // namespace halo

using namespace halo;

extern "C" halo_status halo_norm_glue(const halo_norm_shape* shape, int n_tok, const float* h, const void* y,
                                      const void* w_post, const void* gate, long long gate_stride, float res_scale,
                                      const void* w_pre, float* h_out, void* x_out, void* stream) {
    if (!shape || !h || !h_out || !x_out) return HALO_ERR_ARG;
    if (!y && (w_post || gate)) return HALO_ERR_ARG;
    if ((shape->xdtype != HALO_F32 && shape->xdtype != HALO_BF16) || (shape->ydtype != HALO_F32 && shape->ydtype != HALO_BF16))
        return HALO_ERR_DTYPE;
    const int d = shape->d_model;
    if (d <= 0 || d % 8 != 0 || d > HALO_MAX_NORM_WIDTH || n_tok <= 0) return HALO_ERR_SHAPE;
    if (!(shape->eps > 0.0f) || !isfinite(shape->eps) || !isfinite(res_scale)) return HALO_ERR_ARG;
    if (gate && gate_stride != 0 && gate_stride < d) return HALO_ERR_SHAPE;
    if (!aligned16(h) || !aligned16(y) || !aligned16(w_post) || !aligned16(gate) || !aligned16(w_pre) || !aligned16(h_out) ||
        !aligned16(x_out) || (gate && gate_stride * (shape->xdtype == HALO_F32 ? 4 : 2) % 16 != 0))
        return HALO_ERR_ALIGN;
    GlueArgs a = {d, n_tok, shape->eps, res_scale, gate_stride, h, y, w_post, gate, w_pre, h_out, x_out};
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (shape->ydtype == HALO_F32)
        return shape->xdtype == HALO_F32 ? launch<float, float>(a, st) : launch<float, __nv_bfloat16>(a, st);
    return shape->xdtype == HALO_F32 ? launch<__nv_bfloat16, float>(a, st) : launch<__nv_bfloat16, __nv_bfloat16>(a, st);
}
