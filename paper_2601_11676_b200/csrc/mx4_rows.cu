// halo_quantize_rows_mx4 / halo_dequantize_rows_mx4: rows in microscaled 4-bit floating point.
//
// 32 consecutive elements of a row share a power of two 2^e, e = floor(log2(amax)) - 2, kept as the byte e + 127
// (0 at least; 255 = the block holds a NaN or an infinity); an element is the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6
// times it, ties to the even code, larger ones become 6.  HBM-bound: one pass, every element read once.
//
// Codes: two a byte, the lower element in the low half, rows dense.  Scales: in blocks of 512 bytes for 128 rows x 128
// elements, byte (r % 32) * 16 + (r / 32) * 4 + j for row r of the 128 and block j of the 4, the order in which the
// tensor cores take them from tensor memory (halo_product_mx4 copies a block there as it is).
//
// Four lanes hold a block of 32 (8 elements each), so a warp reads 256 consecutive elements, writes 128 consecutive
// code bytes, and 16 lanes meet for one 4-byte word of scales.  A warp takes kRun such runs of one row at once: kRun
// independent loads per lane in flight.
#include <cuda_fp16.h>

#include "common.cuh"

namespace halo {
namespace {

constexpr int kThreads = 256;

// 8 elements as they lie in memory; widened only when they are used, so that several are in flight
template <typename T> struct Raw { uint4 w[sizeof(T) / 2]; };
template <typename T>
__device__ __forceinline__ Raw<T> fetch8(const T* p) {
    Raw<T> r;
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i) r.w[i] = ldg_stream16(reinterpret_cast<const uint4*>(p) + i);
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
// bits of the largest magnitude as fp32; a NaN counts as one
template <typename T>
__device__ __forceinline__ uint32_t top8(const Raw<T>& r) {
    if constexpr (sizeof(T) == 4) {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 2; ++i)
            top = max(top, max(max(r.w[i].x & 0x7fffffffu, r.w[i].y & 0x7fffffffu), max(r.w[i].z & 0x7fffffffu, r.w[i].w & 0x7fffffffu)));
        return top;
    } else {
        const uint32_t m = 0x7fff7fffu;
        const uint32_t two = __vmaxu2(__vmaxu2(r.w[0].x & m, r.w[0].y & m), __vmaxu2(r.w[0].z & m, r.w[0].w & m));
        return max(two << 16, two & 0xffff0000u);
    }
}
// two values -> two codes in a byte, the first in the low half (round to nearest even, 6 at most)
__device__ __forceinline__ uint32_t e2m1x2(float lo, float hi) {
    uint32_t r;
    asm("{\n\t.reg .b8 t;\n\tcvt.rn.satfinite.e2m1x2.f32 t, %1, %2;\n\tcvt.u32.u8 %0, t;\n\t}" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// 2^(code - 127); 255 is NaN
__device__ __forceinline__ float scale_of(uint32_t code) {
    return __uint_as_float(code == 0 ? 0x00400000u : code == 255u ? 0x7fc00000u : code << 23);
}

constexpr int kRun = 4;                 // runs of 256 elements a warp takes at once
constexpr int kWarps = kThreads / 32;

// Warp w of the grid: row w / segs, run group w % segs.  The rows behind n_rows up to a multiple of 128 get scales of
// zero.
template <typename T>
__global__ void __launch_bounds__(kThreads)
quantize_mx4_kernel(int d, unsigned n_rows, unsigned segs, unsigned items, const T* __restrict__ W, uint32_t* __restrict__ Q,
                    uint32_t* __restrict__ S) {
    const unsigned item = blockIdx.x * kWarps + (threadIdx.x >> 5);
    if (item >= items) return;
    const int lane = threadIdx.x & 31;
    const unsigned row = item / segs;
    const int c0 = static_cast<int>(item - row * segs) * (256 * kRun) + lane * 8;
    const long long at = static_cast<long long>(row) * d + c0;
    const bool real = row < n_rows;
    Raw<T> raw[kRun];
#pragma unroll
    for (int i = 0; i < kRun; ++i)
        if (real && c0 + i * 256 < d) raw[i] = fetch8(W + at + i * 256);
#pragma unroll
    for (int i = 0; i < kRun; ++i) {
        if (c0 + i * 256 >= d) break;   // d is a multiple of 128: the 16 lanes of a word of scales leave together
        uint32_t word = 0, scale = 0;
        const uint32_t group = 0xffffu << (lane & 16);
        if (real) {
            uint32_t top = top8(raw[i]);
            top = max(top, __shfl_xor_sync(group, top, 1));
            top = max(top, __shfl_xor_sync(group, top, 2));
            const uint32_t field = top >> 23;
            scale = field == 255u ? 255u : field < 2u ? 0u : field - 2u;
            const float inv = __uint_as_float((254u - min(scale, 252u)) << 23);   // 2^(127 - scale), exact
            float f[8];
            widen8(raw[i], f);
#pragma unroll
            for (int e = 0; e < 8; e += 2) word |= e2m1x2(f[e] * inv, f[e + 1] * inv) << (e * 4);
            if (scale == 255u) word = 0;
            Q[(at + i * 256) >> 3] = word;
        }
        uint32_t four = scale << (((lane >> 2) & 3) * 8);
        four |= __shfl_xor_sync(group, four, 4);
        four |= __shfl_xor_sync(group, four, 8);
        if ((lane & 15) == 0) {
            const long long block = static_cast<long long>(row >> 7) * (d >> 7) + ((c0 + i * 256) >> 7);
            S[block * 128 + (row & 31) * 4 + ((row >> 5) & 3)] = four;
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(kThreads)
dequantize_mx4_kernel(int d, unsigned segs, unsigned items, const uint32_t* __restrict__ Q, const uint8_t* __restrict__ S,
                      T* __restrict__ W) {
    const unsigned item = blockIdx.x * kWarps + (threadIdx.x >> 5);
    if (item >= items) return;
    const int lane = threadIdx.x & 31;
    const unsigned row = item / segs;
    const int c0 = static_cast<int>(item - row * segs) * (256 * kRun) + lane * 8;
    const long long at = static_cast<long long>(row) * d + c0;
    const uint8_t* srow = S + static_cast<long long>(row >> 7) * (d >> 7) * 512 + (row & 31) * 16 + ((row >> 5) & 3) * 4;
    uint32_t word[kRun], byte[kRun];
#pragma unroll
    for (int i = 0; i < kRun; ++i) {
        const int c = c0 + i * 256;
        word[i] = c < d ? __ldg(Q + ((at + i * 256) >> 3)) : 0u;
        byte[i] = c < d ? __ldg(srow + static_cast<long long>(c >> 7) * 512 + ((c >> 5) & 3)) : 0u;
    }
#pragma unroll
    for (int i = 0; i < kRun; ++i) {
        if (c0 + i * 256 >= d) break;
        const float scale = scale_of(byte[i]);
        float f[8];
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            uint32_t h;
            asm("{\n\t.reg .b8 t;\n\tcvt.u8.u32 t, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, t;\n\t}" : "=r"(h) : "r"((word[i] >> (e * 4)) & 0xffu));
            const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&h));
            f[e] = v.x * scale;
            f[e + 1] = v.y * scale;
        }
        T* out = W + at + i * 256;
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<float4*>(out) = make_float4(f[0], f[1], f[2], f[3]);
            *reinterpret_cast<float4*>(out + 4) = make_float4(f[4], f[5], f[6], f[7]);
        } else {
            __nv_bfloat162 v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = __floats2bfloat162_rn(f[2 * j], f[2 * j + 1]);   // exact: two significant bits
            *reinterpret_cast<uint4*>(out) =
                make_uint4(*reinterpret_cast<uint32_t*>(&v[0]), *reinterpret_cast<uint32_t*>(&v[1]),
                           *reinterpret_cast<uint32_t*>(&v[2]), *reinterpret_cast<uint32_t*>(&v[3]));
        }
    }
}

unsigned segments(int d) { return (d + 256 * kRun - 1) / (256 * kRun); }

halo_status check_rows(int d_model, long long n_rows, halo_dtype dtype) {
    if (dtype != HALO_F32 && dtype != HALO_BF16) return HALO_ERR_DTYPE;
    if (d_model <= 0 || d_model % 128 != 0 || d_model > HALO_MX4_MAX_WIDTH || n_rows <= 0 || n_rows > HALO_MX4_MAX_ROWS)
        return HALO_ERR_SHAPE;
    return HALO_OK;
}
}  // namespace
}  // namespace halo

using namespace halo;

extern "C" size_t halo_mx4_scale_bytes(int d_model, long long n_rows) {
    if (check_rows(d_model, n_rows, HALO_F32) != HALO_OK) return 0;
    return static_cast<size_t>((n_rows + 127) / 128) * (d_model / 128) * 512;
}

extern "C" halo_status halo_quantize_rows_mx4(int d_model, long long n_rows, halo_dtype wdtype, const void* W, void* Q,
                                              void* scales, void* stream) {
    const halo_status rc = check_rows(d_model, n_rows, wdtype);
    if (rc != HALO_OK) return rc;
    if (!W || !Q || !scales) return HALO_ERR_ARG;
    if (!aligned16(W) || !aligned16(Q) || !aligned16(scales)) return HALO_ERR_ALIGN;
    // warps: rows padded to 128 x runs, below 2^32 by the limits on both
    const unsigned segs = segments(d_model), items = static_cast<unsigned>((n_rows + 127) / 128 * 128 * segs);
    const unsigned grid = (items + kWarps - 1) / kWarps;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (wdtype == HALO_BF16)
        quantize_mx4_kernel<__nv_bfloat16><<<grid, kThreads, 0, st>>>(
            d_model, static_cast<unsigned>(n_rows), segs, items, static_cast<const __nv_bfloat16*>(W), static_cast<uint32_t*>(Q), static_cast<uint32_t*>(scales));
    else
        quantize_mx4_kernel<float><<<grid, kThreads, 0, st>>>(
            d_model, static_cast<unsigned>(n_rows), segs, items, static_cast<const float*>(W), static_cast<uint32_t*>(Q), static_cast<uint32_t*>(scales));
    HALO_CHECK_LAUNCH();
    return HALO_OK;
}

extern "C" halo_status halo_dequantize_rows_mx4(int d_model, long long n_rows, halo_dtype wdtype, const void* Q,
                                                const void* scales, void* W, void* stream) {
    const halo_status rc = check_rows(d_model, n_rows, wdtype);
    if (rc != HALO_OK) return rc;
    if (!W || !Q || !scales) return HALO_ERR_ARG;
    if (!aligned16(W) || !aligned16(Q) || !aligned16(scales)) return HALO_ERR_ALIGN;
    const unsigned segs = segments(d_model), items = static_cast<unsigned>(n_rows * segs);
    const unsigned grid = (items + kWarps - 1) / kWarps;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (wdtype == HALO_BF16)
        dequantize_mx4_kernel<__nv_bfloat16><<<grid, kThreads, 0, st>>>(
            d_model, segs, items, static_cast<const uint32_t*>(Q), static_cast<const uint8_t*>(scales), static_cast<__nv_bfloat16*>(W));
    else
        dequantize_mx4_kernel<float><<<grid, kThreads, 0, st>>>(
            d_model, segs, items, static_cast<const uint32_t*>(Q), static_cast<const uint8_t*>(scales), static_cast<float*>(W));
    HALO_CHECK_LAUNCH();
    return HALO_OK;
}
