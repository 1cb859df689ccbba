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
// Four lanes hold a block of 32 (8 elements each), so a warp reads 256 consecutive elements and writes 128 consecutive
// code bytes; one lane of four writes the block's scale byte.  A warp takes kRun such runs of one row at once: kRun
// independent loads per lane in flight.  11008 x 4096 bf16, there and back (228 MB): 36 us = 6.3 TB/s; 33 rows of 2048
// 5.6 us, the two launches.
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
        const __nv_bfloat162* v = reinterpret_cast<const __nv_bfloat162*>(&r.w[0]);
        const __nv_bfloat162 two = __hmax2_nan(__hmax2_nan(__habs2(v[0]), __habs2(v[1])), __hmax2_nan(__habs2(v[2]), __habs2(v[3])));
        const uint32_t w = *reinterpret_cast<const uint32_t*>(&two);
        return max(w << 16, w & 0xffff0000u);
    }
}
// eight values -> eight codes, the first in the lowest half byte (round to nearest even, 6 at most)
__device__ __forceinline__ uint32_t codes8(const float (&f)[8]) {
    uint32_t r;
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n\t"
        "mov.b32 %0, {b0, b1, b2, b3};\n\t}"
        : "=r"(r) : "f"(f[0]), "f"(f[1]), "f"(f[2]), "f"(f[3]), "f"(f[4]), "f"(f[5]), "f"(f[6]), "f"(f[7]));
    return r;
}
// eight codes -> eight values
__device__ __forceinline__ void values8(uint32_t word, float (&f)[8]) {
    uint32_t h[4];
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\tmov.b32 {b0, b1, b2, b3}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, b0;\n\tcvt.rn.f16x2.e2m1x2 %1, b1;\n\tcvt.rn.f16x2.e2m1x2 %2, b2;\n\tcvt.rn.f16x2.e2m1x2 %3, b3;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(word));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
        f[2 * i] = v.x;
        f[2 * i + 1] = v.y;
    }
}
// 2^(code - 127); 255 is NaN
__device__ __forceinline__ float scale_of(uint32_t code) {
    return __uint_as_float(code == 0 ? 0x00400000u : code == 255u ? 0x7fc00000u : code << 23);
}

constexpr int kRun = 4;                 // runs of 256 elements a warp takes at once
constexpr int kWarps = kThreads / 32;

// A warp takes 1024 elements: run group w % segs of row w / segs (WHOLE: d is a number of such groups; TAIL: the last one of
// a row is shorter), or, for many rows of fewer elements (FLAT), the w-th 1024 elements of all rows, every run of a lane
// finding its row (100000 x 128 bf16: 15.8 us with a warp per row, 7.6 so; 1000 x 128 1.1 and 1.8, 11008 x 2176 11.6 and
// 12.5).  The rows behind n_rows up to a multiple of 128 get scales of zero.
enum Form { WHOLE, TAIL, FLAT };
template <Form F>
struct Places {
    unsigned db, row, rem;   // blocks of 128 elements in a row; the warp's first one: its row, its number in it
    long long at;            // this lane's first element
    long long scale;         // and the offset of its scale (not FLAT)
    unsigned lane;
    __device__ __forceinline__ Places(int d, unsigned segs, unsigned item) {
        lane = threadIdx.x & 31;
        db = static_cast<unsigned>(d) >> 7;
        if constexpr (F == FLAT) {   // below 2^27 blocks by the limit on rows
            row = item * (2 * kRun) / db;
            rem = item * (2 * kRun) - row * db;
            at = static_cast<long long>(item) * (256 * kRun) + lane * 8;
        } else {
            row = item / segs;
            rem = (item - row * segs) * (2 * kRun);
            at = static_cast<long long>(row) * d + rem * 128 + lane * 8;
            scale = offset(row, rem + (lane >> 4));
        }
    }
    __device__ __forceinline__ long long offset(unsigned r, unsigned block) const {
        return (static_cast<long long>(r >> 7) * db + block) * 512 + (r & 31) * 16 + ((r >> 5) & 3) * 4 + ((lane >> 2) & 3);
    }
    __device__ __forceinline__ bool inside(int run) const { return F != TAIL || rem + run * 2 + (lane >> 4) < db; }
    // the row of a run's elements, and the offset of their scale
    __device__ __forceinline__ unsigned find(int run, long long& s) const {
        if constexpr (F == FLAT) {
            const unsigned k = rem + run * 2 + (lane >> 4), over = k / db;
            s = offset(row + over, k - over * db);
            return row + over;
        } else {
            s = scale + run * 1024;
            return row;
        }
    }
};

template <typename T, Form F>
__global__ void __launch_bounds__(kThreads)
quantize_mx4_kernel(int d, unsigned n_rows, unsigned segs, unsigned items, const T* __restrict__ W, uint32_t* __restrict__ Q,
                    uint8_t* __restrict__ S) {
    const unsigned item = blockIdx.x * kWarps + (threadIdx.x >> 5);
    chain_wait();
    if (item >= items) return;
    const int lane = threadIdx.x & 31;
    const Places<F> places(d, segs, item);
    const T* w = W + places.at;
    uint32_t* q = Q + (places.at >> 3);
    const bool writes = (lane & 3) == 0;   // four lanes hold a block
    const unsigned end = (n_rows + 127) / 128 * 128;
    Raw<T> raw[kRun];
    unsigned row[kRun];
    long long scale_at[kRun];
#pragma unroll
    for (int i = 0; i < kRun; ++i) {
        row[i] = places.find(i, scale_at[i]);
        if (row[i] < n_rows && places.inside(i)) raw[i] = fetch8(w + i * 256);
    }
#pragma unroll
    for (int i = 0; i < kRun; ++i) {
        if (!places.inside(i) || (F == FLAT && row[i] >= end)) break;   // d is a multiple of 128: the lanes of a block leave together
        uint32_t scale = 0;
        if (row[i] < n_rows) {
            const uint32_t group = 0xfu << (lane & 28);
            uint32_t top = top8(raw[i]);
            top = max(top, __shfl_xor_sync(group, top, 1));
            top = max(top, __shfl_xor_sync(group, top, 2));
            const uint32_t field = top >> 23;
            scale = max(field, 2u) - 2u;
            const float inv = __uint_as_float((254u - scale) << 23);   // 2^(127 - scale), exact: scale <= 252
            float f[8];
            widen8(raw[i], f);
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] *= inv;
            uint32_t word = codes8(f);
            if (field == 255u) { scale = 255u; word = 0; }             // a NaN or an infinity
            q[i * 32] = word;
        }
        if (writes) S[scale_at[i]] = static_cast<uint8_t>(scale);
    }
}

template <typename T, Form F>
__global__ void __launch_bounds__(kThreads)
dequantize_mx4_kernel(int d, unsigned n_rows, unsigned segs, unsigned items, const uint32_t* __restrict__ Q,
                      const uint8_t* __restrict__ S, T* __restrict__ W) {
    const unsigned item = blockIdx.x * kWarps + (threadIdx.x >> 5);
    chain_wait();
    if (item >= items) return;
    const Places<F> places(d, segs, item);
    const uint32_t* q = Q + (places.at >> 3);
    uint32_t word[kRun], byte[kRun];
    bool there[kRun];
#pragma unroll
    for (int i = 0; i < kRun; ++i) {
        long long scale_at;
        there[i] = places.find(i, scale_at) < n_rows && places.inside(i);
        if (there[i]) {
            word[i] = ldg_waited(q + i * 32);
            byte[i] = ldg_waited(S + scale_at);
        }
    }
#pragma unroll
    for (int i = 0; i < kRun; ++i) {
        if (!there[i]) break;
        const float scale = scale_of(byte[i]);
        float f[8];
        values8(word[i], f);
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] *= scale;
        T* out = W + places.at + i * 256;
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

// The form for rows of d elements, run groups per row (0: FLAT), and warps for so many rows: below 2^32 by the limits.
struct Split {
    Form form;
    unsigned segs, items;
    Split(int d, long long rows) {
        constexpr int kGroup = 256 * kRun;
        form = d < kGroup && rows >= 8192 ? FLAT : d % kGroup ? TAIL : WHOLE;
        segs = form == FLAT ? 0 : (d + kGroup - 1) / kGroup;
        items = static_cast<unsigned>(form == FLAT ? (rows * d + kGroup - 1) / kGroup : rows * segs);
    }
};

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
    const Split split(d_model, (n_rows + 127) / 128 * 128);
    const unsigned grid = (split.items + kWarps - 1) / kWarps;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const auto go = [&](auto kernel, auto* w) {
        return launch_chained(kernel, grid, kThreads, 0, st, d_model, static_cast<unsigned>(n_rows), split.segs, split.items, w,
                              static_cast<uint32_t*>(Q), static_cast<uint8_t*>(scales));
    };
    const auto form = [&](auto t) {
        using T = decltype(t);
        const T* w = static_cast<const T*>(W);
        return split.form == WHOLE  ? go(quantize_mx4_kernel<T, WHOLE>, w)
               : split.form == TAIL ? go(quantize_mx4_kernel<T, TAIL>, w)
                                    : go(quantize_mx4_kernel<T, FLAT>, w);
    };
    return wdtype == HALO_BF16 ? form(__nv_bfloat16()) : form(float());
}

extern "C" halo_status halo_dequantize_rows_mx4(int d_model, long long n_rows, halo_dtype wdtype, const void* Q,
                                                const void* scales, void* W, void* stream) {
    const halo_status rc = check_rows(d_model, n_rows, wdtype);
    if (rc != HALO_OK) return rc;
    if (!W || !Q || !scales) return HALO_ERR_ARG;
    if (!aligned16(W) || !aligned16(Q) || !aligned16(scales)) return HALO_ERR_ALIGN;
    const Split split(d_model, n_rows);
    const unsigned grid = (split.items + kWarps - 1) / kWarps;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const auto go = [&](auto kernel, auto* w) {
        return launch_chained(kernel, grid, kThreads, 0, st, d_model, static_cast<unsigned>(n_rows), split.segs, split.items, static_cast<const uint32_t*>(Q),
                              static_cast<const uint8_t*>(scales), w);
    };
    const auto form = [&](auto t) {
        using T = decltype(t);
        T* w = static_cast<T*>(W);
        return split.form == WHOLE  ? go(dequantize_mx4_kernel<T, WHOLE>, w)
               : split.form == TAIL ? go(dequantize_mx4_kernel<T, TAIL>, w)
                                    : go(dequantize_mx4_kernel<T, FLAT>, w);
    };
    return wdtype == HALO_BF16 ? form(__nv_bfloat16()) : form(float());
}
