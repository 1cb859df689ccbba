// halo_paged_norm_append: the keys and values of new tokens go to their pages in the caches' type or as 8-bit rows, queries
// and keys normed per head and turned by their position on the way; halo_paged_kv_read: rows back out of the pages.
// Every element is read once and written once.  8297 tokens, 32 + 2 * 8 heads of 128, into 8-bit rows: 47 us where HBM would
// take 28 (187 MB; the instructions bound it), read back in 9 to 11 (52 MB: 8).  Into bf16 rows 44 (204 MB: 31), fp32 69 (408 MB: 62).
//
//   y = x / sqrt(mean(x^2) + eps) * w over a head's elements (queries and keys that have a gain), then pair i of the first
//   rotary elements by the angle pos * inv_freq[i], times turn_scale.  Angles are reduced to one turn in fp64 as in
//   halo_paged_kv_append; their cosines and sines, once per token and through shared memory, come in fp64 too and are rounded once:
//   keys of 8 bits fall on another code than in exact arithmetic more rarely (8297 tokens: 0.000078 off, with fp32 0.000097), and it costs
//   0.2 us of 46.  Everything else between the load and the one rounding of the store is fp32.
//
// A lane has two 16-byte words' worth of elements (eight of each) of a head: those of its pairs (i, i + rotary / 2), or two
// neighbours; it walks over the heads of q, k and v alike, so cosines and sines stay in registers, and no element of a pair has to
// be fetched from another lane.  LANES lanes hold a head, a power of two, and sum its squares and find its largest element by
// shuffles.  One head of a lane is in flight at a time: three took more registers, and 8297 tokens into 8-bit rows 64 us and not 59.
// An element costs about ten instructions; with one word to a lane (and its partners' from another) it was twice that,
// and the instructions were what bounded it.  Pairs whose distance is no whole number of eight elements go by that form
// (paged_norm_append_any_kernel): through a row of shared memory that only the warp's own lanes touch.  8297 tokens of 32 + 2 * 8 heads of 80, of
// which 40 are turned: 107 us into 8-bit rows, 87 into bf16.
#include <math.h>

#include "eight.cuh"

namespace halo {
halo_status check_paged_shape(const halo_paged_shape* s);
halo_status check_eight(const halo_paged_shape& s, const void* K_scale, const void* V_scale);
long long paged_stride(const halo_paged_shape& s);

namespace {

constexpr int kThreads = 64;     // each warp sees to its token's page and angles: with 128, 8297 tokens 59 us and not 50, 32 tokens 4.0 and not 3.6
constexpr int kOwn = 8;      // elements per lane

struct NormAppendArgs {
    int H, Hk, dh, page_size, n_pages, max_pages, n_seq, rotary;
    long long page_stride, q_stride, k_stride, v_stride, qo_stride;
    float eps, turn_scale;
    const void* q;
    const void* k;
    const void* v;
    const void* w_q;
    const void* w_k;
    const int32_t* pos;
    const int32_t* seq;
    const int32_t* table;
    const double* inv_freq;
    void* q_out;
    void* K;
    void* V;
    uint8_t* K_scale;
    uint8_t* V_scale;
    uint32_t* status;
};

template <typename T>
struct Own {      // eight elements as they lie in memory
    uint4 w[sizeof(T) / 2];
    __device__ __forceinline__ void load(const T* p) {
#pragma unroll
        for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i) w[i] = reinterpret_cast<const uint4*>(p)[i];
    }
    __device__ __forceinline__ void store(T* p) const {
#pragma unroll
        for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i) reinterpret_cast<uint4*>(p)[i] = w[i];
    }
    __device__ __forceinline__ void widen(float (&x)[kOwn]) const {
        const T* e = reinterpret_cast<const T*>(w);
#pragma unroll
        for (int i = 0; i < kOwn; ++i) x[i] = to_float(e[i]);
    }
    __device__ __forceinline__ void narrow(const float (&x)[kOwn]) {
        T* e = reinterpret_cast<T*>(w);
#pragma unroll
        for (int i = 0; i < kOwn; ++i) e[i] = from_float<T>(x[i]);
    }
};

template <int LANES>
__device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
template <int LANES>
__device__ __forceinline__ uint32_t lanes_max(uint32_t v) {
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) v = max(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}

// 1 / sqrt(mean(x^2) + eps) of rows of dh elements, N of which a lane has; by whole warps.  Rows whose squares pass the largest number become
// 2^-70 of themselves where they are normed (eps is nothing beside them), and so does their factor's reference.
template <int LANES, int N>
__device__ __forceinline__ float norm_factor(float (&f)[N], bool normed, int dh, float eps) {
    float sum = 0.0f;
#pragma unroll
    for (int e = 0; e < N; ++e) sum = fmaf(f[e], f[e], sum);
    sum = lanes_sum<LANES>(sum);
    const bool past = !(sum < INFINITY);
    if (__any_sync(0xffffffffu, past)) {
        float less = 0.0f;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float x = f[e] * 0x1p-70f;
            less = fmaf(x, x, less);
            if (past && normed) f[e] = x;
        }
        less = lanes_sum<LANES>(less);
        if (past) {
            sum = less;
            eps = 0.0f;
        }
    }
    return rsqrtf(sum / static_cast<float>(dh) + eps);
}

// Thread block (token, part): heads part * groups + group, ... in steps of groups * parts.
template <typename T, int LANES, bool EIGHT>
__global__ void __launch_bounds__(kThreads)
paged_norm_append_any_kernel(const __grid_constant__ NormAppendArgs a, int parts) {
    constexpr int kGroups = kThreads / LANES;
    constexpr int kRow = LANES * kOwn + 4;     // floats; rows of neighbouring groups start in other banks
    __shared__ float2 turn[128];               // [rotary / 2] cosine, sine
    __shared__ __align__(16) float rows[kGroups][kRow];
    const int tid = threadIdx.x, group = tid / LANES, c = tid % LANES, el = c * kOwn;
    const int tok = blockIdx.x / parts, part = blockIdx.x % parts;
    chain_wait();
    // everything that depends on the token alone is requested at once
    const int pos = ldg_waited(a.pos + tok);
    const int s = a.seq ? ldg_waited(a.seq + tok) : tok;
    const int half = a.rotary / 2, heads = a.H + 2 * a.Hk, step = kGroups * parts;
    const bool in = el < a.dh;                 // lanes behind the head's end hold zeros
    const T* q = static_cast<const T*>(a.q) + static_cast<long long>(tok) * a.q_stride + el;
    const T* k = static_cast<const T*>(a.k) + static_cast<long long>(tok) * a.k_stride + el;
    const T* v = static_cast<const T*>(a.v) + static_cast<long long>(tok) * a.v_stride + el;
    Own<T> x;
    const auto fetch = [&](int h) {
        if (in && h < heads) x.load(h < a.H ? q + h * a.dh : h < a.H + a.Hk ? k + (h - a.H) * a.dh : v + (h - a.H - a.Hk) * a.dh);
    };
    const int first = part * kGroups + group;
    double freq = tid < half ? ldg_waited(a.inv_freq + tid) : 0.0;
    fetch(first);
    float wq[kOwn], wk[kOwn];
    const auto gain = [&](const void* w, float (&out)[kOwn]) {
        Own<T> g;
        if (w && in) {
            g.load(static_cast<const T*>(w) + el);
            g.widen(out);
        }
    };
    gain(a.w_q, wq);
    gain(a.w_k, wk);

    if (pos < 0) return;               // a padding row: nothing is written for it
    const int pi = pos / a.page_size;
    int page = -1;
    if (s >= 0 && s < a.n_seq && pi < a.max_pages) page = ldg_waited(a.table + static_cast<long long>(s) * a.max_pages + pi);
    for (int i = tid; i < half; i += kThreads) {
        if (i != tid) freq = ldg_waited(a.inv_freq + i);
        const double turns = static_cast<double>(pos) * freq * 0.15915494309189533577;
        double co, si;
        sincospi(2.0 * (turns - rint(turns)), &si, &co);
        turn[i] = make_float2(static_cast<float>(co * a.turn_scale), static_cast<float>(si * a.turn_scale));
    }
    if (page < 0 || page >= a.n_pages) {   // the same in every thread
        if (tid == 0 && part == 0) flag_status(a.status, HALO_DEV_BAD_INDEX);
        return;
    }
    __syncthreads();
    // out = own * co + other * si, the sign of the pair's first element in si
    float co[kOwn], si[kOwn];
#pragma unroll
    for (int e = 0; e < kOwn; ++e) {
        const int at = el + e;
        co[e] = 1.0f;
        si[e] = 0.0f;
        if (at < a.rotary) {
            const bool second = at >= half;
            const float2 t = turn[second ? at - half : at];
            co[e] = t.x;
            si[e] = second ? t.y : -t.y;
        }
    }
    const bool turned = el < a.rotary;                 // elements behind the last pair are left as they are (infinity * 0 would not be)
    const long long row = static_cast<long long>(page) * a.Hk * a.page_size + pos % a.page_size;   // of the scales
    const long long base = static_cast<long long>(page) * a.page_stride + static_cast<long long>(pos % a.page_size) * a.dh + el;
    const long long plane = static_cast<long long>(a.page_size) * a.dh;
    T* qo = static_cast<T*>(a.q_out) + static_cast<long long>(tok) * a.qo_stride + el;
    float* mine = rows[group];

    // every lane of a warp takes every step: lanes meet in the shuffles
    for (int h = first, b0 = part * kGroups; b0 < heads; h += step, b0 += step) {      // b0: the same in every lane of the block
        if (h != first) fetch(h);
        const bool there = in && h < heads, is_q = h < a.H, is_v = h >= a.H + a.Hk;
        float f[kOwn];
#pragma unroll
        for (int e = 0; e < kOwn; ++e) f[e] = 0.0f;
        if (there) x.widen(f);
        const bool normed = !is_v && (is_q ? a.w_q : a.w_k) != nullptr;
        if (a.w_q || a.w_k) {
            const float n = norm_factor<LANES>(f, normed, a.dh, a.eps);
            if (there && normed) {
#pragma unroll
                for (int e = 0; e < kOwn; ++e) f[e] = f[e] * n * (is_q ? wq[e] : wk[e]);
            }
        }
        {
            __syncwarp();
            *reinterpret_cast<float4*>(mine + el) = make_float4(f[0], f[1], f[2], f[3]);
            *reinterpret_cast<float4*>(mine + el + 4) = make_float4(f[4], f[5], f[6], f[7]);
            __syncwarp();
            if (turned && !is_v) {
                float o[kOwn];
#pragma unroll
                for (int e = 0; e < kOwn; ++e) {
                    const int at = el + e;
                    o[e] = at < a.rotary ? mine[at < half ? at + half : at - half] : 0.0f;
                }
#pragma unroll
                for (int e = 0; e < kOwn; ++e)
                    if (el + e < a.rotary) f[e] = f[e] * co[e] + o[e] * si[e];
            }
        }
        if (EIGHT && b0 + kGroups > a.H) {      // a head of this pass is a key or a value
            uint32_t top = 0;                               // sizes of finite numbers, ordered as their bits are
#pragma unroll
            for (int e = 0; e < kOwn; ++e) top = max(top, __float_as_uint(f[e]) & 0x7fffffffu);
            top = lanes_max<LANES>(top);
            if (there && !is_q) {
                const bool sound = top < 0x7f800000u;
                const int ex = eight_exponent(__uint_as_float(top));
                const float n = eight_power(-ex);
                uint32_t w[2];
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    w[j] = sound ? eight_pair(f[4 * j] * n, f[4 * j + 1] * n) | eight_pair(f[4 * j + 2] * n, f[4 * j + 3] * n) << 16 : 0u;
                const int kv = is_v ? h - a.H - a.Hk : h - a.H;
                *reinterpret_cast<uint2*>(static_cast<uint8_t*>(is_v ? a.V : a.K) + base + kv * plane) = make_uint2(w[0], w[1]);
                if (c == 0)
                    (is_v ? a.V_scale : a.K_scale)[row + static_cast<long long>(kv) * a.page_size] =
                        static_cast<uint8_t>(sound ? ex + 127 : kEightNan);
            }
        }
        if (there && (is_q || !EIGHT)) {
            x.narrow(f);
            x.store(is_q ? qo + h * a.dh
                       : is_v ? static_cast<T*>(a.V) + base + (h - a.H - a.Hk) * plane
                              : static_cast<T*>(a.K) + base + (h - a.H) * plane);
        }
    }
}

// Thread block (token, part): heads part * groups + group, ... in steps of groups * parts.  Units of 16 elements, LANES a head.
template <typename T, int LANES, bool EIGHT, bool INTERLEAVED>
__global__ void __launch_bounds__(kThreads)
paged_norm_append_kernel(const __grid_constant__ NormAppendArgs a, int parts) {
    constexpr int kGroups = kThreads / LANES;
    __shared__ float2 turn[128];                         // [rotary / 2] cosine, sine
    __shared__ __align__(16) float gain[2][LANES * 16];  // of queries, of keys; 1 where there is no norm
    const int tid = threadIdx.x, group = tid / LANES, u = tid % LANES;
    const int tok = blockIdx.x / parts, part = blockIdx.x % parts;
    chain_wait();
    // everything that depends on the token alone is requested at once
    const int pos = ldg_waited(a.pos + tok);
    const int s = a.seq ? ldg_waited(a.seq + tok) : tok;
    const int half = a.rotary / 2, heads = a.H + 2 * a.Hk, step = kGroups * parts;
    const bool in = u * 16 < a.dh;                       // lanes behind the head's end hold zeros
    // the unit's two words: eight pairs' first and second elements, or sixteen neighbours
    const int hu = half / 8;
    const bool across = !INTERLEAVED && u < hu;
    const int el0 = across || INTERLEAVED ? u * (INTERLEAVED ? 16 : 8) : a.rotary + (u - hu) * 16, el1 = across ? el0 + half : el0 + 8;
    const T* q = static_cast<const T*>(a.q) + static_cast<long long>(tok) * a.q_stride;
    const T* k = static_cast<const T*>(a.k) + static_cast<long long>(tok) * a.k_stride - a.H * a.dh;
    const T* v = static_cast<const T*>(a.v) + static_cast<long long>(tok) * a.v_stride - (a.H + a.Hk) * a.dh;
    Own<T> x[2];
    const auto fetch = [&](int h) {
        if (in && h < heads) {
            const T* src = (h < a.H ? q : h < a.H + a.Hk ? k : v) + h * a.dh;
            x[0].load(src + el0);
            x[1].load(src + el1);
        }
    };
    const int first = part * kGroups + group;
    double freq = tid < half ? ldg_waited(a.inv_freq + tid) : 0.0;
    fetch(first);
    for (int i = tid; i < 2 * a.dh; i += kThreads) {
        const bool key = i >= a.dh;
        const T* w = static_cast<const T*>(key ? a.w_k : a.w_q);
        gain[key][key ? i - a.dh : i] = w ? to_float(w[key ? i - a.dh : i]) : 1.0f;
    }

    if (pos < 0) return;               // a padding row: nothing is written for it
    const int pi = pos / a.page_size, in_page = pos - pi * a.page_size;
    int page = -1;
    if (s >= 0 && s < a.n_seq && pi < a.max_pages) page = ldg_waited(a.table + static_cast<long long>(s) * a.max_pages + pi);
    for (int i = tid; i < half; i += kThreads) {
        if (i != tid) freq = ldg_waited(a.inv_freq + i);
        const double turns = static_cast<double>(pos) * freq * 0.15915494309189533577;
        double co, si;
        sincospi(2.0 * (turns - rint(turns)), &si, &co);
        turn[i] = make_float2(static_cast<float>(co * a.turn_scale), static_cast<float>(si * a.turn_scale));
    }
    if (page < 0 || page >= a.n_pages) {   // the same in every thread
        if (tid == 0 && part == 0) flag_status(a.status, HALO_DEV_BAD_INDEX);
        return;
    }
    __syncthreads();
    float co[kOwn], si[kOwn];          // of pairs 8 u to 8 u + 7; those that are not turned are left as they are (infinity * 0 would not be)
#pragma unroll
    for (int e = 0; e < kOwn; ++e) {
        const float2 t = u * 8 + e < half ? turn[u * 8 + e] : make_float2(1.0f, 0.0f);
        co[e] = t.x;
        si[e] = t.y;
    }
    const long long row = static_cast<long long>(page) * a.Hk * a.page_size + in_page;   // of the scales
    const long long base = static_cast<long long>(page) * a.page_stride + static_cast<long long>(in_page) * a.dh;
    const long long plane = static_cast<long long>(a.page_size) * a.dh;
    T* qo = static_cast<T*>(a.q_out) + static_cast<long long>(tok) * a.qo_stride;

    // every lane of a warp takes every step: lanes meet in the shuffles
    for (int h = first, b0 = part * kGroups; b0 < heads; h += step, b0 += step) {      // b0: the same in every lane of the block
        if (h != first) fetch(h);
        const bool there = in && h < heads, is_q = h < a.H, is_v = h >= a.H + a.Hk;
        float f[2][kOwn];
        if (there) {
            x[0].widen(f[0]);
            x[1].widen(f[1]);
        } else {
#pragma unroll
            for (int e = 0; e < kOwn; ++e) f[0][e] = f[1][e] = 0.0f;
        }
        if (__any_sync(0xffffffffu, there && !is_v)) {       // queries or keys among the warp's heads
            const bool normed = !is_v && (is_q ? a.w_q : a.w_k) != nullptr;
            float n = 1.0f;
            if (a.w_q || a.w_k) n = norm_factor<LANES>(reinterpret_cast<float(&)[2 * kOwn]>(f), normed, a.dh, a.eps);
            if (!is_v && there) {
                if (normed) {      // first of all: a gain or a turn could carry the elements themselves out of range
                    const float* g = gain[is_q ? 0 : 1];
#pragma unroll
                    for (int w = 0; w < 2; ++w)
#pragma unroll
                        for (int e = 0; e < kOwn; e += 4) {
                            const float4 by = *reinterpret_cast<const float4*>(g + (w ? el1 : el0) + e);
                            f[w][e] = f[w][e] * n * by.x;
                            f[w][e + 1] = f[w][e + 1] * n * by.y;
                            f[w][e + 2] = f[w][e + 2] * n * by.z;
                            f[w][e + 3] = f[w][e + 3] * n * by.w;
                        }
                }
#pragma unroll
                for (int e = 0; e < kOwn; ++e) {
                    // pair e: its elements lie in the two words, or side by side
                    float& one = INTERLEAVED ? f[e >> 2][(e & 3) * 2] : f[0][e];
                    float& two = INTERLEAVED ? f[e >> 2][(e & 3) * 2 + 1] : f[1][e];
                    if (INTERLEAVED ? u * 8 + e < half : across) {
                        const float p = one, o = two;
                        one = p * co[e] - o * si[e];
                        two = p * si[e] + o * co[e];
                    }
                }
            }
        }
        if (EIGHT && __any_sync(0xffffffffu, there && !is_q)) {
            uint32_t top = 0;                               // sizes of finite numbers, ordered as their bits are
#pragma unroll
            for (int e = 0; e < kOwn; ++e)
                top = max(top, max(__float_as_uint(f[0][e]) & 0x7fffffffu, __float_as_uint(f[1][e]) & 0x7fffffffu));
            top = lanes_max<LANES>(top);
            if (there && !is_q) {
                const bool sound = top < 0x7f800000u;
                const int ex = eight_exponent(__uint_as_float(top));
                const float by = eight_power(-ex);
                const int kv = is_v ? h - a.H - a.Hk : h - a.H;
                uint8_t* to = static_cast<uint8_t*>(is_v ? a.V : a.K) + base + kv * plane;
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    uint32_t c[2];
#pragma unroll
                    for (int j = 0; j < 2; ++j)
                        c[j] = sound ? eight_pair(f[w][4 * j] * by, f[w][4 * j + 1] * by) | eight_pair(f[w][4 * j + 2] * by, f[w][4 * j + 3] * by) << 16 : 0u;
                    *reinterpret_cast<uint2*>(to + (w ? el1 : el0)) = make_uint2(c[0], c[1]);
                }
                if (u == 0)
                    (is_v ? a.V_scale : a.K_scale)[row + static_cast<long long>(kv) * a.page_size] =
                        static_cast<uint8_t>(sound ? ex + 127 : kEightNan);
            }
        }
        if (there && (is_q || !EIGHT)) {
            T* to = is_q ? qo + h * a.dh : is_v ? static_cast<T*>(a.V) + base + (h - a.H - a.Hk) * plane : static_cast<T*>(a.K) + base + (h - a.H) * plane;
            if (!is_v) {
                x[0].narrow(f[0]);
                x[1].narrow(f[1]);
            }
            x[0].store(to + el0);
            x[1].store(to + el1);
        }
    }
}

template <int LANES, typename K>
halo_status launch(K kernel, const NormAppendArgs& a, int n_tok, cudaStream_t st) {
    const int groups = kThreads / LANES, heads = a.H + 2 * a.Hk, most = (heads + groups - 1) / groups;
    // few tokens: their heads are spread over thread blocks until the GPU is covered four times
    int parts = (4 * kSmCount + n_tok - 1) / n_tok;
    parts = parts < 1 ? 1 : parts > most ? most : parts;
    return launch_chained(kernel, static_cast<unsigned>(n_tok) * parts, kThreads, 0, st, a, parts);
}
template <typename T, bool EIGHT, bool INTERLEAVED>
halo_status by_width(const NormAppendArgs& a, int n_tok, cudaStream_t st) {
    return a.dh <= 64    ? launch<4>(paged_norm_append_kernel<T, 4, EIGHT, INTERLEAVED>, a, n_tok, st)
           : a.dh <= 128 ? launch<8>(paged_norm_append_kernel<T, 8, EIGHT, INTERLEAVED>, a, n_tok, st)
                         : launch<16>(paged_norm_append_kernel<T, 16, EIGHT, INTERLEAVED>, a, n_tok, st);
}
template <typename T, bool EIGHT>
halo_status by_pairs(const NormAppendArgs& a, int n_tok, int interleaved, cudaStream_t st) {
    if (interleaved) return by_width<T, EIGHT, true>(a, n_tok, st);
    if (a.rotary / 2 % kOwn == 0) return by_width<T, EIGHT, false>(a, n_tok, st);
    return a.dh <= 64    ? launch<8>(paged_norm_append_any_kernel<T, 8, EIGHT>, a, n_tok, st)
           : a.dh <= 128 ? launch<16>(paged_norm_append_any_kernel<T, 16, EIGHT>, a, n_tok, st)
                         : launch<32>(paged_norm_append_any_kernel<T, 32, EIGHT>, a, n_tok, st);
}

struct ReadArgs {
    int Hk, dh, page_size, n_pages, max_pages, n_seq;
    long long page_stride, k_stride, v_stride;
    const int32_t* pos;
    const int32_t* seq;
    const int32_t* table;
    const void* K;
    const void* V;
    const uint8_t* K_scale;
    const uint8_t* V_scale;
    void* k_out;
    void* v_out;
    uint32_t* status;
};

// Thread block: a token (four, with their chains of loads side by side, took 15.1 us and not 12.7 for 8297 tokens, 8 heads of 128 in 8
// bits, in thread blocks of four warps).  A unit is 16 bytes of the cache: of 8-bit rows 16 codes, which leave as 32 bytes of bf16.
template <typename T, bool EIGHT>
__global__ void __launch_bounds__(kThreads) paged_kv_read_kernel(const __grid_constant__ ReadArgs a) {
    constexpr int E = EIGHT ? 16 : Elem<T>::kPerChunk;
    const int tok = blockIdx.x;
    chain_wait();
    const int pos = ldg_waited(a.pos + tok);
    const int s = a.seq ? ldg_waited(a.seq + tok) : tok;
    if (pos < 0) return;               // a padding row
    const int pi = pos / a.page_size, in_page = pos - pi * a.page_size;
    int page = -1;
    if (s >= 0 && s < a.n_seq && pi < a.max_pages) page = ldg_waited(a.table + static_cast<long long>(s) * a.max_pages + pi);
    if (page < 0 || page >= a.n_pages) {
        if (threadIdx.x == 0) flag_status(a.status, HALO_DEV_BAD_INDEX);
        return;
    }
    const int per_head = a.dh / E, per_row = a.Hk * per_head;
    for (int u = threadIdx.x; u < 2 * per_row; u += kThreads) {
        const bool is_v = u >= per_row;
        const int w = is_v ? u - per_row : u, h = w / per_head, el = (w - h * per_head) * E;
        const long long row = static_cast<long long>(h) * a.page_size + in_page, from = page * a.page_stride + row * a.dh + el;
        T* to = (is_v ? static_cast<T*>(a.v_out) + static_cast<long long>(tok) * a.v_stride
                      : static_cast<T*>(a.k_out) + static_cast<long long>(tok) * a.k_stride) + h * a.dh + el;
        if constexpr (EIGHT) {
            const uint4 x = *reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(is_v ? a.V : a.K) + from);
            const float unit = eight_unit((is_v ? a.V_scale : a.K_scale)[static_cast<long long>(page) * a.Hk * a.page_size + row]);
            const uint32_t in[4] = {x.x, x.y, x.z, x.w};
            __align__(16) T out[16];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float f[4];
                eight_widen(in[j], f);
#pragma unroll
                for (int e = 0; e < 4; ++e) out[4 * j + e] = from_float<T>(f[e] * unit);   // exact
            }
            reinterpret_cast<uint4*>(to)[0] = reinterpret_cast<const uint4*>(out)[0];
            reinterpret_cast<uint4*>(to)[1] = reinterpret_cast<const uint4*>(out)[1];
        } else {
            *reinterpret_cast<uint4*>(to) = *reinterpret_cast<const uint4*>(static_cast<const T*>(is_v ? a.V : a.K) + from);
        }
    }
}
template <typename T, bool EIGHT>
halo_status launch_read(const ReadArgs& a, int n_tok, cudaStream_t st) {
    return launch_chained(paged_kv_read_kernel<T, EIGHT>, static_cast<unsigned>(n_tok), kThreads, 0, st, a);
}

}  // namespace

// What an 8-bit cache asks for beside its shape: both scale arrays or neither; queries, keys and values in bf16, which holds
// every value of it; pages that begin on 16 bytes.
halo_status check_eight(const halo_paged_shape& s, const void* K_scale, const void* V_scale) {
    if (!K_scale != !V_scale) return HALO_ERR_ARG;
    if (!K_scale) return HALO_OK;
    if (s.dtype != HALO_BF16) return HALO_ERR_DTYPE;
    if (s.page_stride % 16 != 0) return HALO_ERR_SHAPE;
    return aligned16(K_scale) && aligned16(V_scale) ? HALO_OK : HALO_ERR_ALIGN;
}

}  // namespace halo

using namespace halo;

extern "C" halo_status halo_paged_norm_append(const halo_paged_shape* shape, int n_tok, int n_seq, const void* q, long long q_stride,
                                              const void* k, long long k_stride, const void* v, long long v_stride, const void* w_q,
                                              const void* w_k, float eps, const int32_t* pos, const int32_t* seq_of_tok,
                                              const int32_t* block_table, const double* inv_freq, int rotary_dim, int interleaved,
                                              float turn_scale, void* q_out, long long q_out_stride, void* K_cache, void* V_cache,
                                              uint8_t* K_scale, uint8_t* V_scale, uint32_t* dev_status, void* stream) {
    halo_status rc = check_paged_shape(shape);
    if (rc != HALO_OK) return rc;
    if (!k || !v || !pos || !block_table || !K_cache || !V_cache) return HALO_ERR_ARG;
    if (!q != !q_out || (rotary_dim > 0 && !inv_freq)) return HALO_ERR_ARG;
    if (((w_q || w_k) && !(eps > 0.0f && isfinite(eps))) || !(turn_scale > 0.0f && isfinite(turn_scale))) return HALO_ERR_ARG;
    if (n_tok <= 0 || n_tok > (1 << 24) || n_seq <= 0 || (!seq_of_tok && n_tok > n_seq)) return HALO_ERR_SHAPE;
    if (rotary_dim < 0 || rotary_dim % 2 != 0 || rotary_dim > shape->head_dim) return HALO_ERR_SHAPE;
    const long long q_row = static_cast<long long>(shape->n_heads) * shape->head_dim;
    const long long k_row = static_cast<long long>(shape->n_kv_heads) * shape->head_dim;
    if ((q && (q_stride < q_row || q_out_stride < q_row)) || k_stride < k_row || v_stride < k_row) return HALO_ERR_SHAPE;
    const int elem = shape->dtype == HALO_F32 ? 4 : 2;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(q_out) || !aligned16(K_cache) || !aligned16(V_cache) ||
        !aligned16(w_q) || !aligned16(w_k) || (q && (q_stride * elem % 16 != 0 || q_out_stride * elem % 16 != 0)) ||
        k_stride * elem % 16 != 0 || v_stride * elem % 16 != 0)
        return HALO_ERR_ALIGN;
    rc = check_eight(*shape, K_scale, V_scale);
    if (rc != HALO_OK) return rc;
    if (q && q == q_out && n_tok > 1 && q_stride != q_out_stride) return HALO_ERR_ARG;   // a row would fall on its neighbours
    NormAppendArgs a = {};
    a.H = q ? shape->n_heads : 0;
    a.Hk = shape->n_kv_heads;
    a.dh = shape->head_dim;
    a.page_size = shape->page_size;
    a.n_pages = shape->n_pages;
    a.max_pages = shape->max_pages;
    a.n_seq = n_seq;
    a.rotary = rotary_dim;
    a.page_stride = paged_stride(*shape);
    a.q_stride = q_stride;
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    a.qo_stride = q_out_stride;
    a.eps = eps;
    a.turn_scale = turn_scale;
    a.q = q;
    a.k = k;
    a.v = v;
    a.w_q = q ? w_q : nullptr;
    a.w_k = w_k;
    a.pos = pos;
    a.seq = seq_of_tok;
    a.table = block_table;
    a.inv_freq = inv_freq;
    a.q_out = q_out;
    a.K = K_cache;
    a.V = V_cache;
    a.K_scale = K_scale;
    a.V_scale = V_scale;
    a.status = dev_status;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (shape->dtype == HALO_F32) return by_pairs<float, false>(a, n_tok, interleaved != 0, st);
    return K_scale ? by_pairs<__nv_bfloat16, true>(a, n_tok, interleaved != 0, st)
                   : by_pairs<__nv_bfloat16, false>(a, n_tok, interleaved != 0, st);
}

extern "C" halo_status halo_paged_kv_read(const halo_paged_shape* shape, int n_tok, int n_seq, const int32_t* pos,
                                          const int32_t* seq_of_tok, const int32_t* block_table, const void* K_cache,
                                          const void* V_cache, const uint8_t* K_scale, const uint8_t* V_scale, void* k_out,
                                          long long k_stride, void* v_out, long long v_stride, uint32_t* dev_status, void* stream) {
    halo_status rc = check_paged_shape(shape);
    if (rc != HALO_OK) return rc;
    if (!pos || !block_table || !K_cache || !V_cache || !k_out || !v_out) return HALO_ERR_ARG;
    if (n_tok <= 0 || n_tok > (1 << 24) || n_seq <= 0 || (!seq_of_tok && n_tok > n_seq)) return HALO_ERR_SHAPE;
    const long long k_row = static_cast<long long>(shape->n_kv_heads) * shape->head_dim;
    if (k_stride < k_row || v_stride < k_row) return HALO_ERR_SHAPE;
    const int elem = shape->dtype == HALO_F32 ? 4 : 2;
    if (!aligned16(K_cache) || !aligned16(V_cache) || !aligned16(k_out) || !aligned16(v_out) || k_stride * elem % 16 != 0 ||
        v_stride * elem % 16 != 0)
        return HALO_ERR_ALIGN;
    rc = check_eight(*shape, K_scale, V_scale);
    if (rc != HALO_OK) return rc;
    ReadArgs a = {};
    a.Hk = shape->n_kv_heads;
    a.dh = shape->head_dim;
    a.page_size = shape->page_size;
    a.n_pages = shape->n_pages;
    a.max_pages = shape->max_pages;
    a.n_seq = n_seq;
    a.page_stride = paged_stride(*shape);
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    a.pos = pos;
    a.seq = seq_of_tok;
    a.table = block_table;
    a.K = K_cache;
    a.V = V_cache;
    a.K_scale = K_scale;
    a.V_scale = V_scale;
    a.k_out = k_out;
    a.v_out = v_out;
    a.status = dev_status;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (shape->dtype == HALO_F32) return launch_read<float, false>(a, n_tok, st);
    return K_scale ? launch_read<__nv_bfloat16, true>(a, n_tok, st) : launch_read<__nv_bfloat16, false>(a, n_tok, st);
}
