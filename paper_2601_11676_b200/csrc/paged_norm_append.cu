// halo_paged_norm_append: the keys and values of new tokens go to their pages in the caches' type or as 8-bit rows, queries
// and keys normed per head and turned by their position on the way; halo_paged_kv_read: rows back out of the pages.
// HBM-bound: every element is read once and written once.
//
//   y = x / sqrt(mean(x^2) + eps) * w over a head's elements (queries and keys that have a gain), then pair i of the first
//   rotary elements by the angle pos * inv_freq[i], times turn_scale.  Angles as in halo_paged_kv_append: reduced to one turn in
//   fp64, cosine and sine in fp32, once per token, through shared memory.  Everything between the load and the one rounding
//   of the store is fp32.
//
// A lane keeps eight elements of the head (16 bytes of bf16) and walks over the heads of q, k and v alike, so gains, cosines and
// sines stay in registers; LANES lanes hold a head, a power of two, and sum its squares and find its largest element by
// shuffles.  The other half of a pair (i, i + rotary / 2) is in another lane: normed elements pass through a row of shared memory
// that only the warp's own lanes touch.
#include <math.h>

#include "eight.cuh"

namespace halo {
halo_status check_paged_shape(const halo_paged_shape* s);
halo_status check_eight(const halo_paged_shape& s, const void* K_scale, const void* V_scale);
long long paged_stride(const halo_paged_shape& s);

namespace {

constexpr int kThreads = 128;
constexpr int kOwn = 8;      // elements per lane
constexpr int kHeads = 3;    // heads in flight per lane

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

// Thread block (token, part): heads part * groups + group, ... in steps of groups * parts.
template <typename T, int LANES, bool EIGHT>
__global__ void __launch_bounds__(kThreads)
paged_norm_append_kernel(const __grid_constant__ NormAppendArgs a, int parts, int interleaved) {
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
    Own<T> x[kHeads];
    const auto fetch = [&](int h0) {
#pragma unroll
        for (int i = 0; i < kHeads; ++i) {
            const int h = h0 + i * step;
            if (in && h < heads)
                x[i].load(h < a.H ? q + h * a.dh : h < a.H + a.Hk ? k + (h - a.H) * a.dh : v + (h - a.H - a.Hk) * a.dh);
        }
    };
    const int first = part * kGroups + group;
    const double freq = tid < half ? ldg_waited(a.inv_freq + tid) : 0.0;   // half <= 128 threads
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
    if (tid < half) {
        const double turns = static_cast<double>(pos) * freq * 0.15915494309189533577;
        float co, si;
        sincospif(static_cast<float>(2.0 * (turns - rint(turns))), &si, &co);
        turn[tid] = make_float2(co * a.turn_scale, si * a.turn_scale);
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
            const bool second = interleaved ? at & 1 : at >= half;
            const float2 t = turn[interleaved ? at >> 1 : second ? at - half : at];
            co[e] = t.x;
            si[e] = second ? t.y : -t.y;
        }
    }
    const bool turned = el < a.rotary;                 // elements behind the last pair are left as they are (infinity * 0 would not be)
    const bool whole = half % kOwn == 0;               // the other halves of a lane's pairs are eight neighbours
    const long long row = static_cast<long long>(page) * a.Hk * a.page_size + pos % a.page_size;   // of the scales
    const long long base = static_cast<long long>(page) * a.page_stride + static_cast<long long>(pos % a.page_size) * a.dh + el;
    const long long plane = static_cast<long long>(a.page_size) * a.dh;
    T* qo = static_cast<T*>(a.q_out) + static_cast<long long>(tok) * a.qo_stride + el;
    float* mine = rows[group];

    // every lane of a warp takes every step: lanes meet in the shuffles
    for (int h0 = first, b0 = part * kGroups; b0 < heads; h0 += step * kHeads, b0 += step * kHeads) {
        if (h0 != first) fetch(h0);
#pragma unroll
        for (int i = 0; i < kHeads; ++i) {
            if (b0 + i * step >= heads) break;         // the same in every lane of the block
            const int h = h0 + i * step;
            const bool there = in && h < heads, is_q = h < a.H, is_v = h >= a.H + a.Hk;
            float f[kOwn];
#pragma unroll
            for (int e = 0; e < kOwn; ++e) f[e] = 0.0f;
            if (there) x[i].widen(f);
            const bool normed = !is_v && (is_q ? a.w_q : a.w_k) != nullptr;
            if (a.w_q || a.w_k) {
                float sum = 0.0f;
#pragma unroll
                for (int e = 0; e < kOwn; ++e) sum = fmaf(f[e], f[e], sum);
                sum = lanes_sum<LANES>(sum);
                if (there && normed) {
                    const float n = 1.0f / sqrtf(sum / static_cast<float>(a.dh) + a.eps);
#pragma unroll
                    for (int e = 0; e < kOwn; ++e) f[e] = f[e] * n * (is_q ? wq[e] : wk[e]);
                }
            }
            if (interleaved) {
                if (turned && !is_v) {
#pragma unroll
                    for (int e = 0; e < kOwn; e += 2) {
                        if (el + e >= a.rotary) continue;
                        const float p = f[e], o = f[e + 1];
                        f[e] = p * co[e] + o * si[e];
                        f[e + 1] = o * co[e + 1] + p * si[e + 1];
                    }
                }
            } else if (a.rotary > 0) {
                __syncwarp();
                *reinterpret_cast<float4*>(mine + el) = make_float4(f[0], f[1], f[2], f[3]);
                *reinterpret_cast<float4*>(mine + el + 4) = make_float4(f[4], f[5], f[6], f[7]);
                __syncwarp();
                if (turned && !is_v) {
                    float o[kOwn];
                    if (whole) {
                        const float* from = mine + (el < half ? el + half : el - half);
                        *reinterpret_cast<float4*>(o) = *reinterpret_cast<const float4*>(from);
                        *reinterpret_cast<float4*>(o + 4) = *reinterpret_cast<const float4*>(from + 4);
                    } else {
#pragma unroll
                        for (int e = 0; e < kOwn; ++e) {
                            const int at = el + e;
                            o[e] = at < a.rotary ? mine[at < half ? at + half : at - half] : 0.0f;
                        }
                    }
#pragma unroll
                    for (int e = 0; e < kOwn; ++e)
                        if (el + e < a.rotary) f[e] = f[e] * co[e] + o[e] * si[e];
                }
            }
            if (EIGHT && b0 + i * step + kGroups > a.H) {      // a head of this pass is a key or a value
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
                x[i].narrow(f);
                x[i].store(is_q ? qo + h * a.dh
                           : is_v ? static_cast<T*>(a.V) + base + (h - a.H - a.Hk) * plane
                                  : static_cast<T*>(a.K) + base + (h - a.H) * plane);
            }
        }
    }
}

template <typename T, int LANES, bool EIGHT>
halo_status launch(const NormAppendArgs& a, int n_tok, int interleaved, cudaStream_t st) {
    const int groups = kThreads / LANES, heads = a.H + 2 * a.Hk, most = (heads + groups - 1) / groups;
    // few tokens: their heads are spread over thread blocks until the GPU is covered four times
    int parts = (4 * kSmCount + n_tok - 1) / n_tok;
    parts = parts < 1 ? 1 : parts > most ? most : parts;
    return launch_chained(paged_norm_append_kernel<T, LANES, EIGHT>, static_cast<unsigned>(n_tok) * parts, kThreads, 0, st, a, parts,
                          interleaved);
}
template <typename T, bool EIGHT>
halo_status by_width(const NormAppendArgs& a, int n_tok, int interleaved, cudaStream_t st) {
    return a.dh <= 64    ? launch<T, 8, EIGHT>(a, n_tok, interleaved, st)
           : a.dh <= 128 ? launch<T, 16, EIGHT>(a, n_tok, interleaved, st)
                         : launch<T, 32, EIGHT>(a, n_tok, interleaved, st);
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

// Thread block: a token.  A unit is 16 bytes of the cache: of 8-bit rows 16 codes, which leave as 32 bytes of bf16.
template <typename T, bool EIGHT>
__global__ void __launch_bounds__(kThreads) paged_kv_read_kernel(const __grid_constant__ ReadArgs a) {
    constexpr int E = EIGHT ? 16 : Elem<T>::kPerChunk;
    const int tok = blockIdx.x;
    chain_wait();
    const int pos = ldg_waited(a.pos + tok), s = a.seq ? ldg_waited(a.seq + tok) : tok;
    if (pos < 0) return;
    const int pi = pos / a.page_size, at = pos % a.page_size;
    int page = -1;
    if (s >= 0 && s < a.n_seq && pi < a.max_pages) page = ldg_waited(a.table + static_cast<long long>(s) * a.max_pages + pi);
    if (page < 0 || page >= a.n_pages) {
        if (threadIdx.x == 0) flag_status(a.status, HALO_DEV_BAD_INDEX);
        return;
    }
    const int per_head = a.dh / E, per_row = a.Hk * per_head;
    const long long base = static_cast<long long>(page) * a.page_stride;
    for (int u = threadIdx.x; u < 2 * per_row; u += kThreads) {
        const bool is_v = u >= per_row;
        const int w = is_v ? u - per_row : u, h = w / per_head, el = (w - h * per_head) * E;
        const long long from = base + (static_cast<long long>(h) * a.page_size + at) * a.dh + el;
        T* to = (is_v ? static_cast<T*>(a.v_out) + static_cast<long long>(tok) * a.v_stride
                      : static_cast<T*>(a.k_out) + static_cast<long long>(tok) * a.k_stride) + h * a.dh + el;
        if constexpr (EIGHT) {
            const uint4 codes = *reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(is_v ? a.V : a.K) + from);
            const float unit = eight_unit((is_v ? a.V_scale : a.K_scale)[(static_cast<long long>(page) * a.Hk + h) * a.page_size + at]);
            const uint32_t in[4] = {codes.x, codes.y, codes.z, codes.w};
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
    if (shape->dtype == HALO_F32) return by_width<float, false>(a, n_tok, interleaved != 0, st);
    return K_scale ? by_width<__nv_bfloat16, true>(a, n_tok, interleaved != 0, st)
                   : by_width<__nv_bfloat16, false>(a, n_tok, interleaved != 0, st);
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
    const auto kernel = shape->dtype == HALO_F32 ? paged_kv_read_kernel<float, false>
                        : K_scale                ? paged_kv_read_kernel<__nv_bfloat16, true>
                                                 : paged_kv_read_kernel<__nv_bfloat16, false>;
    return launch_chained(kernel, static_cast<unsigned>(n_tok), kThreads, 0, st, a);
}
