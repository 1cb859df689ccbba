// halo_paged_kv_append: the keys and values of new tokens go to their pages, keys and queries turned by their
// position on the way.  HBM-bound: every element is read once and written once.
//
// Rotation: pair i of a head is turned by the angle pos * inv_freq[i].  The angle is formed and reduced to one turn in
// fp64 (at position 1e5 an fp32 product is off by 4e-3 radians), cosine and sine are taken in fp32 of the reduced
// angle, once per token and pair, and shared by all heads of the token through shared memory.
// A thread block takes one token and part of its heads; the loads of a thread's first units are in flight while the
// angles are computed.
#include "common.cuh"

namespace halo {
halo_status check_paged_shape(const halo_paged_shape* s);
long long paged_stride(const halo_paged_shape& s);

namespace {

constexpr int kThreads = 256;
constexpr int kUnits = 3;   // units in flight per thread

struct AppendArgs {
    int H, Hk, dh, page_size, n_pages, max_pages, n_seq, rotary;
    long long page_stride, q_stride, k_stride, v_stride, qo_stride;
    const void* q;
    const void* k;
    const void* v;
    const int32_t* pos;
    const int32_t* seq;
    const int32_t* table;
    const double* inv_freq;
    void* q_out;
    void* K;
    void* V;
    uint32_t* status;
};

// A unit is one 16-byte chunk (interleaved pairs, or elements that are not turned), or the two chunks that hold pairs
// (i, i + rotary / 2).  WIDE = false: chunks of one element, for rotary sizes whose half is not a whole number of
// 16-byte chunks.
template <typename T, bool INTERLEAVED, bool WIDE>
__global__ void __launch_bounds__(kThreads) paged_append_kernel(const __grid_constant__ AppendArgs a, int parts) {
    constexpr int E = WIDE ? Elem<T>::kPerChunk : (INTERLEAVED ? 2 : 1);
    extern __shared__ float2 turn[];   // [rotary / 2] cosine, sine
    const int tid = threadIdx.x;
    const int tok = blockIdx.x / parts, part = blockIdx.x % parts;
    const int pos = __ldg(a.pos + tok);
    if (pos < 0) return;               // a padding row: nothing of it is read or written
    const int s = a.seq ? __ldg(a.seq + tok) : tok;
    const int pi = pos / a.page_size;
    int page = -1;
    if (s >= 0 && s < a.n_seq && pi < a.max_pages) page = __ldg(a.table + static_cast<long long>(s) * a.max_pages + pi);
    if (page < 0 || page >= a.n_pages) {
        if (tid == 0 && part == 0) flag_status(a.status, HALO_DEV_BAD_INDEX);
        return;
    }
    const int half = a.rotary / 2;
    const int pair_units = INTERLEAVED ? 0 : half / E;                          // units of two chunks per head
    const int turned_units = INTERLEAVED ? (a.rotary + E - 1) / E : pair_units; // units that are turned per head
    const int units = pair_units + (a.dh - (INTERLEAVED ? 0 : a.rotary)) / E;   // units per head
    const int v_units = a.dh / E;
    const int all = (a.H + a.Hk) * units + a.Hk * v_units;
    const int per_part = (all + parts - 1) / parts;
    const int u1 = min(all, (part + 1) * per_part);
    const long long base = static_cast<long long>(page) * a.page_stride + static_cast<long long>(pos % a.page_size) * a.dh;
    const T* q = static_cast<const T*>(a.q) + static_cast<long long>(tok) * a.q_stride;
    const T* k = static_cast<const T*>(a.k) + static_cast<long long>(tok) * a.k_stride;
    const T* v = static_cast<const T*>(a.v) + static_cast<long long>(tok) * a.v_stride;
    T* qo = static_cast<T*>(a.q_out) + static_cast<long long>(tok) * a.qo_stride;

    bool ready = false;
    for (int u = part * per_part + tid; u - tid < u1; u += kThreads * kUnits) {
        alignas(16) T x[kUnits][2][E];
        const T* src[kUnits];
        T* dst[kUnits];
        int gap[kUnits];      // distance of the second chunk, 0: none
        int pair0[kUnits];    // first pair of the unit, -1: not turned
#pragma unroll
        for (int i = 0; i < kUnits; ++i) {
            const int w = u + i * kThreads;
            src[i] = nullptr;
            if (w >= u1) continue;
            int head, c, el = 0;
            gap[i] = 0;
            pair0[i] = -1;
            if (w < (a.H + a.Hk) * units) {
                head = w / units;
                c = w - head * units;
                if (INTERLEAVED) {
                    el = c * E;
                    if (c < turned_units) pair0[i] = el / 2;
                } else if (c < pair_units) {
                    el = c * E;
                    gap[i] = half;
                    pair0[i] = el;
                } else {
                    el = a.rotary + (c - pair_units) * E;
                }
                if (head < a.H) {
                    src[i] = q + head * a.dh + el;
                    dst[i] = qo + head * a.dh + el;
                } else {
                    src[i] = k + (head - a.H) * a.dh + el;
                    dst[i] = static_cast<T*>(a.K) + base + static_cast<long long>(head - a.H) * a.page_size * a.dh + el;
                }
            } else {
                const int r = w - (a.H + a.Hk) * units;
                head = r / v_units;
                el = (r - head * v_units) * E;
                src[i] = v + head * a.dh + el;
                dst[i] = static_cast<T*>(a.V) + base + static_cast<long long>(head) * a.page_size * a.dh + el;
            }
            if constexpr (WIDE) {
                *reinterpret_cast<uint4*>(x[i][0]) = *reinterpret_cast<const uint4*>(src[i]);
                if (gap[i]) *reinterpret_cast<uint4*>(x[i][1]) = *reinterpret_cast<const uint4*>(src[i] + gap[i]);
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e) x[i][0][e] = src[i][e];
                if (gap[i]) x[i][1][0] = src[i][gap[i]];
            }
        }
        if (!ready) {
            for (int i = tid; i < half; i += kThreads) {
                const double turns = static_cast<double>(pos) * __ldg(a.inv_freq + i) * 0.15915494309189533577;
                float c, sn;
                sincospif(static_cast<float>(2.0 * (turns - rint(turns))), &sn, &c);
                turn[i] = make_float2(c, sn);
            }
            __syncthreads();
            ready = true;
        }
#pragma unroll
        for (int i = 0; i < kUnits; ++i) {
            if (!src[i]) continue;
            if (pair0[i] >= 0) {
                if constexpr (INTERLEAVED) {
#pragma unroll
                    for (int e = 0; e < E; e += 2) {
                        if (pair0[i] + e / 2 >= half) break;
                        const float2 cs = turn[pair0[i] + e / 2];
                        const float p = to_float(x[i][0][e]), o = to_float(x[i][0][e + 1]);
                        x[i][0][e] = from_float<T>(p * cs.x - o * cs.y);
                        x[i][0][e + 1] = from_float<T>(p * cs.y + o * cs.x);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        const float2 cs = turn[pair0[i] + e];
                        const float p = to_float(x[i][0][e]), o = to_float(x[i][1][e]);
                        x[i][0][e] = from_float<T>(p * cs.x - o * cs.y);
                        x[i][1][e] = from_float<T>(p * cs.y + o * cs.x);
                    }
                }
            }
            if constexpr (WIDE) {
                *reinterpret_cast<uint4*>(dst[i]) = *reinterpret_cast<const uint4*>(x[i][0]);
                if (gap[i]) *reinterpret_cast<uint4*>(dst[i] + gap[i]) = *reinterpret_cast<const uint4*>(x[i][1]);
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e) dst[i][e] = x[i][0][e];
                if (gap[i]) dst[i][gap[i]] = x[i][1][0];
            }
        }
    }
}

template <typename T>
halo_status launch(const AppendArgs& a, int n_tok, int interleaved, cudaStream_t st) {
    constexpr int E = Elem<T>::kPerChunk;
    const bool wide = interleaved || (a.rotary / 2) % E == 0;
    const int e = wide ? E : 1;
    const int all = (a.H + a.Hk) * (interleaved ? a.dh / e : a.rotary / 2 / e + (a.dh - a.rotary) / e) + a.Hk * (a.dh / e);
    const int most = (all + kThreads * kUnits - 1) / (kThreads * kUnits);
    // few tokens: their heads are spread over thread blocks until the GPU is covered twice
    int parts = (2 * kSmCount + n_tok - 1) / n_tok;
    parts = parts < 1 ? 1 : parts > most ? most : parts;
    const unsigned grid = static_cast<unsigned>(n_tok) * parts;
    const size_t smem = sizeof(float2) * (a.rotary / 2);
    if (interleaved)
        paged_append_kernel<T, true, true><<<grid, kThreads, smem, st>>>(a, parts);
    else if (wide)
        paged_append_kernel<T, false, true><<<grid, kThreads, smem, st>>>(a, parts);
    else
        paged_append_kernel<T, false, false><<<grid, kThreads, smem, st>>>(a, parts);
    HALO_CHECK_LAUNCH();
    return HALO_OK;
}

}  // namespace
}  // namespace halo

using namespace halo;

extern "C" halo_status halo_paged_kv_append(const halo_paged_shape* shape, int n_tok, int n_seq, const void* q,
                                            long long q_stride, const void* k, long long k_stride, const void* v,
                                            long long v_stride, const int32_t* pos, const int32_t* seq_of_tok,
                                            const int32_t* block_table, const double* inv_freq, int rotary_dim,
                                            int interleaved, void* q_out, long long q_out_stride, void* K_cache,
                                            void* V_cache, uint32_t* dev_status, void* stream) {
    const halo_status rc = check_paged_shape(shape);
    if (rc != HALO_OK) return rc;
    if (!k || !v || !pos || !block_table || !K_cache || !V_cache) return HALO_ERR_ARG;
    if (!q != !q_out || (rotary_dim > 0 && !inv_freq)) return HALO_ERR_ARG;
    if (n_tok <= 0 || n_tok > (1 << 24) || n_seq <= 0 || (!seq_of_tok && n_tok > n_seq)) return HALO_ERR_SHAPE;
    if (rotary_dim < 0 || rotary_dim % 2 != 0 || rotary_dim > shape->head_dim) return HALO_ERR_SHAPE;
    const long long q_row = static_cast<long long>(shape->n_heads) * shape->head_dim;
    const long long k_row = static_cast<long long>(shape->n_kv_heads) * shape->head_dim;
    if ((q && (q_stride < q_row || q_out_stride < q_row)) || k_stride < k_row || v_stride < k_row) return HALO_ERR_SHAPE;
    const int elem = shape->dtype == HALO_F32 ? 4 : 2;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(q_out) || !aligned16(K_cache) || !aligned16(V_cache) ||
        (q && (q_stride * elem % 16 != 0 || q_out_stride * elem % 16 != 0)) || k_stride * elem % 16 != 0 ||
        v_stride * elem % 16 != 0)
        return HALO_ERR_ALIGN;
    AppendArgs a = {};
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
    a.q = q;
    a.k = k;
    a.v = v;
    a.pos = pos;
    a.seq = seq_of_tok;
    a.table = block_table;
    a.inv_freq = inv_freq;
    a.q_out = q_out;
    a.K = K_cache;
    a.V = V_cache;
    a.status = dev_status;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    return shape->dtype == HALO_F32 ? launch<float>(a, n_tok, interleaved != 0, st)
                                    : launch<__nv_bfloat16>(a, n_tok, interleaved != 0, st);
}
