// halo_paged_kv_append: the keys and values of new tokens go to their pages, keys and queries turned by their
// position on the way.  HBM-bound: every element is read once and written once.
//
// Rotation: pair i of a head is turned by the angle pos * inv_freq[i].  The angle is formed and reduced to one turn in
// fp64 (at position 1e5 an fp32 product is off by 4e-3 radians), cosine and sine are taken in fp32 of the reduced
// angle, once per token and pair, and shared by all heads of the token through shared memory.
// A thread keeps its place inside a head (one 16-byte chunk, or the two chunks of its pairs) and walks over the heads
// of q, k and v alike, so cosines, sines and offsets stay in registers; the loads of its first heads are in flight
// while the angles are computed.  Few tokens: the heads of a token are spread over several thread blocks.
// Heads of 128, 32 + 2 * 8 of them: 8297 tokens (204 MB read and written) 37 us = 5.5 TB/s, what is left being the two
// dependent loads (position, page) in front of a thread block's stores; fp32 (408 MB) 63 us = 6.5 TB/s; 32 tokens 3.3 to
// 3.7 us, the launch.  Pairs (i, i + rotary / 2) whose distance is no whole number of 16-byte chunks go an element at a time:
// heads of 80 (127 MB) 31 us with 80 elements turned and 67 with 40, heads of 96 (153 MB) 41 with 32 turned and 85 with
// 24; interleaved pairs, fp32 (heads of 80, 40 turned, 255 MB: 42) and few tokens do not have the step.
#include "common.cuh"

namespace halo {
halo_status check_paged_shape(const halo_paged_shape* s);
long long paged_stride(const halo_paged_shape& s);

namespace {

constexpr int kThreads = 128;
constexpr int kHeads = 3;   // heads in flight per thread

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
// 16-byte chunks.  Thread block (token, part): heads part, part + parts, ... in runs of `lanes` heads.
template <typename T, bool INTERLEAVED, bool WIDE>
__global__ void __launch_bounds__(WIDE ? kThreads : 256)
paged_append_kernel(const __grid_constant__ AppendArgs a, int parts, int units, int lanes) {
    constexpr int E = WIDE ? Elem<T>::kPerChunk : 1;
    constexpr int kPairs = INTERLEAVED ? E / 2 : E;
    extern __shared__ float2 turn[];   // [rotary / 2] cosine, sine
    const int tid = threadIdx.x;
    const int tok = blockIdx.x / parts, part = blockIdx.x % parts;
    chain_wait();
    // everything that depends on the token alone is requested at once
    const int pos = ldg_waited(a.pos + tok);
    const int s = a.seq ? ldg_waited(a.seq + tok) : tok;
    const int half = a.rotary / 2;
    const int pair_units = INTERLEAVED ? 0 : half / E;   // units of two chunks per head
    const int c = tid % units, hl = tid / units;
    const int el = INTERLEAVED || c < pair_units ? c * E : a.rotary + (c - pair_units) * E;
    const int gap = c < pair_units ? half : 0;           // distance of the second chunk
    const int pair0 = INTERLEAVED ? el / 2 : el;         // first pair of the unit
    const bool turned = INTERLEAVED ? el < a.rotary : c < pair_units;
    const int heads = a.H + 2 * a.Hk;
    const T* q = static_cast<const T*>(a.q) + static_cast<long long>(tok) * a.q_stride + el;
    const T* k = static_cast<const T*>(a.k) + static_cast<long long>(tok) * a.k_stride + el;
    const T* v = static_cast<const T*>(a.v) + static_cast<long long>(tok) * a.v_stride + el;
    const int step = lanes * parts;
    const int first = hl < lanes ? part * lanes + hl : heads;

    alignas(16) T x[kHeads][2][E];
    auto fetch = [&](int h0) {
#pragma unroll
        for (int i = 0; i < kHeads; ++i) {
            const int h = h0 + i * step;
            if (h >= heads) continue;
            const T* src = h < a.H ? q + h * a.dh : h < a.H + a.Hk ? k + (h - a.H) * a.dh : v + (h - a.H - a.Hk) * a.dh;
            if constexpr (WIDE) {
                *reinterpret_cast<uint4*>(x[i][0]) = *reinterpret_cast<const uint4*>(src);
                if (gap) *reinterpret_cast<uint4*>(x[i][1]) = *reinterpret_cast<const uint4*>(src + gap);
            } else {
                x[i][0][0] = src[0];
                if (gap) x[i][1][0] = src[gap];
            }
        }
    };
    const double freq = tid < half ? ldg_waited(a.inv_freq + tid) : 0.0;   // half <= 128 threads
    fetch(first);

    if (pos < 0) return;               // a padding row: nothing is written for it
    const int pi = pos / a.page_size;
    int page = -1;
    if (s >= 0 && s < a.n_seq && pi < a.max_pages) page = ldg_waited(a.table + static_cast<long long>(s) * a.max_pages + pi);
    if (tid < half) {
        const double turns = static_cast<double>(pos) * freq * 0.15915494309189533577;
        float co, si;
        sincospif(static_cast<float>(2.0 * (turns - rint(turns))), &si, &co);
        turn[tid] = make_float2(co, si);
    }
    if (page < 0 || page >= a.n_pages) {   // the same in every thread
        if (tid == 0 && part == 0) flag_status(a.status, HALO_DEV_BAD_INDEX);
        return;
    }
    __syncthreads();
    float co[kPairs], si[kPairs];
#pragma unroll
    for (int e = 0; e < kPairs; ++e) {
        const bool in = turned && pair0 + e < half;      // an interleaved chunk may end behind the last pair
        co[e] = in ? turn[pair0 + e].x : 1.0f;
        si[e] = in ? turn[pair0 + e].y : 0.0f;
    }
    const long long base = static_cast<long long>(page) * a.page_stride + static_cast<long long>(pos % a.page_size) * a.dh + el;
    const long long plane = static_cast<long long>(a.page_size) * a.dh;
    T* qo = static_cast<T*>(a.q_out) + static_cast<long long>(tok) * a.qo_stride + el;

    for (int h0 = first; h0 < heads; h0 += step * kHeads) {
        if (h0 != first) fetch(h0);
#pragma unroll
        for (int i = 0; i < kHeads; ++i) {
            const int h = h0 + i * step;
            if (h >= heads) continue;
            T* dst = h < a.H           ? qo + h * a.dh
                     : h < a.H + a.Hk ? static_cast<T*>(a.K) + base + (h - a.H) * plane
                                      : static_cast<T*>(a.V) + base + (h - a.H - a.Hk) * plane;
            if (turned && h < a.H + a.Hk) {
#pragma unroll
                for (int e = 0; e < kPairs; ++e) {
                    T& first_of = INTERLEAVED ? x[i][0][2 * e] : x[i][0][e];
                    T& second_of = INTERLEAVED ? x[i][0][2 * e + 1] : x[i][1][e];
                    const float p = to_float(first_of), o = to_float(second_of);
                    // a pair behind the last one is left as it is (infinity * 0 would not be)
                    if (INTERLEAVED && pair0 + e >= half) continue;
                    first_of = from_float<T>(p * co[e] - o * si[e]);
                    second_of = from_float<T>(p * si[e] + o * co[e]);
                }
            }
            if constexpr (WIDE) {
                *reinterpret_cast<uint4*>(dst) = *reinterpret_cast<const uint4*>(x[i][0]);
                if (gap) *reinterpret_cast<uint4*>(dst + gap) = *reinterpret_cast<const uint4*>(x[i][1]);
            } else {
                dst[0] = x[i][0][0];
                if (gap) dst[gap] = x[i][1][0];
            }
        }
    }
}

template <typename T>
halo_status launch(const AppendArgs& a, int n_tok, int interleaved, cudaStream_t st) {
    constexpr int E = Elem<T>::kPerChunk;
    const bool wide = interleaved || (a.rotary / 2) % E == 0;
    const int e = wide ? E : 1;
    const int units = interleaved ? a.dh / e : a.rotary / 2 / e + (a.dh - a.rotary) / e;   // per head, <= 256
    const int threads = wide ? kThreads : 256;
    const int lanes = threads / units;          // heads side by side in a thread block
    const int heads = a.H + 2 * a.Hk;
    const int most = (heads + lanes - 1) / lanes;
    // few tokens: their heads are spread over thread blocks until the GPU is covered four times
    int parts = (4 * kSmCount + n_tok - 1) / n_tok;
    parts = parts < 1 ? 1 : parts > most ? most : parts;
    const unsigned grid = static_cast<unsigned>(n_tok) * parts;
    const size_t smem = sizeof(float2) * (a.rotary / 2);
    const auto kernel = interleaved ? paged_append_kernel<T, true, true>
                        : wide      ? paged_append_kernel<T, false, true>
                                    : paged_append_kernel<T, false, false>;
    return launch_chained(kernel, grid, threads, smem, st, a, parts, units, lanes);
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
    if (q && q == q_out && n_tok > 1 && q_stride != q_out_stride) return HALO_ERR_ARG;   // a row would fall on its neighbours
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
