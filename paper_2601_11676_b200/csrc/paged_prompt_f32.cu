// halo_paged_prompt_mha on fp32 caches, by fused multiply-adds: 64 rows against tiles of 64 keys.  Bound by them: 4 flops per key, row and
// column of the head at 2 * 128 a clock and SM.  3 chunks of up to 300 tokens over up to 400, 8 / 8 heads of 64: 27.6 us (7.6 TFLOP/s of
// some 70: most thread blocks have a tile or two, and the join another 8).
//
// 128 threads; a thread has 8 rows x 4 keys of the scores and 8 rows x DP / 16 columns of the weighted sums, so that twelve 16-byte
// words from shared memory feed 128 multiply-adds.  Rows in shared memory are padded by four floats, which spreads the
// eight rows of a phase over all banks.  The sixteen lanes of a row keep its maximum and sum by shuffles; weights go through
// shared memory that only their own half warp reads.  Copies of the next keys run under the softmax and the weighted sums, of
// the next values under the scores.
#include "prompt_line.cuh"

#include <type_traits>

namespace halo {
namespace prompt {
namespace {

constexpr int kRows = 64, kTile = 64, kThreads = 128, kOver = 1;

template <int DP>
struct Smem {
    static constexpr int kStride = DP + 4, kWeights = kTile + 4;
    float q[kRows * kStride], k[kTile * kStride], v[kTile * kStride], w[kRows * kWeights];
    long long row[2][kTile];     // of the caches' rows: page * page_stride + ..., -1: no such position
    long long sh[kThreads / 32 + 3];
};

__device__ __forceinline__ void cp_async16(float* dst, const void* src, bool valid) {
    const int n = valid ? 16 : 0;   // 0: the 16 bytes are filled with zeros and src is not read
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(static_cast<uint32_t>(__cvta_generic_to_shared(dst))), "l"(src), "r"(n)
                 : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

template <int DP>
__global__ void __launch_bounds__(kThreads) paged_prompt_rows_kernel(const __grid_constant__ Args a) {
    using S_ = Smem<DP>;
    constexpr int kStride = S_::kStride, kWeights = S_::kWeights, kCpr = DP / 4, V = DP / 64;
    extern __shared__ __align__(16) unsigned char raw[];
    S_& sm = *reinterpret_cast<S_*>(raw);
    const int tid = threadIdx.x, lane = tid & 31, tx = tid & 15, ty = tid >> 4;
    chain_wait();
    Found<kRows, kTile, kOver> f = locate<kRows, kTile, kOver, kThreads>(a, sm.sh);
    Walk<kRows, kTile, kOver>& w = f.walk;
    bool bad = false;

    while (w.left > 0) {
        const int kvh = w.kvh, nt = w.reach > 0 ? w.t1 - w.t0 : 0;
        // where the tile's rows are
        const auto places = [&](int t) {
            if (tid >= kTile) return;
            const int p = (w.t0 + t) * kTile + tid;
            long long at = -1;
            if (p < w.reach) {
                const int pi = a.page_shift >= 0 ? p >> a.page_shift : p / a.page_size, in = p - pi * a.page_size;
                const int page = ldg_waited(a.table + static_cast<long long>(w.s) * a.max_pages + pi);
                if (page >= 0 && page < a.n_pages) at = static_cast<long long>(page) * a.page_stride + (static_cast<long long>(kvh) * a.page_size + in) * a.dh;
                else bad = true;
            }
            sm.row[t & 1][tid] = at;
        };
        const auto fetch = [&](float* dst, const void* cache, int t) {
#pragma unroll 4
            for (int i = tid; i < kTile * kCpr; i += kThreads) {
                const int r = i / kCpr, c = i % kCpr;
                const long long at = sm.row[t & 1][r];
                const bool there = at >= 0 && c * 4 < a.dh;
                cp_async16(dst + r * kStride + c * 4, static_cast<const float*>(cache) + (there ? at + c * 4 : 0), there);
            }
            cp_commit();
        };

        // the rows
        {
            const int i = tid & (kRows - 1);
            const Row row = row_at<kRows>(a, w.r, kvh, w.rb, i);
            const float* q = static_cast<const float*>(a.q) + static_cast<long long>(row.token) * a.q_stride + static_cast<long long>(row.head) * a.dh;
#pragma unroll 4
            for (int c = tid / kRows; c < kCpr; c += kThreads / kRows)
                *reinterpret_cast<float4*>(sm.q + i * kStride + c * 4) =
                    row.there && c * 4 < a.dh ? *reinterpret_cast<const float4*>(q + c * 4) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        }
        int sees[8];
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            const Row row = row_at<kRows>(a, w.r, kvh, w.rb, ty * 8 + r);
            sees[r] = row.kept ? row.sees : 0;
        }
        // every row sees what the item's first token sees
        const int all_see = w.r.len - w.r.n + w.rb * kRows / a.G + 1;
        if (nt > 0) {
            places(0);
            places(1);
            __syncthreads();
            fetch(sm.k, a.K, 0);
            fetch(sm.v, a.V, 0);
        } else {
            __syncthreads();
        }

        float o[8][V * 4], m[8], l[8];
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            m[r] = -INFINITY;
            l[r] = 0.0f;
#pragma unroll
            for (int j = 0; j < V * 4; ++j) o[r][j] = 0.0f;
        }
        for (int t = 0; t < nt; ++t) {
            cp_wait<1>();
            __syncthreads();
            float sc[8][4] = {};
#pragma unroll 2
            for (int d = 0; d < DP; d += 4) {
                float4 k[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) k[j] = *reinterpret_cast<const float4*>(sm.k + (tx + 16 * j) * kStride + d);
#pragma unroll
                for (int r = 0; r < 8; ++r) {
                    const float4 q = *reinterpret_cast<const float4*>(sm.q + (ty * 8 + r) * kStride + d);
#pragma unroll
                    for (int j = 0; j < 4; ++j) sc[r][j] = fmaf(q.x, k[j].x, fmaf(q.y, k[j].y, fmaf(q.z, k[j].z, fmaf(q.w, k[j].w, sc[r][j]))));
                }
            }
            const int p0 = (w.t0 + t) * kTile;
            bool there[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) there[j] = sm.row[t & 1][tx + 16 * j] >= 0;
            __syncthreads();
            if (t + 1 < nt) fetch(sm.k, a.K, t + 1);
            else cp_commit();
#pragma unroll
            for (int r = 0; r < 8; ++r) {
                float mx = m[r];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    sc[r][j] = there[j] && p0 + tx + 16 * j < sees[r] ? sc[r][j] * a.scale_log2 : -INFINITY;
                    mx = fmaxf(mx, sc[r][j]);
                }
#pragma unroll
                for (int d = 1; d < 16; d <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
                const float base = mx == -INFINITY ? 0.0f : mx, g = pow2(m[r] - base);
                m[r] = mx;
                float sum = 0.0f;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float e = pow2(sc[r][j] - base);
                    sum += e;
                    sm.w[(ty * 8 + r) * kWeights + tx + 16 * j] = e;
                }
                l[r] = fmaf(l[r], g, sum);       // of this lane's keys; the lanes meet at the end
#pragma unroll
                for (int j = 0; j < V * 4; ++j) o[r][j] *= g;
            }
            cp_wait<1>();
            __syncthreads();
            const bool whole = p0 + kTile <= all_see;   // else: what a row does not see meets nothing, as its value may be infinite or NaN
#pragma unroll 1
            for (int k0 = 0; k0 < kTile; k0 += 4) {
                float4 v[4][V];
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int g = 0; g < V; ++g) v[e][g] = *reinterpret_cast<const float4*>(sm.v + (k0 + e) * kStride + tx * 4 + 64 * g);
#pragma unroll
                for (int r = 0; r < 8; ++r) {
                    const float4 e4 = *reinterpret_cast<const float4*>(sm.w + (ty * 8 + r) * kWeights + k0);
                    const float e[4] = {e4.x, e4.y, e4.z, e4.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if (!whole && p0 + k0 + i >= sees[r]) continue;
#pragma unroll
                        for (int g = 0; g < V; ++g) {
                            o[r][4 * g] = fmaf(e[i], v[i][g].x, o[r][4 * g]);
                            o[r][4 * g + 1] = fmaf(e[i], v[i][g].y, o[r][4 * g + 1]);
                            o[r][4 * g + 2] = fmaf(e[i], v[i][g].z, o[r][4 * g + 2]);
                            o[r][4 * g + 3] = fmaf(e[i], v[i][g].w, o[r][4 * g + 3]);
                        }
                    }
                }
            }
            __syncthreads();
            if (t + 1 < nt) fetch(sm.v, a.V, t + 1);
            else cp_commit();
            if (t + 2 < nt) places(t + 2);
        }
        cp_wait<0>();

        const bool complete = w.complete();
        float* slot = w.slot(a);
#pragma unroll
        for (int r = 0; r < 8; ++r) {
#pragma unroll
            for (int d = 1; d < 16; d <<= 1) l[r] += __shfl_xor_sync(0xffffffffu, l[r], d);
            const int i = ty * 8 + r;
            if (complete) {
                const Row row = row_at<kRows>(a, w.r, kvh, w.rb, i);
                if (!row.there) continue;
                const bool some = l[r] != 0.0f && row.kept;
                const float n = some ? 1.0f / l[r] : 0.0f;
                const long long at = static_cast<long long>(row.token) * a.H + row.head;
                float* out = static_cast<float*>(a.out) + at * a.dh;
#pragma unroll
                for (int g = 0; g < V; ++g)
                    if (tx * 4 + 64 * g < a.dh)
                        *reinterpret_cast<float4*>(out + tx * 4 + 64 * g) = some ? make_float4(o[r][4 * g] * n, o[r][4 * g + 1] * n, o[r][4 * g + 2] * n, o[r][4 * g + 3] * n)
                                                                                 : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                if (tx == 0 && a.lse) a.lse[at] = some ? (m[r] + log2f(l[r])) * kLn2 : -INFINITY;
            } else if (i < a.rows) {
                if (tx == 0) {
                    slot[i] = m[r];
                    slot[a.rows + i] = l[r];
                }
#pragma unroll
                for (int g = 0; g < V; ++g)
                    if (tx * 4 + 64 * g < a.dh)
                        reinterpret_cast<float4*>(slot + 2 * a.rows)[(tx + 16 * g) * a.rows + i] =
                            make_float4(o[r][4 * g], o[r][4 * g + 1], o[r][4 * g + 2], o[r][4 * g + 3]);
            }
        }
        if (tid == 0 && w.opens()) a.openings[blockIdx.x] = w.opening(f.total);
        w.next(a);
        __syncthreads();
    }
    if (__any_sync(0xffffffffu, bad) && lane == 0) flag_status(a.status, HALO_DEV_BAD_INDEX);
}

template <int DP>
int blocks_of(const halo_paged_shape& sh, int n_tok, int n_seq) {
    constexpr int kFit = 227 * 1024 / static_cast<int>(sizeof(Smem<DP>) + 1024);
    return line_blocks(sh, n_tok, n_seq, kRows, kTile, kOver, kSmCount * (kFit < 4 ? kFit : 4));
}
template <typename F>
auto by_width(const halo_paged_shape& sh, F f) {
    return sh.head_dim <= 64    ? f(std::integral_constant<int, 64>())
           : sh.head_dim <= 128 ? f(std::integral_constant<int, 128>())
                                : f(std::integral_constant<int, 256>());
}

}  // namespace

size_t f32_workspace(const halo_paged_shape& sh, int n_tok, int n_seq) {
    return by_width(sh, [&](auto dp) {
        return static_cast<size_t>(blocks_of<decltype(dp)::value>(sh, n_tok, n_seq)) *
               (sizeof(Opening) + 2 * sizeof(float) * slot_floats(slot_rows(kRows, n_tok, sh), sh.head_dim));
    });
}
halo_status f32_launch(const Args& args, const halo_paged_shape& sh, void* workspace, cudaStream_t st) {
    return by_width(sh, [&](auto dp) -> halo_status {
        constexpr int DP = decltype(dp)::value;
        static bool done[64];
        if (!ensure_dynamic_smem(paged_prompt_rows_kernel<DP>, sizeof(Smem<DP>), done)) return HALO_ERR_CUDA;
        Args a = args;
        a.blocks = blocks_of<DP>(sh, a.n_tok, a.n_seq);
        a.rows = slot_rows(kRows, a.n_tok, sh);
        a.slot = slot_floats(a.rows, a.dh);
        a.lower = 0.0f;
        a.raise = 1.0f;
        a.openings = static_cast<Opening*>(workspace);
        a.ws = reinterpret_cast<float*>(a.openings + a.blocks);
        const halo_status rc = launch_chained(paged_prompt_rows_kernel<DP>, a.blocks, kThreads, sizeof(Smem<DP>), st, a);
        return rc != HALO_OK ? rc : launch_join<float, kRows>(a, st);
    });
}

}  // namespace prompt
}  // namespace halo
