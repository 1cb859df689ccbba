// halo_paged_mha: attention of one new token per sequence over a paged K/V cache, split over the cache's length and
// joined.  HBM-bound: every K and V row is read once, 4 * G flops per element of it (G = query heads per K/V head).
//
// Work line.  The cache is cut into tiles of kTile positions; an item is one (sequence, K/V head, block of 16 query
// heads).  All tiles of all items, item after item, form one line of T tiles and thread block c of C takes the tiles
// [c*T/C, (c+1)*T/C): whatever the lengths are, every thread block streams the same number of tiles.  A piece that
// covers a whole item writes its output; the at most two pieces of a thread block that do not (its first and its last)
// leave (maximum, sum, weighted sum of values) in the workspace and a second kernel, resident before the first ends
// (programmatic dependent launch), joins them in line order, so results do not depend on timing.  Every thread block
// computes the line from seq_len itself; the host never reads a length.
//
// Inside a thread block each warp takes 16 positions of a tile at a time through a shared-memory ring of its own
// (cp.async, no block barrier in the loop) and keeps a running maximum and sum per query head.  Scores and weighted
// sums go through mma.sync with the query heads as the 16 rows of A: one new token makes a matrix of at most 16 rows
// that cannot fill a tcgen05 tile of 128, and the stream of K and V bounds the kernel, not the tensor pipe.
//   bf16: m16n8k16, probabilities rounded to bf16 for the second product (relative 2^-9, below the rounding of the
//         output), sums of probabilities in fp32 before that rounding.
//   fp32: m16n8k8 tf32 with both operands split into two tf32 parts, three products (hi*hi + hi*lo + lo*hi): what is
//         dropped is 2^-22 of a product.
#include <math.h>

#include "common.cuh"

namespace halo {
namespace {

constexpr int kMaxSplitRows = 16;   // query heads per item

struct PagedArgs {
    int n_seq, H, Hk, G, qblocks, dh, page_size, n_pages, max_pages;
    long long page_stride, q_stride;
    float scale_log2;
    const void* q;
    const void* K;
    const void* V;
    const int32_t* table;
    const int32_t* seq_len;
    const uint8_t* keep;
    void* out;
    float* lse;
    float* ws;
    uint32_t* status;
    int whole;   // one thread block per item: no line, no join
};

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool valid) {
    const int n = valid ? 16 : 0;   // 0: the 16 bytes are filled with zeros and src is not read
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t a) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t (&r)[4], uint32_t a) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void mma_bf16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_tf32(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t tf32_of(float x) {
    uint32_t r;
    asm("cvt.rna.tf32.f32 %0, %1;" : "=r"(r) : "f"(x));
    return r;
}
// x = hi + lo + at most 2^-22 |x|; hi is cut off, not rounded, so it never overflows.
__device__ __forceinline__ void split_tf32(float x, uint32_t& hi, uint32_t& lo) {
    hi = __float_as_uint(x) & 0xffffe000u;
    lo = tf32_of(x - __uint_as_float(hi));
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// Tile shapes per element type and padded head size.  Ring bytes per SM are what keeps HBM busy: 6.5 TB/s x ~1 us of
// latency / 148 SMs = 44 KB have to be in flight; stages x warps x thread blocks per SM below give 96 to 128 KB.
template <typename T, int DP>
struct Cfg {
    static constexpr bool kF32 = sizeof(T) == 4;
    static constexpr int kWarps = (kF32 && DP == 256) ? 2 : 4;
    static constexpr int kStages = (kF32 && DP == 256) ? 2 : 3;
    static constexpr int kTile = kWarps * 16;
    static constexpr int kRowBytes = kF32 ? (DP + 4) * 4 : DP * 2;   // fp32: rows padded by 16 bytes; bf16: swizzled
    static constexpr int kHalf = 16 * kRowBytes;                     // keys (or values) of one stage of one warp
    static constexpr int kStage = 2 * kHalf;
    static constexpr int kRing = kWarps * kStages * kStage;
    static constexpr int kQ = kF32 ? 2 * 16 * (DP + 4) * 4 : 0;      // fp32: the query rows split into two tf32 parts
    static constexpr int kMerge = kWarps * 16 * (DP + 4) * 4;        // the warps' sums meet here, over the ring
    static constexpr int kSmem = (kRing > kMerge ? kRing : kMerge) + kQ;
    static constexpr int kBlocksPerSm = kSmem <= 56 * 1024 ? 4 : kSmem <= 113 * 1024 ? 2 : 1;
    static constexpr int kSlot = 2 * 16 + 16 * DP;                   // floats of a workspace slot: maxima, sums, values
};

__device__ __forceinline__ int valid_len(const PagedArgs& a, int s, bool flag) {
    const int n = __ldg(a.seq_len + s);
    if (n < 0 || static_cast<long long>(n) > static_cast<long long>(a.max_pages) * a.page_size) {
        if (flag) flag_status(a.status, HALO_DEV_BAD_INDEX);
        return 0;
    }
    return n;
}
template <int TILE>
__device__ __forceinline__ long long tiles_of(const PagedArgs& a, int s) {
    const int n = valid_len(a, s, false);
    return n > 0 ? (n + TILE - 1) / TILE : 1;   // an empty sequence keeps one tile, which writes its zeros
}

// The line: total number of tiles of one head's sequences (times items per sequence = T), and the sequence in which
// line position x(T) falls.  All threads of the block call it.
struct LinePos {
    long long total;   // T
    long long start;   // first line position of sequence s
    int s;
};
template <int TILE, int THREADS, typename F>
__device__ __forceinline__ LinePos locate(const PagedArgs& a, F position_of, long long* sh /*[THREADS / 32 + 3]*/) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int per = (a.n_seq + THREADS - 1) / THREADS;
    const int s0 = min(tid * per, a.n_seq), s1 = min(s0 + per, a.n_seq);
    const long long items = static_cast<long long>(a.Hk) * a.qblocks;
    long long own = 0;
    for (int s = s0; s < s1; ++s) own += tiles_of<TILE>(a, s);
    long long incl = own;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long v = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += v;
    }
    if (lane == 31) sh[warp] = incl;
    __syncthreads();
    long long before = 0, total = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) {
        if (w < warp) before += sh[w];
        total += sh[w];
    }
    const long long x = position_of(total * items);
    long long at = (before + incl - own) * items;
    if (x >= at && x < at + own * items) {
        for (int s = s0; s < s1; ++s) {
            const long long n = tiles_of<TILE>(a, s) * items;
            if (x < at + n) {
                sh[THREADS / 32] = at;
                sh[THREADS / 32 + 1] = s;
                break;
            }
            at += n;
        }
    }
    __syncthreads();
    LinePos r;
    r.total = total * items;
    r.start = sh[THREADS / 32];
    r.s = static_cast<int>(sh[THREADS / 32 + 1]);
    return r;
}
__device__ __forceinline__ long long cut(long long T, int c, int C) { return T * c / C; }

__device__ __forceinline__ bool head_kept(const PagedArgs& a, int h) { return !a.keep || a.keep[h] != 0; }

template <typename T>
__device__ __forceinline__ void write_head(const PagedArgs& a, int s, int h, int j, float v) {
    static_cast<T*>(a.out)[(static_cast<long long>(s) * a.H + h) * a.dh + j] = from_float<T>(v);
}

template <typename T, int DP>
__global__ void __launch_bounds__(Cfg<T, DP>::kWarps * 32, Cfg<T, DP>::kBlocksPerSm)
paged_mha_kernel(const __grid_constant__ PagedArgs a) {
    using C_ = Cfg<T, DP>;
    constexpr bool kF32 = C_::kF32;
    constexpr int kThreads = C_::kWarps * 32;
    constexpr int kE = kF32 ? 4 : 8;              // elements per 16 bytes
    constexpr int kCpr = DP / kE;                 // 16-byte chunks per padded row
    constexpr int kRowsPer = 32 / (kCpr < 32 ? kCpr : 32);   // rows a warp copies per instruction
    constexpr int kChunkIters = kCpr / 32 > 0 ? kCpr / 32 : 1;   // instructions per row where a row is longer
    constexpr int NT = DP / 8;                    // 8-wide column tiles of the output
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ long long scan[C_::kWarps + 3];
    __shared__ float wm[C_::kWarps][16], wl[C_::kWarps][16];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int items = a.Hk * a.qblocks;

    asm volatile("griddepcontrol.launch_dependents;");
    long long x, x_end, start;
    int s;
    if (a.whole) {
        s = blockIdx.x / items;
        const long long t = tiles_of<C_::kTile>(a, s);
        start = 0;                                 // line positions relative to the sequence
        x = (blockIdx.x % items) * t;
        x_end = x + t;
    } else {
        const LinePos p = locate<C_::kTile, kThreads>(
            a, [&](long long T_) { return cut(T_, blockIdx.x, gridDim.x); }, scan);
        x = cut(p.total, blockIdx.x, gridDim.x);
        x_end = cut(p.total, blockIdx.x + 1, gridDim.x);
        start = p.start;
        s = p.s;
    }
    if (x >= x_end) return;
    const long long x_first = x;

    unsigned char* ring = smem + warp * (C_::kStages * C_::kStage);
    const uint32_t ring_a = smem_addr(ring);
    if (a.dh != DP) {   // columns behind the head's own stay zero: they meet zeros of q and give unused output columns
        for (int i = tid * 16; i < C_::kRing; i += kThreads * 16) *reinterpret_cast<uint4*>(smem + i) = make_uint4(0, 0, 0, 0);
        __syncthreads();
    }
    const int g = lane >> 2, t4 = lane & 3;

    while (x < x_end) {
        // ---- the piece: sequence s, item hi, tiles [t0, t1) of nt -------------------------------------------------
        const int len_all = valid_len(a, s, x == x_first && tid == 0);
        const long long nt = len_all > 0 ? (len_all + C_::kTile - 1) / C_::kTile : 1;
        const int hi = static_cast<int>((x - start) / nt);
        const int t0 = static_cast<int>((x - start) - hi * nt);
        const int t1 = static_cast<int>(min(nt, t0 + (x_end - x)));
        const int kvh = hi / a.qblocks, r0 = (hi % a.qblocks) * 16;
        const int rows = min(16, a.G - r0), h0 = kvh * a.G + r0;
        bool any = false;
        for (int r = 0; r < rows; ++r) any |= head_kept(a, h0 + r);
        const int len = any ? len_all : 0;

        // ---- query rows -------------------------------------------------------------------------------------------
        uint32_t qf[kF32 ? 1 : DP / 16][4];
        float* q_hi = reinterpret_cast<float*>(smem + C_::kSmem - C_::kQ);
        float* q_lo = q_hi + 16 * (DP + 4);
        const T* qrow = static_cast<const T*>(a.q) + static_cast<long long>(s) * a.q_stride + static_cast<long long>(h0) * a.dh;
        if constexpr (!kF32) {
#pragma unroll
            for (int k = 0; k < DP / 16; ++k)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int r = g + (j & 1) * 8, c = k * 16 + (j >> 1) * 8 + t4 * 2;
                    qf[k][j] = (r < rows && c < a.dh)
                                   ? __ldg(reinterpret_cast<const uint32_t*>(qrow + static_cast<long long>(r) * a.dh + c)) : 0u;
                }
        } else {
            for (int i = tid; i < 16 * DP; i += kThreads) {
                const int r = i / DP, c = i % DP;
                uint32_t hi_, lo_;
                split_tf32((r < rows && c < a.dh) ? __ldg(reinterpret_cast<const float*>(qrow) + static_cast<long long>(r) * a.dh + c) : 0.0f,
                           hi_, lo_);
                q_hi[r * (DP + 4) + c] = __uint_as_float(hi_);
                q_lo[r * (DP + 4) + c] = __uint_as_float(lo_);
            }
            __syncthreads();
        }

        float o[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int j = 0; j < 4; ++j) o[n][j] = 0.0f;
        float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.0f, l1 = 0.0f;

        // ---- this warp's runs of 16 positions: first position (t0 * kWarps + warp) * 16, every kTile ------------
        const int p_begin = t0 * C_::kTile + warp * 16;
        const int p_end = min(len, t1 * C_::kTile);
        const int n_run = p_end > p_begin ? (p_end - p_begin + C_::kTile - 1) / C_::kTile : 0;
        const int32_t* trow = a.table + static_cast<long long>(s) * a.max_pages;
        // page of position p + lane % 16, -1 behind the end
        auto page_at = [&](int run) {
            const int p = p_begin + run * C_::kTile + (lane & 15);
            return run < n_run && p < p_end ? __ldg(trow + p / a.page_size) : -1;
        };
        uint32_t masks[C_::kStages];
#pragma unroll
        for (int i = 0; i < C_::kStages; ++i) masks[i] = 0;
        int page_next = page_at(0);
        bool bad = false;
        auto issue = [&](int run) -> uint32_t {   // starts the copies of a run; returns its mask of present positions
            uint32_t mask = 0;
            if (run < n_run) {
                const int p = p_begin + run * C_::kTile + (lane & 15);
                const int page = page_next;
                const bool in = p < p_end, ok = in && page >= 0 && page < a.n_pages;
                bad |= in && !ok;
                mask = __ballot_sync(0xffffffffu, ok) & 0xffffu;
                const long long off = ok ? static_cast<long long>(page) * a.page_stride +
                                               (static_cast<long long>(kvh) * a.page_size + p % a.page_size) * a.dh
                                         : 0;
                const uint32_t st = ring_a + (run % C_::kStages) * C_::kStage;
#pragma unroll
                for (int it = 0; it < 16 / kRowsPer; ++it) {
                    const int r = it * kRowsPer + (kCpr < 32 ? lane / kCpr : 0);
                    const long long ro = __shfl_sync(0xffffffffu, off, r);
                    const bool have = (mask >> r) & 1u;
#pragma unroll
                    for (int ci = 0; ci < kChunkIters; ++ci) {
                        const int c = (lane % (kCpr < 32 ? kCpr : 32)) + ci * 32;
                        if (c * kE < a.dh) {
                            const uint32_t d = st + r * C_::kRowBytes + (kF32 ? c * 16 : ((c & ~7) | ((c ^ r) & 7)) * 16);
                            cp_async16(d, static_cast<const T*>(a.K) + ro + c * kE, have);
                            cp_async16(d + C_::kHalf, static_cast<const T*>(a.V) + ro + c * kE, have);
                        }
                    }
                }
            }
            page_next = page_at(run + 1);
            cp_commit();
            return mask;
        };
#pragma unroll
        for (int i = 0; i < C_::kStages - 1; ++i) masks[i] = issue(i);

        for (int run = 0; run < n_run; ++run) {
            masks[C_::kStages - 1] = issue(run + C_::kStages - 1);
            cp_wait<C_::kStages - 1>();
            __syncwarp();
            const uint32_t mask = masks[0];
#pragma unroll
            for (int i = 0; i + 1 < C_::kStages; ++i) masks[i] = masks[i + 1];
            const uint32_t st = ring_a + (run % C_::kStages) * C_::kStage;
            // scores of 16 heads x 16 positions
            float sc[2][4] = {};
            if constexpr (!kF32) {
                float sc2[2][4] = {};   // a second chain: products of odd steps
                const int key = (lane >> 4) * 8 + (lane & 7), half = (lane >> 3) & 1;
#pragma unroll
                for (int k = 0; k < DP / 16; ++k) {
                    const int c = k * 2 + half;
                    uint32_t b[4];
                    ldsm4(b, st + key * C_::kRowBytes + ((c & ~7) | ((c ^ key) & 7)) * 16);
                    mma_bf16(k & 1 ? sc2[0] : sc[0], qf[k], b[0], b[1]);
                    mma_bf16(k & 1 ? sc2[1] : sc[1], qf[k], b[2], b[3]);
                }
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int j = 0; j < 4; ++j) sc[n][j] += sc2[n][j];
            } else {
                const float* kp = reinterpret_cast<const float*>(ring + (run % C_::kStages) * C_::kStage);
                for (int k = 0; k < DP / 8; ++k) {
                    uint32_t ah[4], al[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int at = (g + (j & 1) * 8) * (DP + 4) + k * 8 + (j >> 1) * 4 + t4;
                        ah[j] = __float_as_uint(q_hi[at]);
                        al[j] = __float_as_uint(q_lo[at]);
                    }
#pragma unroll
                    for (int n = 0; n < 2; ++n) {
                        uint32_t bh[2], bl[2];
#pragma unroll
                        for (int j = 0; j < 2; ++j)
                            split_tf32(kp[(n * 8 + g) * (DP + 4) + k * 8 + j * 4 + t4], bh[j], bl[j]);
                        mma_tf32(sc[n], al, bh[0], bh[1]);
                        mma_tf32(sc[n], ah, bl[0], bl[1]);
                        mma_tf32(sc[n], ah, bh[0], bh[1]);
                    }
                }
            }
            // running softmax; a lane holds rows g and g + 8, positions 2 * t4 + {0, 1} and 8 more
            float mx0 = m0, mx1 = m1;
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int key = n * 8 + t4 * 2 + (j & 1);
                    sc[n][j] = (mask >> key) & 1u ? sc[n][j] * a.scale_log2 : -INFINITY;
                    if (j < 2) mx0 = fmaxf(mx0, sc[n][j]); else mx1 = fmaxf(mx1, sc[n][j]);
                }
#pragma unroll
            for (int d = 1; d < 4; d <<= 1) {
                mx0 = fmaxf(mx0, __shfl_xor_sync(0xffffffffu, mx0, d));
                mx1 = fmaxf(mx1, __shfl_xor_sync(0xffffffffu, mx1, d));
            }
            const float b0 = mx0 == -INFINITY ? 0.0f : mx0, b1 = mx1 == -INFINITY ? 0.0f : mx1;
            const float f0 = exp2f(m0 - b0), f1 = exp2f(m1 - b1);
            if (__any_sync(0xffffffffu, m0 != mx0 || m1 != mx1)) {
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    o[n][0] *= f0; o[n][1] *= f0;
                    o[n][2] *= f1; o[n][3] *= f1;
                }
            }
            m0 = mx0; m1 = mx1;
            float a0 = 0.0f, a1 = 0.0f;
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    sc[n][j] = exp2f(sc[n][j] - (j < 2 ? b0 : b1));
                    if (j < 2) a0 += sc[n][j]; else a1 += sc[n][j];
                }
            l0 = fmaf(l0, f0, a0);
            l1 = fmaf(l1, f1, a1);
            // weighted sum of the values
            if constexpr (!kF32) {
                const uint32_t pa[4] = {pack_bf16(sc[0][0], sc[0][1]), pack_bf16(sc[0][2], sc[0][3]),
                                        pack_bf16(sc[1][0], sc[1][1]), pack_bf16(sc[1][2], sc[1][3])};
                const int key = ((lane >> 3) & 1) * 8 + (lane & 7), half = lane >> 4;
#pragma unroll
                for (int n = 0; n < NT; n += 2) {
                    const int c = n + half;
                    uint32_t b[4];
                    ldsm4t(b, st + C_::kHalf + key * C_::kRowBytes + ((c & ~7) | ((c ^ key) & 7)) * 16);
                    mma_bf16(o[n], pa, b[0], b[1]);
                    mma_bf16(o[n + 1], pa, b[2], b[3]);
                }
            } else {
                // positions 2 * t4 and 2 * t4 + 1 of an 8-run stand at k = t4 and t4 + 4, in A and in B alike
                const float* vp = reinterpret_cast<const float*>(ring + (run % C_::kStages) * C_::kStage + C_::kHalf);
                uint32_t ph[2][4], pl[2][4];
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    split_tf32(sc[n][0], ph[n][0], pl[n][0]);
                    split_tf32(sc[n][2], ph[n][1], pl[n][1]);
                    split_tf32(sc[n][1], ph[n][2], pl[n][2]);
                    split_tf32(sc[n][3], ph[n][3], pl[n][3]);
                }
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int kk = 0; kk < 2; ++kk) {
                        uint32_t bh[2], bl[2];
#pragma unroll
                        for (int j = 0; j < 2; ++j)
                            split_tf32(vp[(kk * 8 + t4 * 2 + j) * (DP + 4) + n * 8 + g], bh[j], bl[j]);
                        mma_tf32(o[n], pl[kk], bh[0], bh[1]);
                        mma_tf32(o[n], ph[kk], bl[0], bl[1]);
                        mma_tf32(o[n], ph[kk], bh[0], bh[1]);
                    }
            }
            __syncwarp();   // the stage is free for the copies that the next round starts
        }
        cp_wait<0>();
        if (__any_sync(0xffffffffu, bad) && lane == 0) flag_status(a.status, HALO_DEV_BAD_INDEX);

        // ---- the warps meet ---------------------------------------------------------------------------------------
#pragma unroll
        for (int d = 1; d < 4; d <<= 1) {
            l0 += __shfl_xor_sync(0xffffffffu, l0, d);
            l1 += __shfl_xor_sync(0xffffffffu, l1, d);
        }
        __syncthreads();   // every ring is drained: the sums go over it
        float* mg = reinterpret_cast<float*>(smem);
        if (t4 == 0) {
            wm[warp][g] = m0; wm[warp][g + 8] = m1;
            wl[warp][g] = l0; wl[warp][g + 8] = l1;
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float* p0 = mg + (warp * 16 + g) * (DP + 4) + n * 8 + t4 * 2;
            if (g < rows) { p0[0] = o[n][0]; p0[1] = o[n][1]; }
            if (g + 8 < rows) { p0[8 * (DP + 4)] = o[n][2]; p0[8 * (DP + 4) + 1] = o[n][3]; }
        }
        __syncthreads();
        const bool complete = t0 == 0 && t1 == nt;
        float* slot = complete ? nullptr : a.ws + (static_cast<long long>(blockIdx.x) * 2 + (x == x_first ? 0 : 1)) * C_::kSlot;
        for (int i = tid; i < rows * a.dh; i += kThreads) {
            const int r = i / a.dh, j = i % a.dh;
            float M = wm[0][r];
#pragma unroll
            for (int w = 1; w < C_::kWarps; ++w) M = fmaxf(M, wm[w][r]);
            const float base = M == -INFINITY ? 0.0f : M;
            float L = 0.0f, v = 0.0f;
#pragma unroll
            for (int w = 0; w < C_::kWarps; ++w) {
                const float f = exp2f(wm[w][r] - base);
                L = fmaf(wl[w][r], f, L);
                v = fmaf(mg[(w * 16 + r) * (DP + 4) + j], f, v);
            }
            if (complete) {
                const bool kept = head_kept(a, h0 + r);
                write_head<T>(a, s, h0 + r, j, L != 0.0f && kept ? v / L : 0.0f);
                if (j == 0 && a.lse)
                    a.lse[static_cast<long long>(s) * a.H + h0 + r] =
                        L != 0.0f && kept ? (M + log2f(L)) * 0.693147180559945309f : -INFINITY;
            } else {
                slot[32 + r * DP + j] = v;
                if (j == 0) { slot[r] = M; slot[16 + r] = L; }
            }
        }
        if (a.dh != DP) {   // the sums were written over the padding
            __syncthreads();
            for (int i = tid * 16; i < C_::kRing; i += kThreads * 16) *reinterpret_cast<uint4*>(smem + i) = make_uint4(0, 0, 0, 0);
        }
        __syncthreads();
        // ---- next piece -------------------------------------------------------------------------------------------
        x += t1 - t0;
        if (x - start >= nt * items) {
            start += nt * items;
            ++s;
        }
        if (x < x_end && x == start && tid == 0) (void)valid_len(a, s, true);
    }
}

// Joins the pieces of the items that were cut.  Block (c, r): the item that holds line position cut(c) strictly inside,
// if thread block c - 1 of the first kernel is the one that began it; query head r of it.
template <typename T, int DP>
__global__ void __launch_bounds__(128) paged_mha_join_kernel(const __grid_constant__ PagedArgs a, int C) {
    using C_ = Cfg<T, DP>;
    __shared__ long long scan[128 / 32 + 3];
    const int c = blockIdx.x + 1, r = blockIdx.y, tid = threadIdx.x;
    const LinePos p = locate<C_::kTile, 128>(a, [&](long long T_) { return cut(T_, c, C); }, scan);
    const long long x = cut(p.total, c, C);
    asm volatile("griddepcontrol.wait;" ::: "memory");   // in every block: this grid may not end before the first one
    const long long nt = tiles_of<C_::kTile>(a, p.s);
    const int hi = static_cast<int>((x - p.start) / nt);
    const long long first = p.start + hi * nt, end = first + nt;
    const long long prev = cut(p.total, c - 1, C);
    if (x == first || prev > first) return;   // not cut here / begun by an earlier thread block
    const int kvh = hi / a.qblocks, r0 = (hi % a.qblocks) * 16;
    if (r >= min(16, a.G - r0)) return;
    const int h = kvh * a.G + r0 + r;
    const float* head = a.ws + (static_cast<long long>(c - 1) * 2 + (prev == first ? 0 : 1)) * C_::kSlot;
    // pieces: `head`, then slot 0 of thread blocks c, c + 1, ... as long as they begin inside the item
    float M = __ldcg(head + r);
    int last = c;
    for (int k = c; k < C; ++k) {
        const long long b = cut(p.total, k, C);
        if (b >= end) break;
        last = k + 1;
        if (cut(p.total, k + 1, C) == b) continue;   // an empty range
        M = fmaxf(M, __ldcg(a.ws + static_cast<long long>(k) * 2 * C_::kSlot + r));
    }
    const float base = M == -INFINITY ? 0.0f : M;
    float f = exp2f(__ldcg(head + r) - base);
    float L = __ldcg(head + 16 + r) * f;
    float v[(DP + 127) / 128];
#pragma unroll
    for (int i = 0; i < (DP + 127) / 128; ++i) {
        const int j = tid + i * 128;
        v[i] = j < a.dh ? __ldcg(head + 32 + r * DP + j) * f : 0.0f;
    }
#pragma unroll 4
    for (int k = c; k < last; ++k) {
        if (cut(p.total, k, C) == cut(p.total, k + 1, C)) continue;
        const float* sl = a.ws + static_cast<long long>(k) * 2 * C_::kSlot;
        f = exp2f(__ldcg(sl + r) - base);
        L = fmaf(__ldcg(sl + 16 + r), f, L);
#pragma unroll
        for (int i = 0; i < (DP + 127) / 128; ++i) {
            const int j = tid + i * 128;
            if (j < a.dh) v[i] = fmaf(__ldcg(sl + 32 + r * DP + j), f, v[i]);
        }
    }
    const bool some = L != 0.0f && head_kept(a, h);
#pragma unroll
    for (int i = 0; i < (DP + 127) / 128; ++i) {
        const int j = tid + i * 128;
        if (j < a.dh) write_head<T>(a, p.s, h, j, some ? v[i] / L : 0.0f);
    }
    if (tid == 0 && a.lse)
        a.lse[static_cast<long long>(p.s) * a.H + h] = some ? (M + log2f(L)) * 0.693147180559945309f : -INFINITY;
}

// Thread blocks of the first kernel, or 0 for one per item.
struct LaunchPlan {
    int blocks, whole;
    size_t slot_floats;
};
template <typename T, int DP>
LaunchPlan plan_of(const halo_paged_shape& sh, int n_seq) {
    using C_ = Cfg<T, DP>;
    const long long cap = static_cast<long long>(sh.max_pages) * sh.page_size;
    const long long tiles = (cap + C_::kTile - 1) / C_::kTile;
    const long long items = static_cast<long long>(n_seq) * sh.n_kv_heads * ((sh.n_heads / sh.n_kv_heads + 15) / 16);
    const long long resident = static_cast<long long>(kSmCount) * C_::kBlocksPerSm;
    LaunchPlan p;
    p.slot_floats = C_::kSlot;
    p.whole = tiles <= 2;
    const long long want = tiles * items < resident ? tiles * items : resident;
    p.blocks = static_cast<int>(p.whole ? items : want);
    return p;
}

template <typename T, int DP>
halo_status launch(const PagedArgs& args, const LaunchPlan& p, cudaStream_t st) {
    using C_ = Cfg<T, DP>;
    static bool done[64];
    if (!ensure_dynamic_smem(paged_mha_kernel<T, DP>, C_::kSmem, done)) return HALO_ERR_CUDA;
    PagedArgs a = args;
    a.whole = p.whole;
    paged_mha_kernel<T, DP><<<p.blocks, C_::kWarps * 32, C_::kSmem, st>>>(a);
    HALO_CHECK_LAUNCH();
    if (p.whole || p.blocks < 2) return HALO_OK;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(p.blocks - 1, a.G < 16 ? a.G : 16);
    cfg.blockDim = dim3(128);
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cuda_status(cudaLaunchKernelEx(&cfg, paged_mha_join_kernel<T, DP>, a, p.blocks));
}

template <typename F>
auto by_type(const halo_paged_shape& sh, F f) {
    const int dp = sh.head_dim <= 64 ? 64 : sh.head_dim <= 128 ? 128 : 256;
    if (sh.dtype == HALO_BF16) {
        if (dp == 64) return f(__nv_bfloat16(), std::integral_constant<int, 64>());
        if (dp == 128) return f(__nv_bfloat16(), std::integral_constant<int, 128>());
        return f(__nv_bfloat16(), std::integral_constant<int, 256>());
    }
    if (dp == 64) return f(float(), std::integral_constant<int, 64>());
    if (dp == 128) return f(float(), std::integral_constant<int, 128>());
    return f(float(), std::integral_constant<int, 256>());
}

LaunchPlan plan_for(const halo_paged_shape& sh, int n_seq) {
    return by_type(sh, [&](auto t, auto dp) { return plan_of<decltype(t), decltype(dp)::value>(sh, n_seq); });
}

}  // namespace

halo_status check_paged_shape(const halo_paged_shape* s) {
    if (!s) return HALO_ERR_ARG;
    if (s->dtype != HALO_F32 && s->dtype != HALO_BF16) return HALO_ERR_DTYPE;
    if (s->n_heads <= 0 || s->n_kv_heads <= 0 || s->n_heads > HALO_MAX_GROUPS || s->n_heads % s->n_kv_heads != 0)
        return HALO_ERR_SHAPE;
    if (s->head_dim <= 0 || s->head_dim % 16 != 0 || s->head_dim > 256) return HALO_ERR_SHAPE;
    if (s->page_size <= 0 || s->n_pages <= 0 || s->max_pages <= 0) return HALO_ERR_SHAPE;
    if (static_cast<long long>(s->max_pages) * s->page_size > 0x7fffff00ll) return HALO_ERR_SHAPE;
    const long long dense = static_cast<long long>(s->n_kv_heads) * s->page_size * s->head_dim;
    if (s->page_stride != 0 && (s->page_stride < dense || s->page_stride % 8 != 0)) return HALO_ERR_SHAPE;
    return HALO_OK;
}
long long paged_stride(const halo_paged_shape& s) {
    return s.page_stride ? s.page_stride : static_cast<long long>(s.n_kv_heads) * s.page_size * s.head_dim;
}

}  // namespace halo

using namespace halo;

extern "C" size_t halo_paged_mha_workspace_bytes(const halo_paged_shape* shape, int n_seq) {
    if (check_paged_shape(shape) != HALO_OK || n_seq <= 0 || n_seq > HALO_MAX_SEQUENCES) return 0;
    const LaunchPlan p = plan_for(*shape, n_seq);
    return p.whole || p.blocks < 2 ? 0 : sizeof(float) * 2 * p.slot_floats * static_cast<size_t>(p.blocks);
}

extern "C" halo_status halo_paged_mha(const halo_paged_shape* shape, int n_seq, const void* q, long long q_stride,
                                      const void* K_cache, const void* V_cache, const int32_t* block_table,
                                      const int32_t* seq_len, const uint8_t* keep, float scale, void* out, float* lse,
                                      void* workspace, size_t workspace_bytes, uint32_t* dev_status, void* stream) {
    const halo_status rc = check_paged_shape(shape);
    if (rc != HALO_OK) return rc;
    if (!q || !K_cache || !V_cache || !block_table || !seq_len || !out) return HALO_ERR_ARG;
    if (!isfinite(scale)) return HALO_ERR_ARG;
    if (n_seq <= 0 || n_seq > HALO_MAX_SEQUENCES) return HALO_ERR_SHAPE;
    const int elem = shape->dtype == HALO_F32 ? 4 : 2;
    const long long row = static_cast<long long>(shape->n_heads) * shape->head_dim;
    if (q_stride < row) return HALO_ERR_SHAPE;
    if (!aligned16(q) || !aligned16(K_cache) || !aligned16(V_cache) || !aligned16(out) || q_stride * elem % 16 != 0)
        return HALO_ERR_ALIGN;
    const size_t need = halo_paged_mha_workspace_bytes(shape, n_seq);
    if (need > 0 && (!workspace || workspace_bytes < need)) return HALO_ERR_WORKSPACE;
    if (need > 0 && !aligned16(workspace)) return HALO_ERR_ALIGN;
    PagedArgs a = {};
    a.n_seq = n_seq;
    a.H = shape->n_heads;
    a.Hk = shape->n_kv_heads;
    a.G = a.H / a.Hk;
    a.qblocks = (a.G + kMaxSplitRows - 1) / kMaxSplitRows;
    a.dh = shape->head_dim;
    a.page_size = shape->page_size;
    a.n_pages = shape->n_pages;
    a.max_pages = shape->max_pages;
    a.page_stride = paged_stride(*shape);
    a.q_stride = q_stride;
    a.scale_log2 = scale * 1.44269504088896340736f;
    a.q = q;
    a.K = K_cache;
    a.V = V_cache;
    a.table = block_table;
    a.seq_len = seq_len;
    a.keep = keep;
    a.out = out;
    a.lse = lse;
    a.ws = static_cast<float*>(workspace);
    a.status = dev_status;
    const LaunchPlan p = plan_for(*shape, n_seq);
    return by_type(*shape, [&](auto t, auto dp) {
        return launch<decltype(t), decltype(dp)::value>(a, p, static_cast<cudaStream_t>(stream));
    });
}
