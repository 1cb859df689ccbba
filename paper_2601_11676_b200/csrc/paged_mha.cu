// halo_paged_mha: attention of one new token per sequence over a paged K/V cache, split over the cache's length and
// joined.  HBM-bound: every K and V row is read once, 4 * G flops per element of it (G = query heads per K/V head).
//
// Work line.  The cache is cut into tiles of 16 positions per warp; an item is one (sequence, K/V head, block of 16
// query heads; fp32: of 4).  All tiles of all items, item after item, form one line of T tiles and thread block c of C (at most T)
// takes the tiles [c*T/C, (c+1)*T/C): whatever the lengths are, every thread block streams the same number of tiles.  A
// piece that covers a whole item writes its output; the at most two pieces of a range that do not (its first and its
// last) leave (maximum, sum, weighted sum of values) in the workspace and a second kernel, launched before the first
// ends (programmatic dependent launch), joins them in line order, so results do not depend on timing.  Every thread
// block computes the line from seq_len itself; the host never reads a length.
//
// The warps of a thread block take 16 positions of a tile each, with a shared-memory ring (cp.async), a running maximum
// and a running sum per query head of their own; they meet once per piece.  Copies run ahead across pieces, so that a
// short sequence's first rows are on their way while the one before it is still being summed.
//   bf16: scores and weighted sums through mma.sync m16n8k16 with the query heads as the 16 rows of A: one new token
//     makes a matrix of at most 16 rows that cannot fill a tcgen05 tile of 128, and the stream of K and V bounds the
//     kernel, not the tensor pipe.  A weight meets the values as two bf16 numbers, its upper bits and what they leave
//     (together 2^-15 of it): one of them alone would be as far off as the output's own rounding.  With up to 8 heads
//     the second numbers take the rows of A that are otherwise empty and cost no product of their own (64 sequences of up to
//     4096 positions 92.7 us with one number, 93.1 with two; 128 of up to 300 positions, 32 / 32 heads, 96 and 99; 16 heads on
//     one, a sequence of 131071 29.0 and 29.8).
//   fp32: fused multiply-adds, two lanes per position for the scores, a column per lane for the weighted sums.
//   8-bit rows (halo_paged_mha_f8): mma.sync on fp16, keys and values as the 16 rows of A, heads as the 8 columns of B; codes are fp16
//     numbers exactly (one conversion for two of them), so no product is rounded, and a lane's codes decide the order of the
//     elements, which the queries' registers follow.
//     Queries come as fp16, a row times the power of two that brings its largest element to 2^14: its smallest step is 2^-24 there, so
//     that their 8 bits fit from 2^-17, 2^-31 of the largest, on, and smaller elements are off by 2^-25, 2^-39 of the largest, at most.
//     A position's power of two of the keys multiplies its scores; that of the values its weights, relative to the largest so far.  Weights are relative to a reference that a score may pass by 2^6 before it
//     moves, and rounded to fp16 once, times 2^9 (off by at most 2^-11 of themselves, an eighth of what the output's own
//     rounding is; those below 2^-23 lose bits, 2^-34 at most).
//
// bf16, 32 / 8 heads of 128, both kernels: one sequence of 131071 positions 91 us (537 MB: 5.9 TB/s; HBM, and the join
// behind it), 64 sequences of up to 4096 positions 93 to 95 us (besides, a piece's start and meeting); one sequence of 700
// positions, 32 / 4 heads of 64: 6.3 us (launch, one chain of loads, a cluster's meeting), 8.5 under a table of 131072
// positions (the line: the plan goes by the table's width); fp32, 7 sequences of up to 1500 positions, 8 / 8 heads of 64:
// 9.3 us (the same chain, 18 MB).
// 8-bit rows: the one of 131071 56 to 58 us (271 MB: 4.8 TB/s), the 64 sequences 64, the one of 700 6.8.  The conversions keep them off
// HBM's rate: 436 instructions of a warp to 16 positions, two a clock and SM.
#include <cooperative_groups.h>
#include <math.h>

#include <type_traits>

#include "eight.cuh"

namespace halo {
halo_status check_eight(const halo_paged_shape& s, const void* K_scale, const void* V_scale);

namespace {

// Query heads per item, at most.  bf16: the rows of an mma.  fp32: more rows per warp would leave few warps per SM that take
// long over a run; the cache is read once per four heads instead, from L2 but for the first (64 sequences of up to 1000
// positions, 8 heads of 128 on one: 46 us with 16 rows, 25; one of 29000, 16 heads of 256 on one: 92 and 50; with the cache
// not in L2 when the call begins 29 and 54).
__host__ __device__ constexpr int item_rows(bool f32) { return f32 ? 4 : 16; }

// What the join has to know of a range whose last piece begins an item that it does not end; in front of the slots, at the
// start of a workspace that the caller aligns to 16 bytes and no more.
struct __align__(16) Cut {
    int opens, s, hi, rest;   // rest: tiles of the item behind the range
    long long total;          // T
    int fills, unused;        // the item's first piece is the whole range
};
static_assert(alignof(Cut) == 16 && sizeof(Cut) == 32, "two 16-byte words, anywhere in a workspace");

// Element types: of queries and outputs, and of the caches' rows.
struct Eight {};
template <typename T> struct Kind {
    using Io = T;
    using Row = T;
};
template <> struct Kind<Eight> {
    using Io = __nv_bfloat16;
    using Row = uint8_t;
};

struct PagedArgs {
    int n_seq, H, Hk, G, qblocks, dh, page_size, page_shift, n_pages, max_pages;   // page_shift: -1 = no power of two
    int slot;    // floats of a workspace slot
    int rows;    // query heads of an item, at most
    int block;   // query heads from one item of a K/V head to the next
    int merge;   // bytes in front of the rings where the warps meet
    long long page_stride, q_stride;
    float scale_log2;
    float raise;   // a part's sum of weights is times 1 / raise: 8-bit rows
    const void* q;
    const void* K;
    const void* V;
    const uint8_t* K_scale;   // 8-bit rows
    const uint8_t* V_scale;
    const int32_t* table;
    const int32_t* seq_len;
    const uint8_t* keep;
    void* out;
    float* lse;
    Cut* cuts;   // [C], then the slots: two per range
    float* ws;
    uint32_t* status;
    int split;   // > 0: a cluster of that many thread blocks per item, no line and no join kernel
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
__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Codes 0 and 1 of a word, and 2 and 3, as fp16 numbers: exactly
__device__ __forceinline__ uint32_t low_codes(uint32_t w) {
    uint32_t r;
    asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, lo;\n\t}" : "=r"(r) : "r"(w));
    return r;
}
__device__ __forceinline__ uint32_t high_codes(uint32_t w) {
    uint32_t r;
    asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, hi;\n\t}" : "=r"(r) : "r"(w));
    return r;
}
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
    return r;
}
// An 8 x 8 matrix of 16-bit numbers, a row to four lanes, turned
__device__ __forceinline__ uint32_t turn8(uint32_t a) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(a));
    return r;
}
// 2^n for n <= 127, exactly; 0 below 2^-126
__device__ __forceinline__ float power(int n) { return n < -126 ? 0.0f : eight_power(n); }
// 2^x, results below 2^-126 as 0
__device__ __forceinline__ float pow2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// A weight p of at most 1 as two bf16 numbers, neither negative: its upper 16 bits, and the rest rounded.  The rest is kept
// above 2^-126 (weights are relative to the largest, 1, and smaller ones count as 0), so that a value of infinity meets two
// positive factors where the weight is positive, and not the zero that the rest of a power of two would be.
__device__ __forceinline__ uint32_t upper_bf16(float a, float b) {
    return __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x7632);
}
__device__ __forceinline__ float rest_of(float p) { return fmaxf(p - __uint_as_float(__float_as_uint(p) & 0xffff0000u), 0x1p-126f); }
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
}

constexpr int kRun = 16;            // positions of a tile that one warp takes
constexpr float kLn2 = 0.693147180559945309f;
constexpr int kSlotHead = 32;       // floats in front of a slot's values: maxima, sums
// Shapes per element type, padded head size DP and padded number of query heads GR (bf16: 8 or 16 of 16 rows in use).
// Ring bytes are what keeps HBM busy: 6.5 TB/s x ~1 us of latency / 148 SMs = 44 KB have to be in flight; the shapes below hold 100 to 210 KB.
template <typename T, int DP, int GR>
struct Cfg {
    static constexpr bool kF32 = std::is_same<T, float>::value, kEight = std::is_same<T, Eight>::value;
    static constexpr int kWarps = kF32 && (DP == 256 || (DP == 128 && GR == 1)) ? 3 : 4;
    // fp32: two stages, so that two thread blocks of four warps fit an SM at head sizes up to 64, or of three at 128 with
    // one query head per K/V head.  64 sequences of up to 2000 positions, 32 / 8 heads of 64: 77 us with three stages and
    // one thread block, 59 so; 5 of up to 900, 8 / 8 heads of 128: 13.1 us with one thread block of four warps, 10.4 so.
    // 8-bit rows: the widening of codes bounds them, and more warps help more than more stages: with two and 8 heads, four thread
    // blocks of 128 columns fit an SM, with three stages three (128 sequences of up to 600 positions, 32 heads of 128: 117 us with two, 131 with three; 16
    // heads on one have registers for two thread blocks only: 64 sequences of 4000 108 us with two, 84 with three).
    static constexpr int kStages = kF32 ? 2 : kEight && GR <= 8 ? 2 : 3;
    static constexpr int kTile = kWarps * kRun;
    static constexpr int kRowBytes = kF32 ? (DP + 8) * 4 : kEight ? DP : DP * 2;   // fp32: rows padded against bank conflicts; else swizzled
    static constexpr int kHalf = kRun * kRowBytes;                   // keys (or values) of one stage
    static constexpr int kStage = 2 * kHalf;
    static constexpr int kRing = kStages * kStage;
    static constexpr int kOwn = kF32 ? GR * DP * 4 + GR * kRun * 4 : 0;   // fp32: query rows and weights of the warp
    static constexpr int kWarpBytes = kRing + kOwn;
    static constexpr int kRings = kWarps * kWarpBytes;
    static constexpr int kMergeRow = DP + 4;                         // floats
    // two warps' sums at a time, of the item's query heads
    static constexpr int merge_bytes(int rows) { return 2 * rows * kMergeRow * 4; }
    static constexpr int kMaxSmem = kRings + merge_bytes(GR);
    // an SM has 228 KB; a thread block takes its own, wm and wl, and 1 KB of the system's
    static constexpr int kFit = 228 * 1024 / (kMaxSmem + 2 * kWarps * 16 * 4 + 1024);
    static constexpr int kBlocksPerSm = kFit > 4 ? 4 : kFit;
    static_assert(kMaxSmem <= 225 * 1024 && (kWarps == 3 || kWarps == 4), "shared memory; the warps meet in two steps");
};

__device__ __forceinline__ int valid_len(const PagedArgs& a, int s, bool flag) {
    const int n = ldg_waited(a.seq_len + s);
    if (n < 0 || static_cast<long long>(n) > static_cast<long long>(a.max_pages) * a.page_size) {
        if (flag) flag_status(a.status, HALO_DEV_BAD_INDEX);
        return 0;
    }
    return n;
}
template <int TILE>
__device__ __forceinline__ int tiles_in(int len) {
    return len > 0 ? (len - 1) / TILE + 1 : 1;   // an empty sequence keeps one tile, which writes its zeros
}
template <int TILE>
__device__ __forceinline__ int tiles_of(const PagedArgs& a, int s) { return tiles_in<TILE>(valid_len(a, s, false)); }

// The line: its length T, and the sequence that holds position_of(T) (T or more: none).  All threads of the block call
// it.
struct LinePos {
    long long total;
    long long start;   // first line position of sequence s
    int s;
};
template <int TILE, int THREADS, typename F>
__device__ __forceinline__ LinePos locate(const PagedArgs& a, F position_of, long long* sh /*[THREADS / 32 + 2]*/) {
    constexpr int W = THREADS / 32;
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
    for (int w = 0; w < W; ++w) {
        if (w < warp) before += sh[w];
        total += sh[w];
    }
    const long long x = position_of(total * items);
    long long at = (before + incl - own) * items;
    if (x >= at && x < at + own * items) {
        for (int s = s0; s < s1; ++s) {
            const long long n = tiles_of<TILE>(a, s) * items;
            if (x < at + n) {
                sh[W] = at;
                sh[W + 1] = s;
                break;
            }
            at += n;
        }
    }
    __syncthreads();
    return {total * items, sh[W], static_cast<int>(sh[W + 1])};
}
// Thread blocks that have a range (none of them empty), and where the c-th range begins.
__device__ __forceinline__ int ranges(long long T, int blocks) { return T < blocks ? static_cast<int>(T) : blocks; }
__device__ __forceinline__ long long cut(long long T, int c, int C) { return T * c / C; }
// the range that holds line position x: the last c with T * c / C <= x
__device__ __forceinline__ int range_of(long long T, long long x, int C) { return static_cast<int>(((x + 1) * C - 1) / T); }

__device__ __forceinline__ bool head_kept(const PagedArgs& a, int h) { return !a.keep || a.keep[h] != 0; }

template <typename T>
__device__ __forceinline__ void write_head(const PagedArgs& a, int s, int h, int j, float v) {
    using Io = typename Kind<T>::Io;
    static_cast<Io*>(a.out)[(static_cast<long long>(s) * a.H + h) * a.dh + j] = from_float<Io>(v);
}

// The way along a range: piece after piece.
template <int TILE>
struct Walk {
    long long left;     // tiles from t0 of this piece to the end of the range
    int s, hi;          // sequence and item of it
    int len, nt;        // its valid length and tiles
    int t0, t1;         // tiles of the piece
    int reach;          // positions that take part: len, or 0 where every head of the item is lost
    __device__ __forceinline__ void item(const PagedArgs& a) {
        t1 = static_cast<int>(min(static_cast<long long>(nt), t0 + left));
        reach = len;
        if (a.keep) {
            const int first = hi % a.qblocks * a.block, h0 = hi / a.qblocks * a.G + first, n = min(a.block, a.G - first);
            bool any = false;
            for (int r = 0; r < n; ++r) any |= head_kept(a, h0 + r);
            if (!any) reach = 0;
        }
    }
    __device__ __forceinline__ void begin(const PagedArgs& a, int s_, long long at, long long n) {   // at: tiles behind the sequence's first
        s = s_;
        left = n;
        len = valid_len(a, s, false);
        nt = tiles_in<TILE>(len);
        hi = static_cast<int>(at / nt);
        t0 = static_cast<int>(at - static_cast<long long>(hi) * nt);
        item(a);
    }
    __device__ __forceinline__ void next(const PagedArgs& a) {
        left -= t1 - t0;
        if (left <= 0) return;
        t0 = 0;
        if (++hi == a.Hk * a.qblocks) {
            hi = 0;
            ++s;
            len = valid_len(a, s, false);
            nt = tiles_in<TILE>(len);
        }
        item(a);
    }
};

// Where 16-byte chunk c of row r of 8-bit rows lies in it: eight rows' same chunks fall on all banks, also where a row is 64 bytes.
template <int DP>
__device__ __forceinline__ uint32_t eight_chunk(int r, int c) {
    return (DP == 64 ? c ^ ((r >> 1) & 3) : (c & ~7) | ((c ^ r) & 7)) * 16;
}

template <typename T, int DP, int GR>
__global__ void __launch_bounds__(Cfg<T, DP, GR>::kWarps * 32, Cfg<T, DP, GR>::kBlocksPerSm)
paged_mha_kernel(const __grid_constant__ PagedArgs a) {
    using C_ = Cfg<T, DP, GR>;
    using Io = typename Kind<T>::Io;
    using Row = typename Kind<T>::Row;
    constexpr bool kF32 = C_::kF32, kEight = C_::kEight;
    constexpr int S = C_::kStages;
    constexpr int kThreads = C_::kWarps * 32;
    constexpr int kE = 16 / static_cast<int>(sizeof(Row));   // elements per 16 bytes
    constexpr int kCpr = DP / kE;                 // 16-byte chunks per padded row
    constexpr int kLanesPerRow = kCpr < 32 ? kCpr : 32;
    constexpr int kRowsPer = 32 / kLanesPerRow;   // rows a warp copies per instruction
    constexpr int kChunkIters = kCpr / kLanesPerRow;
    constexpr int NT = DP / 8;                    // bf16: 8-wide column tiles of the output
    constexpr int V = DP / 32;                    // fp32: output columns per lane
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ float wm[C_::kWarps][16], wl[C_::kWarps][16];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int items = a.Hk * a.qblocks;

    // Only the join may start early: another kernel behind this one may read before it waits.
    if (!a.split && gridDim.x > 1) asm volatile("griddepcontrol.launch_dependents;");
    chain_wait();
    Walk<C_::kTile> con, iss;     // the piece that is summed, the piece whose rows are fetched
    long long total = 0;
    if (a.split) {
        const int rank = blockIdx.x % a.split, item = blockIdx.x / a.split, s = item / items;
        const int nt = tiles_of<C_::kTile>(a, s);
        const int t0 = static_cast<int>(static_cast<long long>(nt) * rank / a.split);
        con.begin(a, s, static_cast<long long>(item % items) * nt, 0);
        con.t0 = t0;
        con.t1 = static_cast<int>(static_cast<long long>(nt) * (rank + 1) / a.split);
        con.left = con.t1 - t0;     // may be 0: the thread block still meets the others
    } else {
        const LinePos p = locate<C_::kTile, kThreads>(
            a, [&](long long t) {
                const int C = ranges(t, gridDim.x);
                return static_cast<int>(blockIdx.x) < C ? cut(t, blockIdx.x, C) : t;
            }, reinterpret_cast<long long*>(smem));   // where the warps meet later
        total = p.total;
        const int C = ranges(total, gridDim.x);
        if (static_cast<int>(blockIdx.x) >= C) return;
        const long long x = cut(total, blockIdx.x, C);
        con.begin(a, p.s, x - p.start, cut(total, blockIdx.x + 1, C) - x);
    }
    iss = con;
    const long long range = con.left;

    float* mg = reinterpret_cast<float*>(smem);       // the warps meet here
    unsigned char* ring = smem + a.merge + warp * C_::kWarpBytes;
    const uint32_t ring_a = smem_addr(ring);
    if (a.dh != DP) {   // columns behind the head's own stay zero: they meet zeros of q and give unused output columns
        for (int i = lane * 16; i < C_::kRing; i += 32 * 16) *reinterpret_cast<uint4*>(ring + i) = make_uint4(0, 0, 0, 0);
        __syncwarp();
    }

    // ---- fetching ---------------------------------------------------------------------------------------------------
    int it = iss.t0, slot_in = 0;
    const auto page_at = [&]() {   // page of this lane's position of the next run, -1 behind the end
        const int p = it * C_::kTile + warp * kRun + (lane & 15);
        if (iss.left <= 0 || p >= iss.reach) return -1;
        return ldg_waited(a.table + static_cast<long long>(iss.s) * a.max_pages + (a.page_shift >= 0 ? p >> a.page_shift : p / a.page_size));
    };
    int page_next = page_at();
    bool bad = false;
    // Pages of whole runs: a run's positions are neighbours in memory and share a page.
    const bool neighbours = a.page_size % kRun == 0;
    const int lr = lane / kLanesPerRow, lc = lane % kLanesPerRow;
    const auto put_row = [&](uint32_t st, int i, int ci, const Row* k, const Row* v, bool have) {
        const int r = i * kRowsPer + lr, c = lc + ci * 32;   // the swizzle: c ^ r, as i * kRowsPer and lr have no bit in common
        const uint32_t d = st + r * C_::kRowBytes +
                           (kF32 ? c * 16 : kEight ? eight_chunk<DP>(r, c) : ((c & ~7) | (((c ^ lr) ^ (i * kRowsPer)) & 7)) * 16);
        cp_async16(d, k, have);
        cp_async16(d + C_::kHalf, v, have);
    };
    [[maybe_unused]] uint32_t bytes[S];   // 8-bit rows: scale byte of a run's position, of its key in lanes 0 to 15, of its value behind
    const auto issue = [&]() -> uint32_t {   // starts the copies of the next run; returns its mask of present positions
        uint32_t mask = 0;
        if constexpr (kEight) bytes[S - 1] = 0;
        if (iss.left > 0) {
            const int p0 = it * C_::kTile + warp * kRun, p = p0 + (lane & 15);
            const bool in = p < iss.reach, ok = in && page_next >= 0 && page_next < a.n_pages;
            bad |= in && !ok;
            mask = __ballot_sync(0xffffffffu, ok) & 0xffffu;
            if (mask) {
                const int kvh = a.qblocks == 1 ? iss.hi : iss.hi / a.qblocks;
                const uint32_t st = ring_a + slot_in * C_::kStage;
                if constexpr (kEight) {
                    const int in_page = a.page_shift >= 0 ? p & (a.page_size - 1) : p % a.page_size;
                    if (ok) bytes[S - 1] = ldg_waited((lane < 16 ? a.K_scale : a.V_scale) + (static_cast<long long>(page_next) * a.Hk + kvh) * a.page_size + in_page);
                }
                if (neighbours) {
                    const int page = __shfl_sync(0xffffffffu, page_next, 0);   // mask: position 0 is there
                    const int in_page = a.page_shift >= 0 ? p0 & (a.page_size - 1) : p0 % a.page_size;
                    const long long off = static_cast<long long>(page) * a.page_stride +
                                          (static_cast<long long>(kvh) * a.page_size + in_page + lr) * a.dh + lc * kE;
                    const Row* k = static_cast<const Row*>(a.K) + off;
                    const Row* v = static_cast<const Row*>(a.V) + off;
                    const int step = kRowsPer * a.dh;
#pragma unroll
                    for (int i = 0; i < kRun / kRowsPer; ++i) {
#pragma unroll
                        for (int ci = 0; ci < kChunkIters; ++ci)
                            if ((lc + ci * 32) * kE < a.dh)
                                put_row(st, i, ci, k + ci * 32 * kE, v + ci * 32 * kE, (mask >> (i * kRowsPer + lr)) & 1u);
                        k += step;
                        v += step;
                    }
                } else {
                    const int in_page = a.page_shift >= 0 ? p & (a.page_size - 1) : p % a.page_size;
                    const long long off = ok ? static_cast<long long>(page_next) * a.page_stride +
                                                   (static_cast<long long>(kvh) * a.page_size + in_page) * a.dh
                                             : 0;
#pragma unroll
                    for (int i = 0; i < kRun / kRowsPer; ++i) {
                        const long long ro = __shfl_sync(0xffffffffu, off, i * kRowsPer + lr) + lc * kE;
#pragma unroll
                        for (int ci = 0; ci < kChunkIters; ++ci)
                            if ((lc + ci * 32) * kE < a.dh)
                                put_row(st, i, ci, static_cast<const Row*>(a.K) + ro + ci * 32 * kE,
                                        static_cast<const Row*>(a.V) + ro + ci * 32 * kE, (mask >> (i * kRowsPer + lr)) & 1u);
                    }
                }
            }
            if (++it == iss.t1) {
                iss.next(a);
                it = iss.t0;
            }
            page_next = page_at();
        }
        if (++slot_in == S) slot_in = 0;
        cp_commit();
        return mask;
    };
    uint32_t masks[S];
#pragma unroll
    for (int i = 0; i < S - 1; ++i) {
        masks[i] = issue();
        if constexpr (kEight) bytes[i] = bytes[S - 1];
    }

    // ---- summing ----------------------------------------------------------------------------------------------------
    const int g = lane >> 2, t4 = lane & 3;
    int slot_out = 0;
    bool first = true;
    while (con.left > 0 || (first && a.split)) {
        first = false;
        const int kvh = con.hi / a.qblocks, r0 = (con.hi % a.qblocks) * a.block;
        const int rows = min(a.block, a.G - r0), h0 = kvh * a.G + r0;
        const Io* qrow = static_cast<const Io*>(a.q) + static_cast<long long>(con.s) * a.q_stride + static_cast<long long>(h0) * a.dh;
        const bool complete = con.t0 == 0 && con.t1 == con.nt;
        float* slot = a.ws + (static_cast<long long>(blockIdx.x) * 2 + (con.left == range ? 0 : 1)) * a.slot;

        if constexpr (!kF32 && !kEight) {
            constexpr int kK = GR > 8 ? 2 : 1;    // rows of a lane: g, and g + 8 where an item has more than 8 heads
            uint32_t qf[DP / 16][4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int r = g + (j & 1) * 8;
                const bool there = (kK == 2 || !(j & 1)) && r < rows;
                const Io* q = qrow + static_cast<long long>(r) * a.dh + (j >> 1) * 8 + t4 * 2;
#pragma unroll
                for (int k = 0; k < DP / 16; ++k)
                    qf[k][j] = there && k * 16 < a.dh ? ldg_waited(reinterpret_cast<const uint32_t*>(q + k * 16)) : 0u;   // dh % 16 == 0
            }
            float o[NT][4];
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int j = 0; j < 4; ++j) o[n][j] = 0.0f;
            float m[kK], l[kK];
#pragma unroll
            for (int k = 0; k < kK; ++k) {
                m[k] = -INFINITY;
                l[k] = 0.0f;
            }

            for (int t = con.t0; t < con.t1; ++t) {
                masks[S - 1] = issue();
                cp_wait<S - 1>();
                __syncwarp();
                const uint32_t mask = masks[0];
#pragma unroll
                for (int i = 0; i + 1 < S; ++i) masks[i] = masks[i + 1];
                const uint32_t st = ring_a + slot_out * C_::kStage;
                if (++slot_out == S) slot_out = 0;
                if (mask == 0) continue;
                // scores of 16 heads x 16 positions, even and odd steps in two chains
                float sc[2][4] = {}, sc2[2][4] = {};
                {
                    const int key = (lane >> 4) * 8 + (lane & 7), half = (lane >> 3) & 1;
#pragma unroll
                    for (int k = 0; k < DP / 16; ++k) {
                        const int c = k * 2 + half;
                        uint32_t b[4];
                        ldsm4(b, st + key * C_::kRowBytes + ((c & ~7) | ((c ^ key) & 7)) * 16);
                        mma_bf16(k & 1 ? sc2[0] : sc[0], qf[k], b[0], b[1]);
                        mma_bf16(k & 1 ? sc2[1] : sc[1], qf[k], b[2], b[3]);
                    }
                }
                // running softmax; a lane holds rows g (and g + 8), positions 2 * t4 + {0, 1} and 8 more
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int j = 0; j < 2 * kK; ++j) sc[n][j] = (sc[n][j] + sc2[n][j]) * a.scale_log2;
                if (mask != 0xffffu) {
#pragma unroll
                    for (int n = 0; n < 2; ++n)
#pragma unroll
                        for (int j = 0; j < 2 * kK; ++j)
                            if (!((mask >> (n * 8 + t4 * 2 + (j & 1))) & 1u)) sc[n][j] = -INFINITY;
                }
                float f[kK];
                bool moved = false;
#pragma unroll
                for (int k = 0; k < kK; ++k) {
                    float mx = fmaxf(fmaxf(sc[0][2 * k], sc[0][2 * k + 1]), fmaxf(sc[1][2 * k], sc[1][2 * k + 1]));
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
                    mx = fmaxf(mx, m[k]);
                    const float base = mx == -INFINITY ? 0.0f : mx;
                    f[k] = pow2(m[k] - base);
                    moved |= m[k] != mx;
                    m[k] = mx;
#pragma unroll
                    for (int n = 0; n < 2; ++n)
#pragma unroll
                        for (int j = 2 * k; j < 2 * k + 2; ++j) sc[n][j] = pow2(sc[n][j] - base);
                    l[k] = fmaf(l[k], f[k], (sc[0][2 * k] + sc[0][2 * k + 1]) + (sc[1][2 * k] + sc[1][2 * k + 1]));
                }
                if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int j = 0; j < 4; ++j) o[n][j] *= f[kK == 2 ? j >> 1 : 0];
                }
                // weighted sum of the values: the weights' upper bits and their rests, these in the rows 8 to 15 of the
                // same product (up to 8 heads; o[n][2], o[n][3] are their sums) or in one of their own
                uint32_t pa[4], pr[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float* w = &sc[j >> 1][kK == 2 ? (j & 1) * 2 : 0];
                    if (kK == 2 || !(j & 1)) pa[j] = upper_bf16(w[0], w[1]);
                    if (kK == 2 || (j & 1)) (kK == 2 ? pr : pa)[j] = pack_bf16(rest_of(w[0]), rest_of(w[1]));
                }
                const int key = ((lane >> 3) & 1) * 8 + (lane & 7), half = lane >> 4;
#pragma unroll
                for (int n = 0; n < NT; n += 2) {
                    const int c = n + half;
                    uint32_t b[4];
                    ldsm4t(b, st + C_::kHalf + key * C_::kRowBytes + ((c & ~7) | ((c ^ key) & 7)) * 16);
                    mma_bf16(o[n], pa, b[0], b[1]);
                    mma_bf16(o[n + 1], pa, b[2], b[3]);
                    if constexpr (kK == 2) {
                        mma_bf16(o[n], pr, b[0], b[1]);
                        mma_bf16(o[n + 1], pr, b[2], b[3]);
                    }
                }
                __syncwarp();   // the stage is free for the copies that the next round starts
            }
            if constexpr (kK == 1) {
#pragma unroll
                for (int n = 0; n < NT; ++n) { o[n][0] += o[n][2]; o[n][1] += o[n][3]; }
            }
            // the warps meet: common maxima and sums, then the weighted sums of warps 2 and 3 go to 0 and 1, of 1 to 0
#pragma unroll
            for (int k = 0; k < kK; ++k) {
                l[k] += __shfl_xor_sync(0xffffffffu, l[k], 1);
                l[k] += __shfl_xor_sync(0xffffffffu, l[k], 2);
                if (t4 == 0) { wm[warp][g + k * 8] = m[k]; wl[warp][g + k * 8] = l[k]; }
            }
            __syncthreads();
            float M[kK], L[kK];
#pragma unroll
            for (int k = 0; k < kK; ++k) {
                const int r = g + k * 8;
                M[k] = wm[0][r];
#pragma unroll
                for (int w = 1; w < C_::kWarps; ++w) M[k] = fmaxf(M[k], wm[w][r]);
                const float base = M[k] == -INFINITY ? 0.0f : M[k];
                L[k] = 0.0f;
#pragma unroll
                for (int w = 0; w < C_::kWarps; ++w) L[k] = fmaf(wl[w][r], pow2(wm[w][r] - base), L[k]);
                const float f = pow2(m[k] - base);
#pragma unroll
                for (int n = 0; n < NT; ++n) { o[n][2 * k] *= f; o[n][2 * k + 1] *= f; }
            }
            const auto put = [&](int b) {
#pragma unroll
                for (int k = 0; k < kK; ++k)
                    if (g + k * 8 < rows) {
#pragma unroll
                        for (int n = 0; n < NT; ++n)
                            *reinterpret_cast<float2*>(mg + (b * rows + g + k * 8) * C_::kMergeRow + n * 8 + t4 * 2) =
                                make_float2(o[n][2 * k], o[n][2 * k + 1]);
                    }
            };
            const auto add = [&](int b) {
#pragma unroll
                for (int k = 0; k < kK; ++k)
                    if (g + k * 8 < rows) {
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            const float2 v = *reinterpret_cast<const float2*>(mg + (b * rows + g + k * 8) * C_::kMergeRow + n * 8 + t4 * 2);
                            o[n][2 * k] += v.x;
                            o[n][2 * k + 1] += v.y;
                        }
                    }
            };
            if (warp >= 2) put(warp - 2);
            __syncthreads();
            if (warp < 2) add(warp);
            if (warp == 1) put(1);
            __syncthreads();
            if (warp == 0) {
                add(1);
                if (a.split > 1) {
                    put(0);
#pragma unroll
                    for (int k = 0; k < kK; ++k)
                        if (t4 == 0) { wm[0][g + k * 8] = M[k]; wl[0][g + k * 8] = L[k]; }
                }
#pragma unroll
                for (int k = 0; k < kK; ++k) {
                    const int r = g + k * 8;
                    if (r >= rows || a.split > 1) continue;
                    if (complete) {
                        const bool some = L[k] != 0.0f && head_kept(a, h0 + r);
                        const long long row = static_cast<long long>(con.s) * a.H + h0 + r;
                        const float f = some ? 1.0f / L[k] : 0.0f;
                        uint32_t* out = reinterpret_cast<uint32_t*>(static_cast<Io*>(a.out) + row * a.dh);
#pragma unroll
                        for (int n = 0; n < NT; ++n)
                            if (n * 8 + t4 * 2 < a.dh) out[n * 4 + t4] = some ? pack_bf16(o[n][2 * k] * f, o[n][2 * k + 1] * f) : 0u;
                        if (t4 == 0 && a.lse) a.lse[row] = some ? (M[k] + log2f(L[k])) * kLn2 : -INFINITY;
                    } else {
                        if (t4 == 0) { slot[r] = M[k]; slot[16 + r] = L[k]; }
#pragma unroll
                        for (int n = 0; n < NT; ++n)
                            *reinterpret_cast<float2*>(slot + kSlotHead + r * DP + n * 8 + t4 * 2) = make_float2(o[n][2 * k], o[n][2 * k + 1]);
                    }
                }
            }
        } else if constexpr (kEight) {
            // Keys and values are the rows of A and the query heads the eight columns of B, so that no part of a product is
            // empty: S^T = K Q^T, O^T = V^T P^T.  A lane has scores of keys g and g + 8, heads 2 t4 and 2 t4 + 1 (of eight).
            constexpr int NB = GR / 8, NC = DP / 16;
            constexpr float kLag = 6.0f;      // powers of two that a reference may lag behind: weights up to 2^6, times 2^9, fit fp16
            uint32_t qf[NC][NB][2];
            float unit[NB][2];                // what a head's products are multiplied with
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                // head g: elements 4 t4 to 4 t4 + 3 of every 16, where a lane has the keys' codes
                const int r = b * 8 + g;
                uint2 w[NC];
                uint32_t top = 0;
#pragma unroll
                for (int k = 0; k < NC; ++k) {
                    const unsigned long long v = r < rows && k * 16 < a.dh   // dh % 16 == 0
                        ? ldg_waited(reinterpret_cast<const unsigned long long*>(qrow + static_cast<long long>(r) * a.dh + k * 16 + t4 * 4)) : 0ull;
                    w[k] = make_uint2(static_cast<uint32_t>(v), static_cast<uint32_t>(v >> 32));
                    top = max(max(top, w[k].x & 0x7fffu), (w[k].x >> 16) & 0x7fffu);
                    top = max(max(top, w[k].y & 0x7fffu), (w[k].y >> 16) & 0x7fffu);
                }
                top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
                top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
                // 2^up brings the largest element below 2^15; at least 2^-114, at most 2^120 (tiny rows stay smaller)
                const int up = min(14 + 127 - static_cast<int>(top >> 7), 120);
                const float n = eight_power(up), own = a.scale_log2 * eight_power(-up);
                unit[b][0] = __shfl_sync(0xffffffffu, own, t4 * 8);
                unit[b][1] = __shfl_sync(0xffffffffu, own, t4 * 8 + 4);
#pragma unroll
                for (int k = 0; k < NC; ++k) {
                    qf[k][b][0] = pack_f16(bf16_lo(w[k].x) * n, bf16_hi(w[k].x) * n);
                    qf[k][b][1] = pack_f16(bf16_lo(w[k].y) * n, bf16_hi(w[k].y) * n);
                }
            }
            float o[NC][NB][4], m[NB][2], l[NB][2];
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                m[b][0] = m[b][1] = -INFINITY;
                l[b][0] = l[b][1] = 0.0f;
#pragma unroll
                for (int n = 0; n < NC; ++n)
#pragma unroll
                    for (int j = 0; j < 4; ++j) o[n][b][j] = 0.0f;
            }
            int top_byte = 0;      // the largest scale byte of the values so far; o is relative to it

            for (int t = con.t0; t < con.t1; ++t) {
                masks[S - 1] = issue();
                cp_wait<S - 1>();
                __syncwarp();
                const uint32_t mask = masks[0], byte = bytes[0];
#pragma unroll
                for (int i = 0; i + 1 < S; ++i) {
                    masks[i] = masks[i + 1];
                    bytes[i] = bytes[i + 1];
                }
                const uint32_t st = ring_a + slot_out * C_::kStage;
                if (++slot_out == S) slot_out = 0;
                if (mask == 0) continue;
                const int key = ((lane >> 3) & 1) * 8 + (lane & 7), second = lane >> 4;
                float sc[NB][4] = {}, sc2[NB][4] = {};      // even and odd steps in two chains
#pragma unroll
                for (int k = 0; k < NC; k += 2) {
                    uint32_t c[4];
                    ldsm4(c, st + key * C_::kRowBytes + eight_chunk<DP>(key, k + second));
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const uint32_t x[4] = {low_codes(c[2 * e]), low_codes(c[2 * e + 1]), high_codes(c[2 * e]), high_codes(c[2 * e + 1])};
#pragma unroll
                        for (int b = 0; b < NB; ++b) mma_f16(e ? sc2[b] : sc[b], x, qf[k + e][b][0], qf[k + e][b][1]);
                    }
                }
                // lanes 0 to 15: the keys' powers of two; 16 to 31: the values', relative to the largest
                const int most = __reduce_max_sync(0xffffffffu, lane < 16 || byte == kEightNan ? 0 : static_cast<int>(byte));
                float down = 1.0f, own = eight_unit(byte);
                if (most > top_byte) {
                    down = power(top_byte - most);
                    top_byte = most;
                }
                if (lane >= 16 && byte != kEightNan) own = power(static_cast<int>(byte) - top_byte + 9);
                bool ahead = false;
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const float kf = __shfl_sync(0xffffffffu, own, k * 8 + g);
                    const bool there = mask >> (k * 8 + g) & 1u;
#pragma unroll
                    for (int b = 0; b < NB; ++b)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            float& x = sc[b][2 * k + e];
                            x = there ? (x + sc2[b][2 * k + e]) * unit[b][e] * kf : -INFINITY;
                            ahead |= x - m[b][e] > kLag;
                        }
                }
                if (__any_sync(0xffffffffu, ahead || down != 1.0f)) {      // new references
#pragma unroll
                    for (int b = 0; b < NB; ++b)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            float mx = fmaxf(fmaxf(sc[b][e], sc[b][2 + e]), m[b][e]);
#pragma unroll
                            for (int d = 4; d < 32; d <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
                            const float f = mx == -INFINITY ? 1.0f : pow2(m[b][e] - mx);
                            m[b][e] = mx;
                            l[b][e] *= f;
#pragma unroll
                            for (int n = 0; n < NC; ++n) {
                                o[n][b][e] *= f * down;
                                o[n][b][2 + e] *= f * down;
                            }
                        }
                }
                const float v0 = __shfl_sync(0xffffffffu, own, 16 + g), v1 = __shfl_sync(0xffffffffu, own, 24 + g);
                uint32_t pt[NB][2];      // weights, turned: head g, keys 2 t4 and 2 t4 + 1 (and 8 more)
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    float w[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) w[j] = pow2(sc[b][j] - (m[b][j & 1] == -INFINITY ? 0.0f : m[b][j & 1]));
                    l[b][0] += w[0] + w[2];
                    l[b][1] += w[1] + w[3];
                    pt[b][0] = turn8(pack_f16(w[0] * v0, w[1] * v0));
                    pt[b][1] = turn8(pack_f16(w[2] * v1, w[3] * v1));
                }
#pragma unroll
                for (int n = 0; n < NC; n += 2) {      // rows g of a product: columns 2 g of 16; rows g + 8: the odd ones
                    uint32_t c[4];
                    ldsm4t(c, st + C_::kHalf + key * C_::kRowBytes + eight_chunk<DP>(key, n + second));
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        // a word has two columns of two keys
                        const uint32_t k0 = low_codes(c[2 * e]), k1 = high_codes(c[2 * e]), k8 = low_codes(c[2 * e + 1]), k9 = high_codes(c[2 * e + 1]);
                        const uint32_t x[4] = {__byte_perm(k0, k1, 0x5410), __byte_perm(k0, k1, 0x7632), __byte_perm(k8, k9, 0x5410), __byte_perm(k8, k9, 0x7632)};
#pragma unroll
                        for (int b = 0; b < NB; ++b) mma_f16(o[n + e][b], x, pt[b][0], pt[b][1]);
                    }
                }
                __syncwarp();   // the stage is free for the copies that the next round starts
            }
            // The values' own size last, behind the division by the sum: weights are up to 2^6, and a sum of values times them could
            // overflow.  Then the warps meet, as above.
            const float size = 0x1p-9f * eight_unit(static_cast<uint32_t>(top_byte));
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) l[b][e] += __shfl_xor_sync(0xffffffffu, l[b][e], d);
                    const int r = b * 8 + t4 * 2 + e;
                    if (g == 0) { wm[warp][r] = m[b][e]; wl[warp][r] = l[b][e]; }
                }
            __syncthreads();
            float M[NB][2], L[NB][2];
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int r = b * 8 + t4 * 2 + e;
                    M[b][e] = wm[0][r];
#pragma unroll
                    for (int w = 1; w < C_::kWarps; ++w) M[b][e] = fmaxf(M[b][e], wm[w][r]);
                    const float base = M[b][e] == -INFINITY ? 0.0f : M[b][e];
                    L[b][e] = 0.0f;
#pragma unroll
                    for (int w = 0; w < C_::kWarps; ++w) L[b][e] = fmaf(wl[w][r], pow2(wm[w][r] - base), L[b][e]);
                    const float f = L[b][e] == 0.0f ? 0.0f : __fdividef(pow2(m[b][e] - base), L[b][e]);
#pragma unroll
                    for (int n = 0; n < NC; ++n) {
                        o[n][b][e] = o[n][b][e] * f * size;
                        o[n][b][2 + e] = o[n][b][2 + e] * f * size;
                    }
                }
            const auto each = [&](auto use) {      // of this lane's heads and pairs of columns
#pragma unroll
                for (int b = 0; b < NB; ++b)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int r = b * 8 + t4 * 2 + e;
                        if (r < rows) {
#pragma unroll
                            for (int n = 0; n < NC; ++n) use(r, n * 16 + g * 2, o[n][b][e], o[n][b][2 + e]);
                        }
                    }
            };
            const auto put = [&](int at) {
                each([&](int r, int c, float x, float y) { *reinterpret_cast<float2*>(mg + (at * rows + r) * C_::kMergeRow + c) = make_float2(x, y); });
            };
            const auto add = [&](int at) {
                each([&](int r, int c, float& x, float& y) {
                    const float2 v = *reinterpret_cast<const float2*>(mg + (at * rows + r) * C_::kMergeRow + c);
                    x += v.x;
                    y += v.y;
                });
            };
            if (warp >= 2) put(warp - 2);
            __syncthreads();
            if (warp < 2) add(warp);
            if (warp == 1) put(1);
            __syncthreads();
            if (warp == 0) {
                add(1);
                // a part's sum of weights as its reference; parts are 2^-10 each, so that hundreds of them do not overflow
                const float part = 1.0f / a.raise;
                if (a.split > 1) {
                    each([&](int, int, float& x, float& y) { x *= part; y *= part; });
                    put(0);
                }
#pragma unroll
                for (int b = 0; b < NB; ++b)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int r = b * 8 + t4 * 2 + e;
                        const bool none = L[b][e] == 0.0f;
                        const auto whole = [&] { return none ? -INFINITY : M[b][e] + log2f(L[b][e]); };
                        if (a.split > 1) {
                            if (g == 0) { wm[0][r] = whole(); wl[0][r] = none ? 0.0f : part; }
                            continue;
                        }
                        if (r >= rows) continue;
                        if (complete) {
                            const bool some = L[b][e] != 0.0f && head_kept(a, h0 + r);
                            const long long row = static_cast<long long>(con.s) * a.H + h0 + r;
                            uint32_t* out = reinterpret_cast<uint32_t*>(static_cast<Io*>(a.out) + row * a.dh);
#pragma unroll
                            for (int n = 0; n < NC; ++n)
                                if (n * 16 < a.dh) out[n * 8 + g] = some ? pack_bf16(o[n][b][e], o[n][b][2 + e]) : 0u;
                            if (g == 0 && a.lse) a.lse[row] = some ? whole() * kLn2 : -INFINITY;
                        } else {
                            if (g == 0) { slot[r] = whole(); slot[16 + r] = none ? 0.0f : part; }
#pragma unroll
                            for (int n = 0; n < NC; ++n)
                                *reinterpret_cast<float2*>(slot + kSlotHead + r * DP + n * 16 + g * 2) = make_float2(o[n][b][e] * part, o[n][b][2 + e] * part);
                        }
                    }
            }
        } else {
            float* q = reinterpret_cast<float*>(ring + C_::kRing);
            float* w = q + GR * DP;               // [GR][16]
            __syncwarp();
            for (int i = lane; i < GR * DP; i += 32) {
                const int r = i / DP, c = i % DP;
                q[i] = (r < rows && c < a.dh) ? ldg_waited(reinterpret_cast<const float*>(qrow) + static_cast<long long>(r) * a.dh + c) : 0.0f;
            }
            __syncwarp();
            float o[GR][V], m[GR], l[GR];
#pragma unroll
            for (int r = 0; r < GR; ++r) {
                m[r] = -INFINITY;
                l[r] = 0.0f;
#pragma unroll
                for (int v = 0; v < V; ++v) o[r][v] = 0.0f;
            }
            for (int t = con.t0; t < con.t1; ++t) {
                masks[S - 1] = issue();
                cp_wait<S - 1>();
                __syncwarp();
                const uint32_t mask = masks[0];
#pragma unroll
                for (int i = 0; i + 1 < S; ++i) masks[i] = masks[i + 1];
                const float* kp = reinterpret_cast<const float*>(ring + slot_out * C_::kStage);
                const float* vp = kp + C_::kHalf / 4;
                if (++slot_out == S) slot_out = 0;
                if (mask == 0) continue;
                // scores: lanes 2p and 2p + 1 take the even and the odd 16-byte chunks of position p
                const int key = lane >> 1;
                float sc[GR];
#pragma unroll
                for (int r = 0; r < GR; ++r) sc[r] = 0.0f;
#pragma unroll 4
                for (int i = lane & 1; i < DP / 4; i += 2) {
                    const float4 kv = *reinterpret_cast<const float4*>(kp + key * (DP + 8) + i * 4);
#pragma unroll
                    for (int r = 0; r < GR; ++r) {
                        const float4 qv = *reinterpret_cast<const float4*>(q + r * DP + i * 4);
                        sc[r] = fmaf(qv.x, kv.x, fmaf(qv.y, kv.y, fmaf(qv.z, kv.z, fmaf(qv.w, kv.w, sc[r]))));
                    }
                }
                float f[GR];
                bool moved = false;
#pragma unroll
                for (int r = 0; r < GR; ++r) {
                    const float full = sc[r] + __shfl_xor_sync(0xffffffffu, sc[r], 1);
                    sc[r] = (mask >> key) & 1u ? full * a.scale_log2 : -INFINITY;
                    float mx = fmaxf(m[r], sc[r]);
#pragma unroll
                    for (int d = 2; d < 32; d <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
                    const float base = mx == -INFINITY ? 0.0f : mx;
                    f[r] = pow2(m[r] - base);
                    moved |= m[r] != mx;
                    m[r] = mx;
                    const float e = pow2(sc[r] - base);
                    l[r] = fmaf(l[r], f[r], e);
                    if ((lane & 1) == 0) w[r * kRun + key] = e;
                }
                __syncwarp();
                if (moved) {   // the same in every lane
#pragma unroll
                    for (int r = 0; r < GR; ++r)
#pragma unroll
                        for (int v = 0; v < V; ++v) o[r][v] *= f[r];
                }
                // weighted sum of the values: columns lane * 2, or lane * 4 (and 128 more)
#pragma unroll
                for (int kk = 0; kk < kRun; kk += 4) {
                    float vv[4][V];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float* row = vp + (kk + e) * (DP + 8);
                        if constexpr (V == 2) {
                            const float2 x = *reinterpret_cast<const float2*>(row + lane * 2);
                            vv[e][0] = x.x; vv[e][1] = x.y;
                        } else {
#pragma unroll
                            for (int b = 0; b < V / 4; ++b) {
                                const float4 x = *reinterpret_cast<const float4*>(row + lane * 4 + b * 128);
                                vv[e][b * 4] = x.x; vv[e][b * 4 + 1] = x.y; vv[e][b * 4 + 2] = x.z; vv[e][b * 4 + 3] = x.w;
                            }
                        }
                    }
#pragma unroll
                    for (int r = 0; r < GR; ++r) {
                        const float4 wv = *reinterpret_cast<const float4*>(w + r * kRun + kk);
#pragma unroll
                        for (int v = 0; v < V; ++v)
                            o[r][v] = fmaf(wv.x, vv[0][v], fmaf(wv.y, vv[1][v], fmaf(wv.z, vv[2][v], fmaf(wv.w, vv[3][v], o[r][v]))));
                    }
                }
                __syncwarp();   // the stage and the weights are free
            }
            // the warps meet, as above
#pragma unroll
            for (int r = 0; r < GR; ++r) {
#pragma unroll
                for (int d = 2; d < 32; d <<= 1) l[r] += __shfl_xor_sync(0xffffffffu, l[r], d);
                if (lane == 0) { wm[warp][r] = m[r]; wl[warp][r] = l[r]; }
            }
            __syncthreads();
#pragma unroll
            for (int r = 0; r < GR; ++r) {
                float M = wm[0][r];
#pragma unroll
                for (int w2 = 1; w2 < C_::kWarps; ++w2) M = fmaxf(M, wm[w2][r]);
                const float base = M == -INFINITY ? 0.0f : M;
                l[r] = 0.0f;
#pragma unroll
                for (int w2 = 0; w2 < C_::kWarps; ++w2) l[r] = fmaf(wl[w2][r], pow2(wm[w2][r] - base), l[r]);
                const float f = pow2(m[r] - base);
                m[r] = M;
#pragma unroll
                for (int v = 0; v < V; ++v) o[r][v] *= f;
            }
            const auto at = [&](int r, int v) { return V == 2 ? lane * 2 + v : lane * 4 + (v & 3) + (v >> 2) * 128; };
            const auto put = [&](int b) {
#pragma unroll
                for (int r = 0; r < GR; ++r)
                    if (r < rows)
#pragma unroll
                        for (int v = 0; v < V; ++v) mg[(b * rows + r) * C_::kMergeRow + at(r, v)] = o[r][v];
            };
            const auto add = [&](int b) {
#pragma unroll
                for (int r = 0; r < GR; ++r)
                    if (r < rows)
#pragma unroll
                        for (int v = 0; v < V; ++v) o[r][v] += mg[(b * rows + r) * C_::kMergeRow + at(r, v)];
            };
            if (warp >= 2) put(warp - 2);
            __syncthreads();
            if (warp + 2 < C_::kWarps) add(warp);
            if (warp == 1) put(1);
            __syncthreads();
            if (warp == 0) {
                add(1);
                if (a.split > 1) {
                    put(0);
#pragma unroll
                    for (int r = 0; r < GR; ++r)
                        if (lane == 0) { wm[0][r] = m[r]; wl[0][r] = l[r]; }
                }
#pragma unroll
                for (int r = 0; r < GR; ++r) {
                    if (r >= rows || a.split > 1) continue;
                    const bool some = l[r] != 0.0f && head_kept(a, h0 + r);
                    const long long row = static_cast<long long>(con.s) * a.H + h0 + r;
                    float* out = complete ? static_cast<float*>(a.out) + row * a.dh : slot + kSlotHead + r * DP;
                    const float n = complete ? (some ? 1.0f / l[r] : 0.0f) : 1.0f;
                    const bool zero = complete && !some;
#pragma unroll
                    for (int v = 0; v < V; ++v)
                        if (at(r, v) < a.dh || !complete) out[at(r, v)] = zero ? 0.0f : o[r][v] * n;
                    if (lane == 0) {
                        if (!complete) {
                            slot[r] = m[r];
                            slot[16 + r] = l[r];
                        } else if (a.lse) {
                            a.lse[row] = some ? (m[r] + log2f(l[r])) * kLn2 : -INFINITY;
                        }
                    }
                }
            }
        }
        if (a.split > 1) {   // the thread blocks of the item meet: sums through distributed shared memory, in rank order
            namespace cg = cooperative_groups;
            const cg::cluster_group cl = cg::this_cluster();
            cl.sync();
            for (int i = tid + static_cast<int>(cl.block_rank()) * kThreads; i < rows * a.dh; i += kThreads * a.split) {
                const int r = i / a.dh, j = i - r * a.dh;
                float M = -INFINITY;
                for (int k = 0; k < a.split; ++k) M = fmaxf(M, *cl.map_shared_rank(&wm[0][r], k));
                const float base = M == -INFINITY ? 0.0f : M;
                float L = 0.0f, v = 0.0f;
                for (int k = 0; k < a.split; ++k) {
                    const float f = pow2(*cl.map_shared_rank(&wm[0][r], k) - base);
                    L = fmaf(*cl.map_shared_rank(&wl[0][r], k), f, L);
                    v = fmaf(*cl.map_shared_rank(mg + r * C_::kMergeRow + j, k), f, v);
                }
                const bool some = L != 0.0f && head_kept(a, h0 + r);
                write_head<T>(a, con.s, h0 + r, j, some ? v / L : 0.0f);
                if (j == 0 && a.lse)
                    a.lse[static_cast<long long>(con.s) * a.H + h0 + r] = some ? (M + log2f(L * a.raise)) * kLn2 : -INFINITY;
            }
            cl.sync();       // nobody leaves while its sums may still be read
        }
        if (!a.split && tid == 0 && con.left == con.t1 - con.t0)   // the range's last piece
            a.cuts[blockIdx.x] = {con.t0 == 0 && con.t1 < con.nt, con.s, con.hi, con.nt - con.t1, total, con.left == range, 0};
        // a length out of range is reported where the sequence's first tile is
        if (con.t0 == 0 && con.hi == 0 && tid == 0) (void)valid_len(a, con.s, true);
        con.next(a);
    }
    cp_wait<0>();
    if (__any_sync(0xffffffffu, bad) && lane == 0) flag_status(a.status, HALO_DEV_BAD_INDEX);
}

// Joining the pieces of the items that were cut: two kernels, each of which waits for memory twice, for the records and for
// the pieces.  What a range has written of a cut that it opens:
struct Opened {
    int s, kvh, r0, rows;   // the item, and its first query head and their number
    int pieces;
    const float *ws0, *ws1;
    int slot;
    __device__ __forceinline__ Opened(const PagedArgs& a, const int4& head, bool fills, int c0, long long total, int C) {
        s = head.y;
        kvh = head.z / a.qblocks;
        r0 = (head.z % a.qblocks) * a.block;
        rows = min(a.block, a.G - r0);
        pieces = range_of(total, cut(total, c0 + 1, C) + head.w - 1, C) - c0 + 1;
        // piece 0 in the slot of range c0 that holds its end (its first one if the item fills the range), the others in
        // the first slots of the ranges behind it
        ws0 = a.ws + (static_cast<long long>(c0) * 2 + (fills ? 0 : 1)) * a.slot;
        ws1 = a.ws + static_cast<long long>(c0) * 2 * a.slot;
        slot = a.slot;
    }
    __device__ __forceinline__ const float* piece(int k) const { return k == 0 ? ws0 : ws1 + static_cast<long long>(k) * 2 * slot; }
};

// Many items of few pieces.  blockIdx.x = the range that begins an item and does not end it; DP threads, a column each, for
// a query head, several heads per thread block.
constexpr int kRangeJoin = 256;
template <typename T, int DP>
__global__ void __launch_bounds__(kRangeJoin) paged_mha_join_range_kernel(const __grid_constant__ PagedArgs a, int blocks) {
    constexpr int kAhead = 4;
    const int r = blockIdx.y * (kRangeJoin / DP) + threadIdx.x / DP, j = threadIdx.x % DP, c0 = blockIdx.x;
    chain_wait();   // in every block: this grid may not end before the first one
    const int4 head = __ldcg(reinterpret_cast<const int4*>(a.cuts + c0)), line = __ldcg(reinterpret_cast<const int4*>(a.cuts + c0) + 1);
    const long long total = __ldcg(&a.cuts[0].total);
    const int C = ranges(total, blocks);
    if (c0 + 1 >= C || !head.x) return;      // a block behind the last range reads a record that nobody wrote, and drops it
    const Opened o(a, head, line.z, c0, total, C);
    if (r >= o.rows) return;
    float M = -INFINITY, L = 0.0f, v = 0.0f;
    for (int k0 = 0; k0 < o.pieces; k0 += kAhead) {
        float m[kAhead], l[kAhead], x[kAhead];
#pragma unroll
        for (int e = 0; e < kAhead; ++e) {
            const bool there = k0 + e < o.pieces;
            const float* p = o.piece(k0 + e);
            m[e] = there ? __ldcg(p + r) : -INFINITY;
            l[e] = there ? __ldcg(p + 16 + r) : 0.0f;
            x[e] = there ? __ldcg(p + kSlotHead + r * DP + j) : 0.0f;
        }
#pragma unroll
        for (int e = 0; e < kAhead; ++e) {
            const float mx = fmaxf(M, m[e]), base = mx == -INFINITY ? 0.0f : mx;
            const float f = pow2(M - base), w = pow2(m[e] - base);
            M = mx;
            L = fmaf(L, f, l[e] * w);
            v = fmaf(v, f, x[e] * w);
        }
    }
    const int h = o.kvh * a.G + o.r0 + r;
    const bool some = L != 0.0f && head_kept(a, h);
    if (j < a.dh) write_head<T>(a, o.s, h, j, some ? v / L : 0.0f);
    if (j == 0 && a.lse) a.lse[static_cast<long long>(o.s) * a.H + h] = some ? (M + log2f(L * a.raise)) * kLn2 : -INFINITY;
}

// Few items of many pieces.  blockIdx.x = item, blockIdx.y = query head of it; the thread block looks for the item among the
// records of all ranges (a thread block per range would be one of thousands that find nothing to do: one sequence of 32000
// positions, 16 heads on one, 32 us and 20 as here).  Groups of DP threads, a column each, take every kGroups-th piece; the
// first kAhead values of a thread are requested together with the pieces' maxima and sums (one piece per thread).
constexpr int kItemJoin = 512;
template <typename T, int DP>
__global__ void __launch_bounds__(kItemJoin) paged_mha_join_item_kernel(const __grid_constant__ PagedArgs a, int blocks) {
    static_assert(kItemJoin % DP == 0 && DP % 32 == 0, "groups of whole warps");
    constexpr int kGroups = kItemJoin / DP, kAhead = 12, THREADS = kItemJoin;
    constexpr int kMost = (kSmCount * 4 + THREADS - 1) / THREADS;      // records per thread
    __shared__ float red[2][THREADS / 32];
    __shared__ float part[THREADS];
    __shared__ int4 found[2];
    __shared__ int at_range;
    extern __shared__ float weight[];   // [pieces]
    const int r = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid == 0) at_range = -1;
    chain_wait();   // in every block: this grid may not end before the first one
    __syncthreads();
    const long long total = __ldcg(&a.cuts[0].total);
    int4 rec[kMost][2];
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
        const int4* from = reinterpret_cast<const int4*>(a.cuts + min(tid + i * THREADS, blocks - 1));
        rec[i][0] = __ldcg(from);
        rec[i][1] = __ldcg(from + 1);
    }
    const int C = ranges(total, blocks);
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
        const int c = tid + i * THREADS;      // behind the last range: a record that nobody wrote
        if (c + 1 < C && rec[i][0].x && static_cast<long long>(rec[i][0].y) * a.Hk * a.qblocks + rec[i][0].z == blockIdx.x) {
            at_range = c;
            found[0] = rec[i][0];
            found[1] = rec[i][1];
        }
    }
    __syncthreads();
    const int c0 = at_range;
    if (c0 < 0) return;      // not cut
    const Opened o(a, found[0], found[1].z, c0, total, C);
    if (r >= o.rows) return;
    const int s = o.s, pieces = o.pieces, h = o.kvh * a.G + o.r0 + r;
    const auto slot = [&](int k) { return o.piece(k); };
    const int grp = tid / DP, j = tid % DP;
    const int at = kSlotHead + r * DP + j;

    float ahead[kAhead];
#pragma unroll
    for (int e = 0; e < kAhead; ++e) {
        const int k = grp + e * kGroups;
        ahead[e] = k < pieces ? __ldcg(slot(k) + at) : 0.0f;
    }
    float M = -INFINITY, l_own = 0.0f;
    for (int k = tid; k < pieces; k += THREADS) {
        const float m = __ldcg(slot(k) + r);
        if (k == tid) l_own = __ldcg(slot(k) + 16 + r);
        weight[k] = m;
        M = fmaxf(M, m);
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, d));
    if (lane == 0) red[0][warp] = M;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) M = fmaxf(M, red[0][w]);
    const float base = M == -INFINITY ? 0.0f : M;
    float L = 0.0f;
    for (int k = tid; k < pieces; k += THREADS) {
        const float f = exp2f(weight[k] - base);
        weight[k] = f;
        L = fmaf(k == tid ? l_own : __ldcg(slot(k) + 16 + r), f, L);
    }
    L = warp_sum(L);
    if (lane == 0) red[1][warp] = L;
    __syncthreads();
    L = 0.0f;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) L += red[1][w];
    const bool some = L != 0.0f && head_kept(a, h);
    float v = 0.0f;
#pragma unroll
    for (int e = 0; e < kAhead; ++e) {
        const int k = grp + e * kGroups;
        if (k < pieces) v = fmaf(ahead[e], weight[k], v);
    }
#pragma unroll 16
    for (int k = grp + kAhead * kGroups; k < pieces; k += kGroups) v = fmaf(__ldcg(slot(k) + at), weight[k], v);
    part[tid] = v;
    __syncthreads();
    if (grp == 0) {
#pragma unroll
        for (int e = 1; e < kGroups; ++e) v += part[tid + e * DP];
    }
    if (grp == 0 && j < a.dh) write_head<T>(a, s, h, j, some ? v / L : 0.0f);
    if (tid == 0 && a.lse) a.lse[static_cast<long long>(s) * a.H + h] = some ? (M + log2f(L * a.raise)) * kLn2 : -INFINITY;
}

struct LaunchPlan {
    int blocks, split;
    int slot, rows, merge;   // as in PagedArgs
    long long items;
};
template <typename T, int DP, int GR>
LaunchPlan plan_of(const halo_paged_shape& sh, int n_seq) {
    using C_ = Cfg<T, DP, GR>;
    const int G = sh.n_heads / sh.n_kv_heads;
    const long long cap = static_cast<long long>(sh.max_pages) * sh.page_size;
    const long long tiles = (cap + C_::kTile - 1) / C_::kTile;
    LaunchPlan p;
    constexpr int kBlock = item_rows(C_::kF32);
    p.items = static_cast<long long>(n_seq) * sh.n_kv_heads * ((G + kBlock - 1) / kBlock);
    p.rows = G < kBlock ? G : kBlock;
    p.slot = kSlotHead + p.rows * DP;
    p.merge = (C_::merge_bytes(p.rows) + 15) / 16 * 16;
    const long long resident = static_cast<long long>(kSmCount) * C_::kBlocksPerSm;
    // Few and short items: a cluster per item, one launch (one sequence of 700 positions, 32 / 4 heads of 64: 8.6 us as a
    // line with a join, 7.1 as clusters of 8).  A cluster's meeting costs 1.3 us, a tile about 0.8: two tiles are not
    // split (128 positions, 5.5 us and 6.8).  Elsewhere the line: it balances lengths and fills the GPU.
    p.split = 0;
    if (p.items <= resident) {
        int n = 1;
        while (n < 8 && tiles > 2 && 2 * n <= tiles && 2 * n * p.items <= resident) n *= 2;
        if (tiles <= 8ll * n) p.split = n;
    }
    p.blocks = static_cast<int>(p.split ? p.items * p.split : tiles * p.items < resident ? tiles * p.items : resident);
    return p;
}
size_t workspace_of(const LaunchPlan& p) {
    return p.split ? 0 : static_cast<size_t>(p.blocks) * (sizeof(Cut) + sizeof(float) * 2 * p.slot);
}

template <typename T, int DP, int GR>
halo_status launch(const PagedArgs& args, const LaunchPlan& p, cudaStream_t st) {
    using C_ = Cfg<T, DP, GR>;
    static bool done[64];
    if (!ensure_dynamic_smem(paged_mha_kernel<T, DP, GR>, C_::kMaxSmem, done)) return HALO_ERR_CUDA;
    PagedArgs a = args;
    a.split = p.split;
    a.slot = p.slot;
    a.rows = p.rows;
    a.merge = p.merge;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(p.blocks);
    cfg.blockDim = dim3(C_::kWarps * 32);
    cfg.dynamicSmemBytes = C_::kRings + p.merge;
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;   // as in launch_chained
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = p.split > 1 ? p.split : 1;
    at[1].val.clusterDim.y = 1;
    at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = p.split > 1 ? 2 : 1;
    const halo_status rc = cuda_status(cudaLaunchKernelEx(&cfg, paged_mha_kernel<T, DP, GR>, a));
    if (rc != HALO_OK || p.split || p.blocks < 2) return rc;
    if (p.blocks >= 8 * p.items)
        return launch_chained(paged_mha_join_item_kernel<typename Kind<T>::Io, DP>, dim3(static_cast<unsigned>(p.items), p.rows), kItemJoin,
                              sizeof(float) * p.blocks, st, a, p.blocks);
    constexpr int kHeads = kRangeJoin / DP;
    return launch_chained(paged_mha_join_range_kernel<typename Kind<T>::Io, DP>, dim3(p.blocks - 1, (p.rows + kHeads - 1) / kHeads), kRangeJoin, 0, st, a,
                          p.blocks);
}

template <typename T, int DP, typename F>
auto by_rows(const halo_paged_shape& sh, F f) {
    using D = std::integral_constant<int, DP>;
    const int G = sh.n_heads / sh.n_kv_heads;
    if constexpr (!std::is_same<T, float>::value) {
        return G <= 8 ? f(T(), D(), std::integral_constant<int, 8>()) : f(T(), D(), std::integral_constant<int, 16>());
    } else {
        if (G == 1) return f(T(), D(), std::integral_constant<int, 1>());
        return f(T(), D(), std::integral_constant<int, 4>());
    }
}
template <typename T, typename F>
auto by_width(const halo_paged_shape& sh, F f) {
    return sh.head_dim <= 64 ? by_rows<T, 64>(sh, f) : sh.head_dim <= 128 ? by_rows<T, 128>(sh, f) : by_rows<T, 256>(sh, f);
}
template <typename F>
auto by_type(const halo_paged_shape& sh, bool eight, F f) {
    if (eight) return by_width<Eight>(sh, f);
    return sh.dtype == HALO_BF16 ? by_width<__nv_bfloat16>(sh, f) : by_width<float>(sh, f);
}

LaunchPlan plan_for(const halo_paged_shape& sh, int n_seq, bool eight) {
    return by_type(sh, eight, [&](auto t, auto dp, auto gr) { return plan_of<decltype(t), decltype(dp)::value, decltype(gr)::value>(sh, n_seq); });
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

namespace {
// halo_paged_mha and halo_paged_mha_f8 (scales: the latter)
halo_status attend(const halo_paged_shape* shape, int n_seq, const void* q, long long q_stride, const void* K_cache,
                   const void* V_cache, bool eight, const uint8_t* K_scale, const uint8_t* V_scale, const int32_t* block_table,
                   const int32_t* seq_len, const uint8_t* keep, float scale, void* out, float* lse, void* workspace,
                   size_t workspace_bytes, uint32_t* dev_status, void* stream) {
    halo_status rc = check_paged_shape(shape);
    if (rc != HALO_OK) return rc;
    if (!q || !K_cache || !V_cache || !block_table || !seq_len || !out || (eight && (!K_scale || !V_scale))) return HALO_ERR_ARG;
    if (!isfinite(scale)) return HALO_ERR_ARG;
    if (n_seq <= 0 || n_seq > HALO_MAX_SEQUENCES) return HALO_ERR_SHAPE;
    const int elem = shape->dtype == HALO_F32 ? 4 : 2;
    const long long row = static_cast<long long>(shape->n_heads) * shape->head_dim;
    if (q_stride < row) return HALO_ERR_SHAPE;
    if (!aligned16(q) || !aligned16(K_cache) || !aligned16(V_cache) || !aligned16(out) || q_stride * elem % 16 != 0)
        return HALO_ERR_ALIGN;
    rc = check_eight(*shape, K_scale, V_scale);
    if (rc != HALO_OK) return rc;
    const LaunchPlan p = plan_for(*shape, n_seq, eight);
    const size_t need = workspace_of(p);
    if (need > 0 && (!workspace || workspace_bytes < need)) return HALO_ERR_WORKSPACE;
    if (need > 0 && !aligned16(workspace)) return HALO_ERR_ALIGN;
    PagedArgs a = {};
    a.n_seq = n_seq;
    a.H = shape->n_heads;
    a.Hk = shape->n_kv_heads;
    a.G = a.H / a.Hk;
    a.block = item_rows(shape->dtype == HALO_F32);
    a.qblocks = (a.G + a.block - 1) / a.block;
    a.dh = shape->head_dim;
    a.page_size = shape->page_size;
    a.page_shift = -1;
    for (int b = 0; b < 31; ++b)
        if (shape->page_size == 1 << b) a.page_shift = b;
    a.n_pages = shape->n_pages;
    a.max_pages = shape->max_pages;
    a.page_stride = paged_stride(*shape);
    a.q_stride = q_stride;
    a.scale_log2 = scale * 1.44269504088896340736f;
    a.raise = eight ? 1024.0f : 1.0f;
    a.q = q;
    a.K = K_cache;
    a.V = V_cache;
    a.K_scale = K_scale;
    a.V_scale = V_scale;
    a.table = block_table;
    a.seq_len = seq_len;
    a.keep = keep;
    a.out = out;
    a.lse = lse;
    a.status = dev_status;
    a.cuts = static_cast<Cut*>(workspace);
    a.ws = reinterpret_cast<float*>(a.cuts + p.blocks);
    return by_type(*shape, eight, [&](auto t, auto dp, auto gr) {
        return launch<decltype(t), decltype(dp)::value, decltype(gr)::value>(a, p, static_cast<cudaStream_t>(stream));
    });
}

size_t workspace_bytes_of(const halo_paged_shape* shape, int n_seq, bool eight) {
    if (check_paged_shape(shape) != HALO_OK || n_seq <= 0 || n_seq > HALO_MAX_SEQUENCES) return 0;
    return workspace_of(plan_for(*shape, n_seq, eight));
}
}  // namespace
}  // namespace halo

using namespace halo;

extern "C" size_t halo_paged_mha_workspace_bytes(const halo_paged_shape* shape, int n_seq) {
    return workspace_bytes_of(shape, n_seq, false);
}

extern "C" halo_status halo_paged_mha(const halo_paged_shape* shape, int n_seq, const void* q, long long q_stride,
                                      const void* K_cache, const void* V_cache, const int32_t* block_table,
                                      const int32_t* seq_len, const uint8_t* keep, float scale, void* out, float* lse,
                                      void* workspace, size_t workspace_bytes, uint32_t* dev_status, void* stream) {
    return attend(shape, n_seq, q, q_stride, K_cache, V_cache, false, nullptr, nullptr, block_table, seq_len, keep, scale, out, lse,
                  workspace, workspace_bytes, dev_status, stream);
}

extern "C" size_t halo_paged_mha_f8_workspace_bytes(const halo_paged_shape* shape, int n_seq) {
    return shape && shape->dtype == HALO_BF16 ? workspace_bytes_of(shape, n_seq, true) : 0;
}

extern "C" halo_status halo_paged_mha_f8(const halo_paged_shape* shape, int n_seq, const void* q, long long q_stride,
                                         const void* K_cache, const void* V_cache, const uint8_t* K_scale, const uint8_t* V_scale,
                                         const int32_t* block_table, const int32_t* seq_len, const uint8_t* keep, float scale,
                                         void* out, float* lse, void* workspace, size_t workspace_bytes, uint32_t* dev_status,
                                         void* stream) {
    return attend(shape, n_seq, q, q_stride, K_cache, V_cache, true, K_scale, V_scale, block_table, seq_len, keep, scale, out, lse,
                  workspace, workspace_bytes, dev_status, stream);
}
