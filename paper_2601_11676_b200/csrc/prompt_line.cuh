// The work line of halo_paged_prompt_mha, shared by its kernels.
//
// An item is ROWS rows of one (sequence, K/V head): row token * G + g of them is query head g of the G that share the K/V head, so
// keys and values that come into an SM serve all of them.  Its keys, up to the last position that a row sees, are cut
// into tiles of TILE.  An item is as many units long as it has tiles, and OVER more in front of them, which stand for what
// an item costs besides (its rows, an empty pipeline, its outputs).  All items, one after another, form one line of T units and thread
// block c of C takes [c * T / C, (c + 1) * T / C): however long prompts and caches are, every thread block has the same to do, and
// few rows over a long cache fill the GPU as well as many.  A piece that has all of an item's tiles writes its output; the at
// most two pieces of a range that do not leave (maximum, sum, weighted sum of values) per row in the workspace, and a second kernel
// joins them in line order, so results do not depend on timing.  Every thread block computes the line from q_start and seq_len
// itself; the host never reads a length.
#pragma once

#include "eight.cuh"

namespace halo {
namespace prompt {

// What the join has to know of a range whose last piece begins an item that it does not end.
struct __align__(16) Opening {
    int opens, kvh, rb, first, n;   // the item, its sequence's rows of q
    int rest;                       // units of the item behind the range
    long long total;                // T
};
static_assert(sizeof(Opening) == 32, "two 16-byte words");

struct Args {
    int n_tok, n_seq, H, Hk, G, dh, page_size, page_shift, n_pages, max_pages;   // page_shift: -1 = no power of two
    int blocks;              // thread blocks of the first kernel
    int rows;                // rows of a workspace slot
    long long slot;          // floats of it
    long long page_stride, q_stride;
    float scale_log2;
    float lower, raise;      // weights are times 2^-lower; 2^lower
    const void* q;
    const void* K;
    const void* V;
    const uint8_t* K_scale;  // 8-bit rows
    const uint8_t* V_scale;
    const int32_t* q_start;
    const int32_t* table;
    const int32_t* seq_len;
    const uint8_t* keep;
    void* out;
    float* lse;
    Opening* openings;       // [blocks], then the slots: two per thread block
    float* ws;
    uint32_t* status;
};

constexpr float kLn2 = 0.693147180559945309f;

// A slot: maxima [rows], sums [rows], weighted sums [dh / 4][rows][4]: neighbouring rows side by side, as threads hold them.  rows
// is what an item can have.
inline int slot_rows(int item_rows, int n_tok, const halo_paged_shape& sh) {
    const long long all = static_cast<long long>(n_tok) * (sh.n_heads / sh.n_kv_heads);
    return all < item_rows ? static_cast<int>((all + 3) / 4 * 4) : item_rows;
}
__host__ __device__ constexpr long long slot_floats(int rows, int dh) { return static_cast<long long>(rows) * (dh + 2); }

// 2^x, results below 2^-126 as 0
__device__ __forceinline__ float pow2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ bool head_kept(const Args& a, int h) { return !a.keep || a.keep[h] != 0; }

struct Rows {      // of a sequence
    int first, n, len;
};
struct Order {     // of sequences in front
    int end;         // the largest end of those whose rows are in range
    bool falls;      // a start was behind its end
};
__device__ __forceinline__ Rows rows_of(const Args& a, int s, Order& o, bool flag) {
    const int q0 = ldg_waited(a.q_start + s), q1 = ldg_waited(a.q_start + s + 1), len = ldg_waited(a.seq_len + s);
    const bool in = q0 >= 0 && q1 >= q0 && q1 <= a.n_tok, rows = in && q0 >= o.end;      // rows of two sequences belong to the first one
    const bool fits = len >= 0 && len <= static_cast<long long>(a.max_pages) * a.page_size;
    if (flag && !(rows && fits)) flag_status(a.status, HALO_DEV_BAD_INDEX);
    o.falls |= q1 < q0;
    if (in) o.end = max(o.end, q1);
    return {q0, rows ? q1 - q0 : 0, fits ? len : 0};
}

// sum over i < n of floor((step * i + from) / m), by exchanging the roles of step and m until nothing is left (Euclid's way);
// step * n + from < 2^32
__device__ __forceinline__ unsigned long long sum_of_floors(uint32_t n, uint32_t m, uint32_t step, uint32_t from) {
    unsigned long long sum = 0;
    while (n > 0) {
        sum += static_cast<unsigned long long>(n) * (n - 1) / 2 * (step / m) + static_cast<unsigned long long>(n) * (from / m);
        step %= m;
        from %= m;
        const uint32_t top = step * n + from;
        n = top / m;
        from = top - n * m;
        const uint32_t t = m;
        m = step;
        step = t;      // m = 0: n is 0 too
    }
    return sum;
}

// Rows times heads of a call stay below 2^30 (HALO_MAX_PROMPT_ROWS, HALO_MAX_GROUPS).
template <int ROWS, int TILE, int OVER>
struct Line {
    static __device__ __forceinline__ int blocks_of(const Args& a, const Rows& r) { return (r.n * a.G + ROWS - 1) / ROWS; }
    // positions that the last row of an item sees
    static __device__ __forceinline__ int reach(const Args& a, const Rows& r, int rb) {
        const int u = (rb + 1) * ROWS - 1, all = r.n * a.G - 1;
        return max(r.len - r.n + (u < all ? u / a.G : r.n - 1) + 1, 0);
    }
    // an item that sees nothing keeps one tile, which writes its zeros
    static __device__ __forceinline__ int tiles_of(int reach) { return reach > 0 ? (reach - 1) / TILE + 1 : 1; }
    static __device__ __forceinline__ int tiles(const Args& a, const Rows& r, int rb) { return tiles_of(reach(a, r, rb)); }
    // units of all items of one K/V head of a sequence
    static __device__ __forceinline__ long long per_head(const Args& a, const Rows& r) {
        if (r.n == 0) return 0;
        const int nb = blocks_of(a, r), last = tiles_of(r.len);
        if (nb == 1) return last + OVER;
        // item rb < nb - 1: max(1, floor((ROWS * (rb + 1) - 1 + G * (base + TILE)) / (G * TILE))), base = len - n; base = TILE * q + rest
        const int base = r.len - r.n, m = a.G * TILE;
        int ones = base < 0 ? static_cast<int>(min(-static_cast<long long>(base) * a.G / ROWS, nb - 1ll)) : 0;      // items of which no row sees anything
        const int q = base >= 0 ? base / TILE : -((TILE - 1 - base) / TILE), rest = base - q * TILE;
        const int n = nb - 1 - ones;
        const long long some = n > 0 ? static_cast<long long>(n) * (q + 1) + static_cast<long long>(
                                           sum_of_floors(n, m, ROWS, ROWS * (ones + 1) - 1 + rest * a.G)) : 0;
        return last + ones + some + static_cast<long long>(OVER) * nb;
    }
};

// Most lines are short: a division of 32 bits takes a fifth of the time
__device__ __forceinline__ long long quotient(long long x, long long by) {      // of numbers that are not negative
    return (x | by) >> 32 ? x / by : static_cast<uint32_t>(x) / static_cast<uint32_t>(by);
}
// Thread blocks that have a range, and where the c-th range begins.  A unit is enough for one: 8 tokens over 700 take 23.5 us, with
// ranges of at least four units, and so fewer joins, 27.6.
__device__ __forceinline__ int ranges(long long T, int blocks) { return T < 1 ? 1 : T < blocks ? static_cast<int>(T) : blocks; }
__device__ __forceinline__ long long cut(long long T, int c, int C) { return quotient(T * c, C); }
// the range that holds line position x: the last c with T * c / C <= x
__device__ __forceinline__ int range_of(long long T, long long x, int C) { return static_cast<int>(quotient((x + 1) * C - 1, T)); }

// where the sums of a piece that is not complete go: a range's first piece has no first tile, its last one has
__device__ __forceinline__ float* slot_of(const Args& a, int t0) { return a.ws + (static_cast<long long>(blockIdx.x) * 2 + (t0 > 0 ? 0 : 1)) * a.slot; }

// The way along a range: piece after piece.
template <int ROWS, int TILE, int OVER>
struct Walk {
    using L = Line<ROWS, TILE, OVER>;
    long long left;      // units from u0 of this item to the end of the range
    Rows r;
    Order order;         // of the sequences up to this one
    int s, kvh, rb, nb;
    int u0, u1;          // units of the item that the range has
    int nt, t0, t1;      // tiles of the item, and of them this piece's
    int reach;           // positions that take part: 0 where every head of the item is lost
    __device__ __forceinline__ void item(const Args& a) {
        reach = L::reach(a, r, rb);
        nt = L::tiles_of(reach);
        u1 = static_cast<int>(min(static_cast<long long>(nt + OVER), u0 + left));
        t0 = max(u0 - OVER, 0);
        t1 = max(u1 - OVER, 0);
        if (a.keep) {
            bool any = false;
            for (int g = 0; g < a.G; ++g) any |= head_kept(a, kvh * a.G + g);
            if (!any) reach = 0;
        }
    }
    __device__ __forceinline__ bool complete() const { return t0 == 0 && t1 == nt; }
    __device__ __forceinline__ bool opens() const { return t0 == 0 && t1 < nt; }
    __device__ __forceinline__ void next(const Args& a) {
        do {
            left -= u1 - u0;
            if (left <= 0) return;
            u0 = 0;
            if (++rb == nb) {
                rb = 0;
                if (++kvh == a.Hk) {
                    kvh = 0;
                    do r = rows_of(a, ++s, order, false);
                    while (r.n == 0);      // a range ends with the last item: there is one
                    nb = L::blocks_of(a, r);
                }
            }
            item(a);
        } while (t1 <= t0);      // a piece of the units in front alone: its tiles are the next range's
    }
    __device__ __forceinline__ float* slot(const Args& a) const { return slot_of(a, t0); }
    __device__ __forceinline__ Opening opening(long long total) const { return {opens(), kvh, rb, r.first, r.n, nt + OVER - u1, total}; }
};

template <int ROWS, int TILE, int OVER>
struct Found {
    Walk<ROWS, TILE, OVER> walk;
    long long total;
};
// The range of this thread block; all its THREADS threads call it.  left <= 0: nothing to do.
template <int ROWS, int TILE, int OVER, int THREADS>
__device__ __forceinline__ Found<ROWS, TILE, OVER> locate(const Args& a, long long* sh /*[THREADS / 32 + 3]*/) {
    using L = Line<ROWS, TILE, OVER>;
    constexpr int W = THREADS / 32;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int per = (a.n_seq + THREADS - 1) / THREADS;
    const int s0 = min(tid * per, a.n_seq), s1 = min(s0 + per, a.n_seq);
    long long own, first, incl;             // units of one K/V head: of all this thread's sequences, of its first; of all up to it
    Order front = {0, false}, behind;       // of the sequences in front of this thread's, and behind its first one
    const auto count = [&] {
        Order o = front;
        own = first = 0;
        for (int s = s0; s < s1; ++s) {
            const long long n = L::per_head(a, rows_of(a, s, o, blockIdx.x == 0));
            if (s == s0) {
                first = n;
                behind = o;
            }
            own += n;
        }
        incl = own;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const long long v = __shfl_up_sync(0xffffffffu, incl, d);
            if (lane >= d) incl += v;
        }
        if (lane == 31) sh[warp] = incl;
        return o;
    };
    const Order upto = count();
    if (__syncthreads_or(upto.falls)) {     // starts that fall: rows may belong to two sequences; the ends in front of this thread's
        int end = upto.end;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, end, d);
            if (lane >= d) end = max(end, v);
        }
        if (lane == 31) sh[warp] = end;
        __syncthreads();
        end = __shfl_up_sync(0xffffffffu, end, 1);
        if (lane > 0) front.end = end;
        for (int w = 0; w < warp; ++w) front.end = max(front.end, static_cast<int>(sh[w]));
        __syncthreads();
        count();
        __syncthreads();
    }
    long long before = 0, total = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) {
        if (w < warp) before += sh[w];
        total += sh[w];
    }
    Found<ROWS, TILE, OVER> f;
    Walk<ROWS, TILE, OVER>& w = f.walk;
    f.total = total * a.Hk;
    w.left = 0;
    const int C = ranges(f.total, a.blocks);
    if (static_cast<int>(blockIdx.x) >= C) return f;                         // the same in every thread
    if (tid == 0) a.openings[blockIdx.x] = {0, 0, 0, 0, 0, 0, f.total};      // unless a piece opens an item
    if (f.total == 0) return f;
    const long long x = cut(f.total, blockIdx.x, C);
    long long at = (before + incl - own) * a.Hk;
    if (x >= at && x < at + own * a.Hk) {
        Order o = front;
        for (int s = s0; s < s1; ++s) {
            const int end = o.end;
            const long long n = s == s0 ? first : L::per_head(a, rows_of(a, s, o, false));
            if (s == s0) o = behind;
            if (x < at + n * a.Hk) {
                sh[W] = x - at;
                sh[W + 1] = static_cast<long long>(end) << 32 | s;
                sh[W + 2] = n;
                break;
            }
            at += n * a.Hk;
        }
    }
    __syncthreads();
    const long long inside = sh[W], per_head = sh[W + 2];
    w.s = static_cast<int>(sh[W + 1]);
    w.order = {static_cast<int>(sh[W + 1] >> 32), false};
    w.left = cut(f.total, blockIdx.x + 1, C) - x;
    w.r = rows_of(a, w.s, w.order, false);
    w.nb = L::blocks_of(a, w.r);
    w.kvh = static_cast<int>(quotient(inside, per_head));
    // the item: 32 at a time
    long long rem = inside - w.kvh * per_head;
    for (int b = 0;; b += 32) {
        const int n = b + lane < w.nb ? L::tiles(a, w.r, b + lane) + OVER : 0;
        long long upto = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long v = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += v;
        }
        const uint32_t past = __ballot_sync(0xffffffffu, upto > rem);
        if (past) {
            const int at_lane = __ffs(past) - 1;
            w.rb = b + at_lane;
            w.u0 = static_cast<int>(rem - __shfl_sync(0xffffffffu, upto - n, at_lane));
            break;
        }
        rem -= __shfl_sync(0xffffffffu, upto, 31);
    }
    w.item(a);
    if (w.t1 <= w.t0) w.next(a);
    __syncthreads();      // sh may be used for something else
    return f;
}

// Row i of an item: its token and head, or no row.
struct Row {
    int token, head;      // row of q; query head
    int sees;             // positions
    bool there, kept;
};
template <int ROWS>
__device__ __forceinline__ Row row_at(const Args& a, const Rows& r, int kvh, int rb, int i) {
    const int u = rb * ROWS + i;
    Row w;
    w.there = u < r.n * a.G;
    const int token = w.there ? u / a.G : 0;
    w.token = r.first + token;
    w.head = kvh * a.G + (w.there ? u - token * a.G : 0);
    w.kept = w.there && head_kept(a, w.head);
    w.sees = max(r.len - r.n + token + 1, 0);
    return w;
}

// Pieces of cut items: blockIdx.x = the range that begins an item and does not end it, blockIdx.y = 32 rows and 64 columns of it.
// A lane has a row, a warp eight columns.
template <typename Io, int ROWS>
__global__ void __launch_bounds__(256) paged_prompt_join_kernel(const __grid_constant__ Args a) {
    constexpr int kAhead = 4;
    const int lane = threadIdx.x & 31, c0 = blockIdx.x, groups = (a.rows + 31) / 32;
    const int row = (blockIdx.y % groups) * 32 + lane, c4 = (blockIdx.y / groups) * 16 + (threadIdx.x >> 5) * 2;      // of four columns
    chain_wait();   // in every block: this grid may not end before the first one
    const int4 head = __ldcg(reinterpret_cast<const int4*>(a.openings + c0));
    const int4 more = __ldcg(reinterpret_cast<const int4*>(a.openings + c0) + 1);
    const long long total = __ldcg(&a.openings[0].total);
    const int C = ranges(total, a.blocks);
    if (c0 + 1 >= C || !head.x || c4 * 4 >= a.dh) return;   // behind the last range: a record that nobody wrote
    const Row w = row_at<ROWS>(a, {head.w, more.x, 0}, head.y, head.z, row);
    if (!w.there) return;
    const int pieces = range_of(total, cut(total, c0 + 1, C) + more.y - 1, C) - c0 + 1;
    // piece 0 in the second slot of range c0, the others in the first slots of the ranges behind it
    const float* ws = a.ws + static_cast<long long>(c0) * 2 * a.slot;
    const auto four = [&](const float* p, int c) { return __ldcg(reinterpret_cast<const float4*>(p + 2 * a.rows) + static_cast<long long>(c) * a.rows + row); };
    float M = -INFINITY, L = 0.0f, v[8] = {};
    for (int k0 = 0; k0 < pieces; k0 += kAhead) {
        float m[kAhead], l[kAhead];
        float4 x[kAhead][2];
#pragma unroll
        for (int e = 0; e < kAhead; ++e) {
            const bool there = k0 + e < pieces;
            const float* p = ws + (k0 + e == 0 ? 1 : static_cast<long long>(k0 + e) * 2) * a.slot;
            m[e] = there ? __ldcg(p + row) : -INFINITY;
            l[e] = there ? __ldcg(p + a.rows + row) : 0.0f;
#pragma unroll
            for (int h = 0; h < 2; ++h) x[e][h] = there ? four(p, c4 + h) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);      // dh % 16 == 0
        }
#pragma unroll
        for (int e = 0; e < kAhead; ++e) {
            if (l[e] == 0.0f) continue;      // the row sees nothing of the piece, whose sums may be 0 * infinity
            const float mx = fmaxf(M, m[e]), base = mx == -INFINITY ? 0.0f : mx;
            const float f = pow2(M - base), g = pow2(m[e] - base);
            M = mx;
            L = fmaf(L, f, l[e] * g);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                v[4 * h] = fmaf(v[4 * h], f, x[e][h].x * g);
                v[4 * h + 1] = fmaf(v[4 * h + 1], f, x[e][h].y * g);
                v[4 * h + 2] = fmaf(v[4 * h + 2], f, x[e][h].z * g);
                v[4 * h + 3] = fmaf(v[4 * h + 3], f, x[e][h].w * g);
            }
        }
    }
    const bool some = L != 0.0f && w.kept;
    const float n = some ? 1.0f / L : 0.0f;
    const long long at = static_cast<long long>(w.token) * a.H + w.head;
    Io* out = static_cast<Io*>(a.out) + at * a.dh + c4 * 4;
    alignas(16) Io y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = from_float<Io>(some ? v[e] * n : 0.0f);
#pragma unroll
    for (int e = 0; e < static_cast<int>(sizeof(Io) / 2); ++e) reinterpret_cast<uint4*>(out)[e] = reinterpret_cast<const uint4*>(y)[e];
    if (c4 == 0 && a.lse) a.lse[at] = some ? (M + log2f(L * a.raise)) * kLn2 : -INFINITY;
}

template <typename Io, int ROWS>
halo_status launch_join(const Args& a, cudaStream_t st) {
    if (a.blocks < 2) return HALO_OK;
    return launch_chained(paged_prompt_join_kernel<Io, ROWS>, dim3(a.blocks - 1, (a.rows + 31) / 32 * ((a.dh + 63) / 64)), 256, 0, st, a);
}

// Thread blocks for a call: as many as are resident together, no more than the line has ranges whatever the lengths are.
inline int line_blocks(const halo_paged_shape& sh, int n_tok, int n_seq, int rows, int tile, int over, int resident) {
    const long long G = sh.n_heads / sh.n_kv_heads, cap = static_cast<long long>(sh.max_pages) * sh.page_size;
    const long long items = (n_tok * G / rows + (n_seq < n_tok ? n_seq : n_tok) + 1) * sh.n_kv_heads;
    const long long most = items * ((cap + tile - 1) / tile + over);
    return static_cast<int>(most < 1 ? 1 : most < resident ? most : resident);
}

// The f32 form (paged_prompt_f32.cu)
size_t f32_workspace(const halo_paged_shape& sh, int n_tok, int n_seq);
halo_status f32_launch(const Args& a, const halo_paged_shape& sh, void* workspace, cudaStream_t st);

}  // namespace prompt
}  // namespace halo
