// halo_paged_prompt_mha: causal attention of packed chunks of new tokens over a paged K/V cache, on the tensor cores
// (tcgen05).  Bound by them for prompts (4 flops per row, key and column of the head), by HBM for a few rows over a long cache.
//
// Per thread block, one to an SM:
//   - warps 8 to 11 gather K and V rows of 128 keys from their pages into a ring of stages (128 keys x 128 columns a stage, in the
//     128-byte swizzle that the tensor cores read) and an item's rows of Q: boxes of a page's rows by the copy engine, or, where
//     pages are no whole number of eight rows, row by row; 8-bit rows row by row as codes, widened to bf16 on the way to a stage;
//   - one thread of warp 12 issues the products: S = Q K^T into tensor memory, O += P V with P in tensor memory;
//   - warp 13 walks along the thread block's part of the work line and tells the others the pieces;
//   - warps 0 to 3 and 4 to 7 take a row per thread: running maximum and sum, P = 2^(S scale - maximum) as bf16 in place of S.
// An item has 256 rows in two streams of 128: while one stream's rows are in the softmax, the other's products run.  Head sizes
// above 128 (whose O fills half of tensor memory) and items of up to 128 rows have one stream with two S buffers instead.
// 128 keys to a tile: with two halves of 64 in flight per stream, so that a stream's own products and softmax overlap, 8192 tokens of
// 16 heads of 128 took 379 us and not 330, a handover costing the same for half the work.
//
// Weights are powers of two relative to a reference: the row's score of the first key, until a tile's weights sum to more than
// 2^20, then its maximum so far.  So O, which would have to be read, multiplied and written back for every new reference, is hardly
// ever touched, and a tile needs no maximum.  All weights are 2^-lower of that (Args), which costs nothing, as it joins the
// reference: 2^20 for each of the most tiles that the table holds, so that a row's weights never sum to more than 1/2 and O overflows for no
// finite values.  What a weight times a value then leaves below 2^-126 can be lost: 2^-80 of the output's own scale at most.
//
// What a row does not see must not reach it.  Weights of 0 see to that but for values that are infinite or NaN.  Where sums come out as
// such over tiles that a row does not see all of, the thread block takes its whole part of the line a second time, with care: such
// values of those tiles (at most three of an item) are taken out of the stages on their way in, and rows that see them
// get their part behind the sums (add_odd).  One NaN at the third position takes 4096 tokens of 32 / 8 heads of 128 from 185 us to 690;
// only values of an item's last tiles are gone through key by key, so a sequence's length adds nothing.  With care in the first place (two warps
// of their own look through those tiles) every call paid: 4096 tokens of 32 heads of 64 took 180 us and not 144, packed prompts 238
// and not 212.
//
// A weight meets the values as one bf16 number: as two, the sums, half of the products, would be twice as many.  Outputs are then
// 0.0023 (relative) from 64 bits where their own rounding alone is 0.0017.
//
// Measured, both kernels, on different GPUs: 4096 tokens, 32 / 8 heads of 128, 180 to 186 us (0.74 to 0.76 PFLOP/s), of 64 143 to 147;
// 8192 tokens, 16 / 4 heads of 128, 310 to 316 (0.88); 512 tokens over 32000 positions in 8 bits, 32 / 8 heads, 347 to 357 (0.77); 7 packed
// prompts of up to 1500 tokens, 32 / 32 heads, 204 to 212 (0.44); 1 to 8 tokens for each of 16 sequences of up to 4000 positions, 32 / 8
// heads, 45 (3.2 TB/s).
// The tensor pipe is active 35 to 39 % of the time and the unit of the powers of two as much: a tile of a stream is 1800 clocks in its
// softmax and then 1900 until its next scores (its sums, their completion, its scores: 1300 if nothing else asked shared memory).
#include <math.h>

#include <type_traits>

#include "prompt_line.cuh"
#include "umma.cuh"

namespace halo {
halo_status check_paged_shape(const halo_paged_shape* s);
halo_status check_eight(const halo_paged_shape& s, const void* K_scale, const void* V_scale);
long long paged_stride(const halo_paged_shape& s);
bool make_bf16_map_nd(CUtensorMap* map, const void* base, int rank, const uint64_t* dims, const uint64_t* strides, const uint32_t* box);

namespace prompt {
namespace {

constexpr int kTile = 128;         // keys
constexpr int kThreads = 512;
// An item's rows, first scores and outputs cost 6000 to 9000 clocks, a tile 4500 (thread blocks of many short items against ones of
// two long items).  With 1 here, 4096 tokens of 32 heads of 64 took 165 us and not 151; with 4, of heads of 128 197 and not 192.
constexpr int kOver = 2;
constexpr float kSum = 1048576.0f;      // 2^20: a tile's weights relative to the reference, together
constexpr int kFlags = 8;          // tiles whose flags are kept

// DP: head size padded to 64, 128 or 256.  EIGHT: 8-bit rows.
template <int DP, bool EIGHT = false>
struct Cfg {
    static constexpr int kStreams = DP > 128 ? 1 : 2;
    static constexpr int kRows = 128 * kStreams;
    static constexpr int kCols = DP < 128 ? DP : 128;         // of a stage
    static constexpr int kParts = DP / kCols;                 // stages of a K or V tile
    static constexpr int kStage = kTile * kCols * 2;
    static constexpr int kStages = DP == 64 ? 8 : EIGHT ? 4 : 5;
    static constexpr int kRaw = EIGHT ? kTile * kCols : 0;    // codes of a stage
    static constexpr int kQTile = 128 * DP * 2;               // Q of a stream
    static constexpr int kQ = kStreams * kQTile;
    // tensor memory: S at 0 and 128, O behind; P in a place of its own where there is one, else over the S that it comes from
    static constexpr int kO = 256;
    static constexpr bool kApart = DP == 64;
    static constexpr int kP = kApart ? 384 : 0, kPStep = kApart ? 64 : 128;
};

struct Flags {
    uint32_t there[kFlags][4];       // which of a tile's keys are there
};
// Tiles of an item that not every row of it sees all of: its rows see up to 255 positions more than its first one.
constexpr int kEdge = 3;
static_assert(kEdge <= 8, "a bit of a byte each");
// S, P and O of a tile hand over through barriers of the lane that it is in: a stream's own in items of two streams, 0 and 2 in
// turn in items of one.  Lanes 1 and 2 share the buffer behind 0, but not the warps that wait: 1 belongs to the second stream's,
// 0 and 2 to the first's, so that nobody waits for a phase of a barrier without having seen the one before it.
constexpr int kLanes = 3;
constexpr int kPieces = 4;         // that a role can be ahead of another
struct Bars {
    uint64_t full[8], empty[8], q_full, q_empty, s_full[kLanes], p_full[kLanes], pv_done[kLanes];
    uint64_t piece_full[4], piece_empty[4];
    uint64_t raw[4];                 // a gathering warp's own: values of which it hands on a part
    uint64_t drained;                // products that were issued before a wait ran out
    uint64_t looked[2 * kPieces];    // with care: all values of a piece have been looked at, odd is there
    uint32_t tmem;
    int abort, again;                // again: a row's sums ask for care
};
__device__ __forceinline__ bool wait(uint64_t* bar, uint32_t phase, int* abort) {
    if (mbar_wait_bounded(bar, phase & 1u, abort)) return true;
    *reinterpret_cast<volatile int*>(abort) = 1;
    return false;
}
// by a whole warp: the same answer in every lane
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t phase, int* abort) {
    return __all_sync(0xffffffffu, wait(bar, phase, abort));
}
// For a piece of work, which another role may take any time over: until it is there or another role has given up.  Who holds a piece
// up is in a wait with a limit, so this one ends too.
__device__ __forceinline__ bool piece_wait(uint64_t* bar, uint32_t phase, volatile int* abort) {
    while (!__all_sync(0xffffffffu, mbar_wait_bounded(bar, phase & 1u, abort)))
        if (__any_sync(0xffffffffu, *abort)) return false;
    return true;
}
// Products issued by one lane of a warp that runs together: D[tmem] (+)= A * B, A in shared memory or (ts) in tensor memory, B in shared memory.  Descriptors by
// their lower words (address, distance of 64-column blocks); the upper word is the same for every tile here.
constexpr uint32_t kDescHigh = (1024u >> 4) | 1u << 14 | 2u << 29;      // eight rows 1024 bytes, descriptor version, 128-byte swizzle
__device__ __forceinline__ void umma_ss(uint32_t lead, uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool accumulate) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t.reg .b64 x, y;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "setp.ne.b32 q, %6, 0;\n\t"
        "mov.b64 x, {%1, %5};\n\t"
        "mov.b64 y, {%2, %5};\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, p;\n\t}" ::"r"(d),
        "r"(a), "r"(b), "r"(idesc), "r"(static_cast<uint32_t>(accumulate)), "n"(kDescHigh), "r"(lead)
        : "memory");
}
__device__ __forceinline__ void umma_ts(uint32_t lead, uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool accumulate) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t.reg .b64 y;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "setp.ne.b32 q, %6, 0;\n\t"
        "mov.b64 y, {%2, %5};\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], y, %3, p;\n\t}" ::"r"(d),
        "r"(a), "r"(b), "r"(idesc), "r"(static_cast<uint32_t>(accumulate)), "n"(kDescHigh), "r"(lead)
        : "memory");
}
__device__ __forceinline__ void commit(uint32_t lead, uint64_t* bar) {
    asm volatile(
        "{\n\t.reg .pred q;\n\t"
        "setp.ne.b32 q, %1, 0;\n\t"
        "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(smem_u32(bar)), "r"(lead)
        : "memory");
}
// 1 in one lane of the warp
__device__ __forceinline__ uint32_t elect() {
    uint32_t e;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(e));
    return e;
}
__device__ __forceinline__ void tmem_st_32x16(uint32_t taddr, const uint32_t (&v)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
        "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]),
        "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
        : "memory");
}
// tcgen05.ld has delivered v: nothing that uses it can be moved in front of the wait
__device__ __forceinline__ void tmem_ld_wait_for(uint32_t (&v)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]), "+r"(v[9]),
                   "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15]), "+r"(v[16]), "+r"(v[17]), "+r"(v[18]),
                   "+r"(v[19]), "+r"(v[20]), "+r"(v[21]), "+r"(v[22]), "+r"(v[23]), "+r"(v[24]), "+r"(v[25]), "+r"(v[26]), "+r"(v[27]),
                   "+r"(v[28]), "+r"(v[29]), "+r"(v[30]), "+r"(v[31])::"memory");
}
__device__ __forceinline__ void tmem_ld_wait_for(uint32_t (&v)[16]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]), "+r"(v[9]),
                   "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15])::"memory");
}
__device__ __forceinline__ uint32_t tmem_ld_word(uint32_t taddr) {
    uint32_t v;
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];" : "=r"(v) : "r"(taddr) : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" : "+r"(v)::"memory");
    return v;
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
// 512 threads start with 128 registers each: 2 * 128 * 176 + 128 * 88 + 128 * 72 = 512 * 128
constexpr int kRowRegs = 176, kCopyRegs = 88, kIssueRegs = 72;

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool valid) {
    const int n = valid ? 16 : 0;   // 0: the 16 bytes are filled with zeros and src is not read
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ uint32_t times_bf16(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
}
// A piece of an item as every role sees it.  One warp walks along the line and hands the pieces to the others through shared memory: the
// walk's state and its divisions, kept by every warp, went to local memory (7 prompts of up to 1500 tokens: 230 us and not 217; 4096
// tokens of 32 heads of 64: 172 and not 160).
struct __align__(16) Piece {
    int n, streams;      // tiles, -1: no more pieces; blocks of 128 rows
    int first_tiles;     // tiles that the first stream takes part in; the second one takes part in all
    int complete;        // all of the item's tiles
    int t0, s, kvh, rb;
    Rows r;
    int reach;           // positions that take part
    __device__ __forceinline__ int tiles(int stream) const { return stream == 0 ? first_tiles : n; }
    // lane of tile j of a stream; its buffer of S and P
    __device__ __forceinline__ int lane(int stream, int j) const { return streams == 2 ? stream : (j & 1) * 2; }
    static __device__ __forceinline__ int buffer(int lane) { return lane != 0; }
    __device__ __forceinline__ float* slot(const Args& a) const { return slot_of(a, t0); }
    // the first of this piece's tiles that the item's first row does not see all of
    __device__ __forceinline__ int edge(const Args& a, int rows) const {
        return max(max(r.len - r.n + 1 + rb * rows / a.G, 0) / kTile - t0, 0);
    }
};
static_assert(sizeof(Piece) == 48, "three 16-byte words");
constexpr int kReaders = 13;       // warps

template <int DP, bool EIGHT>
struct Smem {
    unsigned char q[Cfg<DP, EIGHT>::kQ];
    unsigned char ring[Cfg<DP, EIGHT>::kStages * Cfg<DP>::kStage];
    unsigned char raw[2 * Cfg<DP, EIGHT>::kRaw + 16];
    long long q_row[Cfg<DP>::kRows];     // where the item's rows of q are, -1: none
    Flags flags;
    Piece pieces[kPieces];
    // With care, per piece and gathering warp: bit j, an infinite or NaN value among the warp's 32 keys of tile edge + j.  A gathering warp
    // is at most kPieces pieces ahead of who reads this, and the phases of `looked` of the pieces before are over: the walk waits for
    // every reader before it writes over a piece.
    alignas(4) unsigned char odd[2 * kPieces][4];
    Bars bars;
    long long sh[kThreads / 32 + 3];
};

// The next piece, by a whole warp; false: there is none.
template <int DP, bool EIGHT>
__device__ __forceinline__ bool next_piece(Smem<DP, EIGHT>& sm, uint32_t& k, Piece& p) {
    const uint32_t at = k % kPieces;
    if (!piece_wait(&sm.bars.piece_full[at], k / kPieces, &sm.bars.abort)) return false;
    ++k;
    p = sm.pieces[at];
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(&sm.bars.piece_empty[at]);
    return p.n >= 0;
}
template <int DP, bool EIGHT>
__device__ void walk_line(const Args& a, Smem<DP, EIGHT>& sm, Walk<Cfg<DP>::kRows, kTile, kOver> w, long long total) {
    using C = Cfg<DP>;
    for (uint32_t k = 0;; ++k) {
        Piece p = {};
        p.n = -1;
        if (w.left > 0) {
            const int base = w.rb * C::kRows, all = w.r.n * a.G;
            p.n = w.reach > 0 ? w.t1 - w.t0 : 0;
            p.streams = C::kStreams == 2 && base + 128 < all ? 2 : 1;
            p.first_tiles = p.n;
            if (p.streams == 2) {      // the first stream's last row may not see the last tiles
                const int sees = w.r.len - w.r.n + 1 + (base + 127) / a.G;
                p.first_tiles = min(p.n, max((sees + kTile - 1) / kTile - w.t0, 0));
            }
            p.complete = w.complete();
            p.t0 = w.t0;
            p.s = w.s;
            p.kvh = w.kvh;
            p.rb = w.rb;
            p.r = w.r;
            p.reach = w.reach;
        }
        const uint32_t at = k % kPieces;
        if (!piece_wait(&sm.bars.piece_empty[at], k / kPieces + 1, &sm.bars.abort)) return;      // the phase before
        if ((threadIdx.x & 31) == 0) {
            sm.pieces[at] = p;
            mbar_arrive(&sm.bars.piece_full[at]);
            if (w.left > 0 && w.opens()) a.openings[blockIdx.x] = w.opening(total);
        }
        if (p.n < 0) return;
        w.next(a);
    }
}

// ---- gathering ------------------------------------------------------------------------------------------------------------------

// What the copy engine is told: the caches as [page][K/V head][row][column], boxes of box_rows rows of a page (a power of two from 8
// to 32 that divides the page) x 64 columns; q as [token][head][column], boxes of 128 rows x 64 columns.
struct Maps {
    CUtensorMap q, K, V;
    int box_rows, whole_q;      // 0: rows are gathered one by one (pages of odd sizes, head sizes below 64, head counts that do not divide 128)
};

// Infinite and NaN values of `rows` rows of a stage, 16 bytes of a row to a lane and eight rows 1024 bytes apart, become zeros; true: there were
// some of this lane's.  at: of row r of the first ones; step: rows that a warp has at once.
__device__ __forceinline__ bool purge(uint32_t at, int r, int chunk, int rows, int step) {
    bool some = false;
    for (; r < rows; r += step) {
        const uint32_t word = at + r * 128 + ((chunk ^ (r & 7)) << 4);
        uint32_t w[4], top = 0;
        asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(word) : "memory");
#pragma unroll
        for (int e = 0; e < 4; ++e) top |= (w[e] & 0x7f807f80u) + 0x00800080u;      // an exponent of ones carries into the sign
        if (!(top & 0x80008000u)) continue;
        some = true;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if ((w[e] & 0x7f80u) == 0x7f80u) w[e] &= 0xffff0000u;
            if ((w[e] & 0x7f800000u) == 0x7f800000u) w[e] &= 0x0000ffffu;
        }
        asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(word), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
    }
    return some;
}

template <int DP, bool EIGHT, bool CARE>
struct Gather {
    using C = Cfg<DP, EIGHT>;
    [[maybe_unused]] static constexpr int kChunks = C::kCols / 8;           // 16-byte chunks of a stage's row
    [[maybe_unused]] static constexpr int kAtOnce = 32 / kChunks;           // rows per instruction
    const Args& a;
    const Maps& maps;
    Smem<DP, EIGHT>& sm;
    int* abort;
    const int warp, lane;
    uint32_t fill = 0, cleared = 0;      // stages filled so far, and stages of values that something was taken out of
    uint32_t odd = 0;                    // this lane's part of sm.odd of the piece
    uint32_t piece_asked = 0;            // pieces whose rows of q were asked for
    uint32_t waiting0 = 0, waiting1 = 0;      // barriers of row copies that are on their way
    int n_waiting = 0;
    bool alive = true;

    __device__ __forceinline__ Gather(const Args& a_, const Maps& m_, Smem<DP, EIGHT>& sm_)
        : a(a_), maps(m_), sm(sm_), abort(&sm_.bars.abort), warp((threadIdx.x >> 5) & 3), lane(threadIdx.x & 31) {}
    __device__ __forceinline__ void signal(uint32_t bar) {
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
    }
    __device__ __forceinline__ void flush() {
        if (n_waiting == 0) return;
        cp_wait<0>();
        signal(waiting0);
        if (n_waiting > 1) signal(waiting1);
        n_waiting = 0;
    }
    // row copies that were just issued: the ones two before them are complete behind the wait
    __device__ __forceinline__ void issued(uint32_t bar) {
        cp_commit();
        if (n_waiting == 2) {
            cp_wait<2>();
            signal(waiting0);
            waiting0 = waiting1;
            waiting1 = bar;
        } else {
            (n_waiting == 0 ? waiting0 : waiting1) = bar;
            ++n_waiting;
        }
    }
    __device__ __forceinline__ bool ready(uint64_t* bar, uint32_t phase) { return __all_sync(0xffffffffu, mbar_try_wait(bar, phase & 1u)); }
    __device__ __forceinline__ void await(uint64_t* bar, uint32_t phase) {
        if (ready(bar, phase)) return;
        flush();             // nobody frees anything before it has what is on its way
        alive = warp_wait(bar, phase, abort) && alive;
    }
    // chunk c of row r of this warp's 32 rows of a stage: block of 64 columns, row of 128 bytes, chunk of 16 turned by the row
    __device__ __forceinline__ uint32_t place(uint32_t stage, int r, int c) const {
        return stage + (c >> 3) * (kTile * 128) + (warp * 32 + r) * 128 + (((c & 7) ^ (r & 7)) << 4);
    }
    // rows of this warp's that are not there become zeros: a box brings whatever the page holds
    __device__ __forceinline__ void clear(uint32_t stage, uint32_t there) {
        const int c = lane % kChunks, r0 = lane / kChunks;
        for (int i = 0; i < 32 / kAtOnce; ++i) {
            const int r = i * kAtOnce + r0;
            if (!(there >> r & 1u)) asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(place(stage, r, c)), "r"(0) : "memory");
        }
    }
    // values of the edge-th tile that not every row sees all of
    __device__ __forceinline__ void look(uint32_t stage, int part, int edge) {
        const int c = lane % kChunks;
        if (part * C::kCols + c * 8 < a.dh && purge(stage + (c >> 3) * (kTile * 128) + warp * (32 * 128), lane / kChunks, c & 7, 32, kAtOnce)) odd |= 1u << edge;
    }
    // 128 keys x kCols columns.  page: of this lane's key, n_pages: none, which reads as zeros; pos: of the tile; there: which of
    // this warp's rows are, the others have to be zeros; edge: as in look, -1: none.
    __device__ __forceinline__ void stage(const CUtensorMap* map, const void* cache, int page, int pos, int kvh, int part, uint32_t there, int edge) {
        const uint32_t s = fill % C::kStages, phase = fill / C::kStages;
        await(&sm.bars.empty[s], phase + 1);     // the phase before: passes at once the first time
        if (!alive) return;
        ++fill;
        const uint32_t dst = smem_u32(sm.ring) + s * C::kStage, full = smem_u32(&sm.bars.full[s]);
        const int first = pos + warp * 32;       // of this warp's keys
        if (maps.box_rows) {
            const int boxes = 32 / maps.box_rows, blocks = min(C::kCols / 64, (a.dh - part * C::kCols + 63) / 64);
            const int box = lane % boxes, block = lane / boxes, row = box * maps.box_rows;
            const int from = __shfl_sync(0xffffffffu, page, row), at = first + row;
            const bool own = there != 0xffffffffu || edge >= 0;
            uint64_t* bar = own ? &sm.bars.raw[warp] : &sm.bars.full[s];
            if (lane == 0) mbar_arrive_expect_tx(bar, blocks * 32 * 128);
            __syncwarp();
            if (block < blocks)
                tma_load_4d(dst + block * (kTile * 128) + (warp * 32 + row) * 128, map, part * C::kCols + block * 64,
                            a.page_shift >= 0 ? at & (a.page_size - 1) : at % a.page_size, kvh, from, smem_u32(bar));
            if (own) {
                alive = warp_wait(bar, cleared++, abort) && alive;
                clear(dst, there);
                if (edge >= 0) look(dst, part, edge);      // a lane has the words that it has cleared
                signal(full);
            }
            return;
        }
        const int mine = first + lane, in_page = a.page_shift >= 0 ? mine & (a.page_size - 1) : mine % a.page_size;
        const long long at = page < a.n_pages ? static_cast<long long>(page) * a.page_stride + (static_cast<long long>(kvh) * a.page_size + in_page) * a.dh : -1;
        const int c = lane % kChunks, r0 = lane / kChunks, col = part * C::kCols + c * 8;
        const bool in = col < a.dh;
        const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(cache) + col;
#pragma unroll
        for (int i = 0; i < 32 / kAtOnce; ++i) {
            const int r = i * kAtOnce + r0;
            const long long from = __shfl_sync(0xffffffffu, at, r);
            if (in) cp_async16(place(dst, r, c), from >= 0 ? src + from : src, from >= 0);
        }
        if (edge < 0) {
            issued(full);
            return;
        }
        cp_commit();
        cp_wait<0>();
        flush();
        look(dst, part, edge);      // a lane has the words that it has copied
        signal(full);
    }
    __device__ __forceinline__ void queries(const Piece& p, uint32_t piece) {
        await(&sm.bars.q_empty, piece + 1);
        if (!alive) return;
        ++piece_asked;
        const uint32_t q = smem_u32(sm.q), full = smem_u32(&sm.bars.q_full);
        if (maps.whole_q) {      // tokens behind the sequence's last come along, and go nowhere
            const int blocks = (a.dh + 63) / 64, boxes = p.streams * blocks, mine = (boxes - warp + 3) / 4;
            if (lane == 0) {
                if (mine > 0) mbar_arrive_expect_tx(&sm.bars.q_full, mine * 128 * 128);
                else mbar_arrive(&sm.bars.q_full);
            }
            __syncwarp();
            if (lane < mine) {
                const int box = lane * 4 + warp, t = box / blocks, block = box - t * blocks;
                const int token = p.r.first + (p.rb * C::kRows + t * 128) / a.G;
                tma_load_3d(q + t * C::kQTile + block * (128 * 128), &maps.q, block * 64, p.kvh * a.G, token, full);
            }
            return;
        }
        constexpr int kOwn = C::kRows / 4, kWide = DP / 8, kRowsAtOnce = 32 / kWide;      // rows of a warp
#pragma unroll
        for (int i = lane; i < kOwn; i += 32) {
            const Row r = row_at<C::kRows>(a, p.r, p.kvh, p.rb, warp * kOwn + i);
            sm.q_row[warp * kOwn + i] = r.there ? static_cast<long long>(r.token) * a.q_stride + static_cast<long long>(r.head) * a.dh : -1;
        }
        __syncwarp();
        const int c = lane % kWide, r0 = lane / kWide;
        const bool in = c * 8 < a.dh;
        const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(a.q) + c * 8;
        const uint32_t dst = q + (c >> 3) * (128 * 128) + ((c & 7) << 4);
#pragma unroll 4
        for (int i = 0; i < kOwn / kRowsAtOnce; ++i) {
            const int r = warp * kOwn + i * kRowsAtOnce + r0;
            const long long from = sm.q_row[r];
            if (in) cp_async16((dst + (r >> 7) * C::kQTile + (r & 127) * 128) ^ ((r & 7) << 4), from >= 0 ? src + from : src, from >= 0);
        }
        __syncwarp();      // q_row may be written again
        issued(full);
        flush();           // the first scores wait for them
    }
    // 8-bit rows: codes of this warp's 32 keys into a slot of their own, 16 a lane and instruction
    [[maybe_unused]] static constexpr int kCodes = C::kCols / 16, kCodeRows = 32 / kCodes;
    __device__ __forceinline__ uint32_t code_place(int slot, int r) const {
        return smem_u32(sm.raw) + slot * C::kRaw + (warp * 32 + r) * C::kCols + (lane % kCodes) * 16;
    }
    __device__ __forceinline__ void codes(const void* cache, long long at, int part, int slot) {
        const int col = part * C::kCols + (lane % kCodes) * 16;
        const uint8_t* src = static_cast<const uint8_t*>(cache) + col;
#pragma unroll
        for (int i = 0; i < 32 / kCodeRows; ++i) {
            const int r = i * kCodeRows + lane / kCodes;
            const long long from = __shfl_sync(0xffffffffu, at, r);
            const bool there = from >= 0 && col < a.dh;
            cp_async16(code_place(slot, r), there ? src + from : src, there);
        }
        cp_commit();
    }
    // Words of a stage to bf16, four loads ahead of their conversions: one behind the other, a load's and its conversion's latencies
    // add up (512 tokens over 32000 positions 496 us and not 362; all eight ahead 359).
    template <bool FAR>
    __device__ __forceinline__ void spread(uint32_t dst, uint32_t steps, int slot) {
        constexpr int kAhead = 4;
        const int c = lane % kCodes;
#pragma unroll
        for (int i0 = 0; i0 < 32 / kCodeRows; i0 += kAhead) {
            uint32_t w[kAhead][4], by[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int r = (i0 + i) * kCodeRows + lane / kCodes;
                asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w[i][0]), "=r"(w[i][1]), "=r"(w[i][2]), "=r"(w[i][3]) : "r"(code_place(slot, r)));
                by[i] = __shfl_sync(0xffffffffu, steps, r);
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int r = (i0 + i) * kCodeRows + lane / kCodes;
                const uint32_t by_one = __byte_perm(by[i], by[i], 0x1010), by_two = __byte_perm(by[i], by[i], 0x3232);
                uint32_t o[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const uint32_t t = __byte_perm(w[i][k >> 1], 0, k & 1 ? 0x3424 : 0x1404);      // a code in the upper byte of each half
                    o[k] = times_bf16(((t >> 4) & 0x07f007f0u) | (t & 0x80008000u), by_one);
                    if (FAR) o[k] = times_bf16(o[k], by_two);
                }
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(place(dst, r, 2 * c + h)), "r"(o[4 * h]), "r"(o[4 * h + 1]),
                                 "r"(o[4 * h + 2]), "r"(o[4 * h + 3]) : "memory");
            }
        }
    }
    // ... and on to a stage as bf16.  A code's bits are a bf16 number's exponent and significand, of 2^-120 of its value; the row's power
    // of two puts that right: without rounding, as every value of a row is a bf16 number.  byte: of this lane's key's row.
    __device__ __forceinline__ void widen(uint32_t byte, int slot) {
        const uint32_t s = fill % C::kStages, phase = fill / C::kStages;
        await(&sm.bars.empty[s], phase + 1);
        if (!alive) return;
        ++fill;
        const uint32_t dst = smem_u32(sm.ring) + s * C::kStage;
        // 2^(120 + e), in two steps where that is past the largest power; 0 for a row that is not there
        const int e = static_cast<int>(byte) - 127;
        const float one = byte == 0 ? 0.0f : byte == kEightNan ? __uint_as_float(0x7fc00000u) : eight_power(120 + min(e, 7));
        const float two = byte == kEightNan ? 1.0f : eight_power(max(e, 7) - 7);
        const uint32_t steps = pack_bf16(one, two);
        if (__any_sync(0xffffffffu, two != 1.0f)) spread<true>(dst, steps, slot);
        else spread<false>(dst, steps, slot);
        signal(smem_u32(&sm.bars.full[s]));
    }
    __device__ void run() {
        bool bad = false;
        uint32_t tile = 0, piece = 0, k = 0;
        for (Piece p; alive && next_piece(sm, k, p);) {
            const auto page_of = [&](int j) {     // of this lane's key of the j-th tile
                const int at = (p.t0 + j) * kTile + warp * 32 + lane;
                if (j >= p.n || at >= p.reach) return -1;
                return ldg_waited(a.table + static_cast<long long>(p.s) * a.max_pages + (a.page_shift >= 0 ? at >> a.page_shift : at / a.page_size));
            };
            int page = page_of(0);
            [[maybe_unused]] const int first_edge = CARE ? p.edge(a, C::kRows) : 0;
            odd = 0;
            // ahead of the keys where the item before is through with its own, else behind the first keys and values
            bool asked = p.n == 0;
            if (!asked && ready(&sm.bars.q_empty, piece + 1)) {
                queries(p, piece);
                asked = true;
            }
            if constexpr (EIGHT) {
                // a stage's codes are on their way while the ones before them are widened
                constexpr int kFills = 2 * C::kParts;
                long long at = -1;               // of this lane's key's rows in the tile whose codes are asked for
                uint32_t kb = 0, vb = 0;         // their scale bytes
                const auto ask = [&](int f) {    // the codes of the f-th stage of the piece
                    const int j = f / kFills, h = f % kFills;
                    if (h == 0) {
                        const int pos = (p.t0 + j) * kTile + warp * 32 + lane;
                        const bool in = pos < p.reach, ok = in && page >= 0 && page < a.n_pages;
                        bad |= in && !ok;
                        const int in_page = a.page_shift >= 0 ? pos & (a.page_size - 1) : pos % a.page_size;
                        const long long row = static_cast<long long>(p.kvh) * a.page_size + in_page;
                        at = ok ? page * a.page_stride + row * a.dh : -1;
                        kb = vb = 0;
                        if (ok) {
                            kb = ldg_waited(a.K_scale + static_cast<long long>(page) * a.Hk * a.page_size + row);
                            vb = ldg_waited(a.V_scale + static_cast<long long>(page) * a.Hk * a.page_size + row);
                        }
                        page = page_of(j + 1);
                    }
                    codes(h < C::kParts ? a.K : a.V, at, h % C::kParts, f & 1);
                };
                if (p.n > 0) ask(0);
                for (int f = 0; f < p.n * kFills && alive; ++f) {
                    const int h = f % kFills;
                    const uint32_t byte = h < C::kParts ? kb : vb, there = __ballot_sync(0xffffffffu, at >= 0);
                    if (h == 0 && lane == 0) sm.flags.there[tile % kFlags][warp] = there;
                    if (h == kFills - 1) ++tile;
                    if (f + 1 < p.n * kFills) {
                        ask(f + 1);
                        cp_wait<1>();
                    } else {
                        cp_wait<0>();
                    }
                    const bool out = CARE && h >= C::kParts && f / kFills >= first_edge && byte == kEightNan;      // a row of NaN
                    if (out) odd |= 1u << (f / kFills - first_edge);
                    widen(out ? 0u : byte, f & 1);
                    if (f == kFills - 1 && !asked && alive) {
                        queries(p, piece);
                        asked = true;
                    }
                }
            } else {
            for (int j = 0; j < p.n && alive; ++j, ++tile) {
                const int next = page_of(j + 1);
                const int pos = (p.t0 + j) * kTile;
                const bool in = pos + warp * 32 + lane < p.reach, ok = in && page >= 0 && page < a.n_pages;
                bad |= in && !ok;
                const uint32_t there = __ballot_sync(0xffffffffu, ok);
                // the slot's last readers are done: their P went into a product behind which stages were freed for this tile
                if (lane == 0) sm.flags.there[tile % kFlags][warp] = there;
                const int from = ok ? page : a.n_pages;
#pragma unroll
                for (int h = 0; h < C::kParts; ++h) stage(&maps.K, a.K, from, pos, p.kvh, h, 0xffffffffu, -1);      // scores of absent keys are masked
#pragma unroll
                for (int h = 0; h < C::kParts; ++h) stage(&maps.V, a.V, from, pos, p.kvh, h, there, CARE ? j - first_edge : -1);
                if (!asked && alive) {
                    queries(p, piece);
                    asked = true;
                }
                page = next;
            }
            }
            if (p.n > 0) ++piece;
            if (CARE) {
                const uint32_t at = (k - 1) % (2 * kPieces), all = __reduce_or_sync(0xffffffffu, odd);
                if (lane == 0) {
                    sm.odd[at][warp] = static_cast<unsigned char>(all);
                    mbar_arrive(&sm.bars.looked[at]);
                }
            }
        }
        flush();
        cp_wait<0>();
        if (lane == 0) {     // for land()
            sm.sh[warp] = fill;
            sm.sh[4 + warp] = piece_asked;
            sm.sh[8 + warp] = cleared;
        }
        if (__any_sync(0xffffffffu, bad) && lane == 0) flag_status(a.status, HALO_DEV_BAD_INDEX);
    }
};

// ---- products -------------------------------------------------------------------------------------------------------------------

template <int N>
using Const = std::integral_constant<int, N>;

// One warp, one lane of which issues.  Lanes (of barriers) are constants, so that counters and addresses stay in registers: the
// tensor cores take a product of 16 columns in 64 clocks, and one must not take longer to issue.  Two streams take fixed turns:
// with tests of what is ready instead, 8192 tokens of 16 heads of 128 took 330 us and not 325, 4096 of 32 heads of 64 took 187 and
// not 173; with a warp for each stream, whose products then share the tensor cores, 393 and 198.  One stream goes by those
// tests: 4096 tokens of 16 / 4 heads of 256 take 247 us, in fixed turns 286.
template <int DP, bool EIGHT>
struct Issue {
    using C = Cfg<DP, EIGHT>;
    const Args& a;
    Smem<DP, EIGHT>& sm;
    Bars& bars;
    int* abort;
    const uint32_t lead, tmem, q0, ring, idesc_s;
    uint32_t first_fill = 0, use0 = 0, use1 = 0, use2 = 0;      // stages of the pieces before; tiles of each lane so far
    int last = 1;                                               // lane that the second buffer was used in last

    __device__ __forceinline__ Issue(const Args& a_, Smem<DP, EIGHT>& sm_)
        : a(a_), sm(sm_), bars(sm_.bars), abort(&sm_.bars.abort), lead(elect()), tmem(sm_.bars.tmem), q0(smem_u32(sm_.q) >> 4),
          ring(smem_u32(sm_.ring) >> 4),
          // a negative scale: -Q instead, so that the largest score stays the largest product
          idesc_s(umma_idesc_bf16(128, kTile, false) | (a_.scale_log2 < 0.0f ? 1u << 13 : 0u)) {}
    static __device__ __forceinline__ bool done(uint64_t* bar, uint32_t phase) { return __all_sync(0xffffffffu, mbar_test(bar, phase & 1u)); }
    // the K (v = 0) or V (1) stages of tile j
    __device__ __forceinline__ bool there(int j, int v) const {
        bool all = true;
#pragma unroll
        for (int h = 0; h < C::kParts; ++h) {
            const uint32_t f = first_fill + (j * 2 + v) * C::kParts + h;
            all = all && done(&bars.full[f % C::kStages], f / C::kStages);
        }
        return all;
    }
    template <int b>
    __device__ __forceinline__ uint32_t& use() { return b == 0 ? use0 : b == 1 ? use1 : use2; }
    // S of lane b may be written: the buffer's last P has been read (its S, where P lies apart and the same warps write the next)
    template <int b>
    __device__ __forceinline__ bool free_scores() {
        const int was = b == 0 ? 0 : last;
        const uint32_t used = was == 0 ? use0 : was == 1 ? use1 : use2;
        if (used == 0) return true;
        return C::kApart && was == b ? done(&bars.p_full[b], used - 1)
                                     : done(was == 0 ? &bars.pv_done[0] : was == 1 ? &bars.pv_done[1] : &bars.pv_done[2], used - 1);
    }
    // stream t, lane b, tile j; end: nobody else needs the stages
    template <int t, int b>
    __device__ __forceinline__ void scores(int j, bool end) {
        tcgen05_fence_after_sync();
        const uint32_t d = tmem + (b != 0) * 128;
        if (b != 0) last = b;
        ++use<b>();
        // what this thread has seen of the gathering warps, the tile's flags among it; in front of the products, as what follows
        // them waits until the tensor cores have taken them
        if (lead) mbar_arrive(&bars.s_full[b]);
        __syncwarp();
#pragma unroll
        for (int h = 0; h < C::kParts; ++h) {
            const uint32_t s = (first_fill + j * 2 * C::kParts + h) % C::kStages;
            const uint32_t q = q0 + ((t * C::kQTile + h * (C::kCols / 64) * (128 * 128)) >> 4), k = ring + s * (C::kStage >> 4);
            const int steps = (a.dh - h * C::kCols) / 16;
            if (steps >= C::kCols / 16) {
#pragma unroll
                for (int e = 0; e < C::kCols / 16; ++e)
                    umma_ss(lead, d, q + (e >> 2) * 1024 + (e & 3) * 2, k + (e >> 2) * 1024 + (e & 3) * 2, idesc_s, h > 0 || e > 0);
            } else {
                for (int e = 0; e < steps; ++e)
                    umma_ss(lead, d, q + (e >> 2) * 1024 + (e & 3) * 2, k + (e >> 2) * 1024 + (e & 3) * 2, idesc_s, h > 0 || e > 0);
            }
            if (end) commit(lead, &bars.empty[s]);
        }
        commit(lead, &bars.s_full[b]);
    }
    template <int t, int b>
    __device__ __forceinline__ void sums(int j, bool end) {
        tcgen05_fence_after_sync();
#pragma unroll
        for (int h = 0; h < C::kParts; ++h) {
            const uint32_t s = (first_fill + (j * 2 + 1) * C::kParts + h) % C::kStages;
            const uint32_t idesc = umma_idesc_bf16(128, min(a.dh - h * C::kCols, C::kCols), true);
            const uint32_t v = (ring + s * (C::kStage >> 4)) | ((kTile * 128) >> 4) << 16;
#pragma unroll
            for (int e = 0; e < kTile / 16; ++e)
                umma_ts(lead, tmem + C::kO + t * DP + h * C::kCols, tmem + C::kP + (b != 0) * C::kPStep + e * 8, v + e * 128, idesc, j > 0 || e > 0);
            if (end) commit(lead, &bars.empty[s]);
        }
        commit(lead, &bars.pv_done[b]);
    }
    __device__ __forceinline__ bool await_stage(int j, int v) {      // items of two streams have a stage to a tile
        const uint32_t f = first_fill + j * 2 + v;
        return warp_wait(&bars.full[f % C::kStages], f / C::kStages, abort);
    }
    // The next turn of stream t of two, whose lane t is: sums of tile j and the scores of the one behind it.
    template <int t>
    __device__ __forceinline__ bool turn(int j, int n, int on) {
        if (j >= n) return true;
        const bool more = j + 1 < n;
        // the second stream's stages are the first one's, where that had them
        if (!(t == 1 && j < on) && !await_stage(j, 1)) return false;
        if (more && !(t == 1 && j + 1 < on) && !await_stage(j + 1, 0)) return false;
        if (!warp_wait(&bars.p_full[t], use<t>() - 1, abort)) return false;
        if (C::kApart && more) scores<t, t>(j + 1, t == 1 || j + 1 >= on);      // S has been read: its place is free
        sums<t, t>(j, t == 1 || j >= on);
        if (!C::kApart && more) {
            if (!warp_wait(&bars.pv_done[t], use<t>() - 1, abort)) return false;
            scores<t, t>(j + 1, t == 1 || j + 1 >= on);
        }
        return true;
    }
    // An item of two streams, which take turns: while the tensor cores have one's products, the other is in its softmax.
    __device__ __forceinline__ bool turns(int n0, int n1) {
        if (use0 > 0 && !warp_wait(&bars.pv_done[0], use0 - 1, abort)) return false;
        const uint32_t used = last == 1 ? use1 : use2;
        if (used > 0 && !warp_wait(last == 1 ? &bars.pv_done[1] : &bars.pv_done[2], used - 1, abort)) return false;
        if (!await_stage(0, 0)) return false;
        if (n0 > 0) scores<0, 0>(0, false);
        scores<C::kStreams - 1, 1>(0, true);
        if (n1 == 1) commit(lead, &bars.q_empty);
        for (int j = 0; j < n1; ++j) {
            if (!turn<0>(j, n0, n1)) return false;
            if (!turn<C::kStreams - 1>(j, n1, n0)) return false;
            if (j + 2 == n1) commit(lead, &bars.q_empty);      // the last scores: n0 <= n1
        }
        return true;
    }
    // One step of a stream on its own, lanes 0 and 2 in turn
    __device__ __forceinline__ bool step_alone(int& q, int& s, int n) {
        if (s < q && done(s & 1 ? &bars.p_full[2] : &bars.p_full[0], (s & 1 ? use2 : use0) - 1) && there(s, 1)) {
            if (s & 1) sums<0, 2>(s, true);
            else sums<0, 0>(s, true);
            ++s;
            return true;
        }
        if (q < n && q - s < 2 && (q & 1 ? free_scores<2>() : free_scores<0>()) && there(q, 0)) {
            if (q & 1) scores<0, 2>(q, true);
            else scores<0, 0>(q, true);
            ++q;
            return true;
        }
        return false;
    }
    // An item of one stream
    __device__ __forceinline__ bool alone(int n) {
        int q = 0, s = 0;      // scores and sums issued
        bool asked = false;
        long long since = 0;
        uint32_t idle = 0;
        while (s < n) {
            const bool any = step_alone(q, s, n);
            if (!asked && q == n) {
                commit(lead, &bars.q_empty);
                asked = true;
            }
            if (any) {
                idle = 0;
            } else if ((++idle & 255u) == 0u) {      // bounded, as every wait
                const long long now = clock64();
                if (idle == 256u) since = now;
                const bool stop = *reinterpret_cast<volatile int*>(abort) || now - since > kWaitLimitCycles;
                if (__any_sync(0xffffffffu, stop)) {
                    *reinterpret_cast<volatile int*>(abort) = 1;
                    return false;
                }
            }
        }
        return true;
    }
    __device__ void run() {
        if (all()) return;
        int never = 0;       // products that are on their way read shared memory and write tensor memory
        commit(lead, &bars.drained);
        mbar_wait_bounded(&bars.drained, 0, &never);
        __syncwarp();
    }
    __device__ __forceinline__ bool all() {
        uint32_t piece = 0, k = 0;
        for (Piece p; next_piece(sm, k, p);) {
            if (p.n == 0) continue;
            if (!warp_wait(&bars.q_full, piece++, abort)) return false;
            if (!(C::kStreams == 2 && p.streams == 2 ? turns(p.first_tiles, p.n) : alone(p.n))) return false;
            first_fill += p.n * 2 * C::kParts;
        }
        // every stage is free again: no arrival is on its way
        bool ok = !*reinterpret_cast<volatile int*>(abort);      // next_piece may have given up
        for (uint32_t f = first_fill > C::kStages ? first_fill - C::kStages : 0; ok && f < first_fill; ++f)
            ok = warp_wait(&bars.empty[f % C::kStages], f / C::kStages, abort);
        if (ok && piece > 0) ok = warp_wait(&bars.q_empty, piece - 1, abort);
        if (ok && use0 > 0) ok = warp_wait(&bars.pv_done[0], use0 - 1, abort);
        if (ok && use1 > 0) ok = warp_wait(&bars.pv_done[1], use1 - 1, abort);
        if (ok && use2 > 0) ok = warp_wait(&bars.pv_done[2], use2 - 1, abort);
        return __all_sync(0xffffffffu, ok);
    }
};

// ---- two fp32 numbers at a time ----
using Pair = unsigned long long;
__device__ __forceinline__ Pair pair_of(float a, float b) {
    Pair r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float2 both(Pair x) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(x));
    return r;
}
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) {
    Pair r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ Pair add2(Pair a, Pair b) {
    Pair r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ Pair twice(float a) { return pair_of(a, a); }
// NaN if one of them is
__device__ __forceinline__ float max2(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
// ---- rows -----------------------------------------------------------------------------------------------------------------------

// One element of the caches
__device__ __forceinline__ float cache_at(const Args& a, const void* cache, const uint8_t* scale, int page, int kvh, int in_page, int c) {
    const long long row = static_cast<long long>(kvh) * a.page_size + in_page, at = page * a.page_stride + row * a.dh + c;
    if (!a.K_scale) return __bfloat162float(static_cast<const __nv_bfloat16*>(cache)[at]);
    float f[4];
    eight_widen(static_cast<const uint8_t*>(cache)[at], f);
    return f[0] * eight_unit(scale[static_cast<long long>(page) * a.Hk * a.page_size + row]);
}

// Infinite and NaN values of a piece's last tiles, which the gathering warps have taken out: their parts are added to O in tensor memory where a
// row sees them.  By a whole warp, a row per lane, which sees `own` positions (0: no row); bounded by kEdge tiles.  k: number of the piece; n:
// tiles of the row's stream.
template <int DP, bool EIGHT>
__device__ __forceinline__ bool add_odd(const Args& a, Smem<DP, EIGHT>& sm, const Piece& p, uint32_t k, int n, int token, int head, int own, float base,
                                     uint32_t o_addr) {
    const uint32_t slot = k % (2 * kPieces);
    if (!warp_wait(&sm.bars.looked[slot], k / (2 * kPieces), &sm.bars.abort)) return false;
    const int edge = p.edge(a, Cfg<DP>::kRows);
    const uint32_t odd = *reinterpret_cast<const volatile uint32_t*>(sm.odd[slot]);
    if (odd == 0) return true;
    const int lane = threadIdx.x & 31;
    const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(a.q) + static_cast<long long>(token) * a.q_stride + static_cast<long long>(head) * a.dh;
    for (int at = edge * kTile; at < n * kTile; ++at) {
        const int j = at / kTile, of = at % kTile, pos = p.t0 * kTile + at;
        if (!(odd >> (of / 32 * 8 + j - edge) & 1u) || pos >= p.reach) continue;
        const int pi = pos / a.page_size, in_page = pos - pi * a.page_size;
        const int page = ldg_waited(a.table + static_cast<long long>(p.s) * a.max_pages + pi);
        if (page < 0 || page >= a.n_pages) continue;
        bool here = false;
        for (int c = lane; c < a.dh; c += 32) here |= !(fabsf(cache_at(a, a.V, a.V_scale, page, p.kvh, in_page, c)) < INFINITY);
        const bool sees = pos < own;
        if (!__any_sync(0xffffffffu, here) || !__any_sync(0xffffffffu, sees)) continue;
        float score = 0.0f;
        if (sees)
            for (int c = 0; c < a.dh; ++c) score = fmaf(__bfloat162float(q[c]), cache_at(a, a.K, a.K_scale, page, p.kvh, in_page, c), score);
        const float w = __bfloat162float(__float2bfloat16_rn(pow2(fmaf(score, a.scale_log2, -base))));
        for (int c = 0; c < a.dh; c += 16) {
            uint32_t o[16];
            __syncwarp();
            tmem_ld_32x16(o_addr + c, o);
            tmem_ld_wait_for(o);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const float v = cache_at(a, a.V, a.V_scale, page, p.kvh, in_page, c + e);
                if (sees && !(fabsf(v) < INFINITY)) o[e] = __float_as_uint(fmaf(w, v, __uint_as_float(o[e])));
            }
            __syncwarp();
            tmem_st_32x16(o_addr + c, o);
            tmem_st_wait();
        }
    }
    return true;
}

// Four lanes with four 16-byte words each, of the rows l, to a word each of four rows: 2 x 2 blocks, then halves of them.  Stores of
// 64 bytes of a row by four neighbours instead of 16 bytes of 32 rows.
__device__ __forceinline__ void turn_words(uint4 (&w)[4], int lane) {
#pragma unroll
    for (int d = 1; d < 4; d <<= 1) {
        const bool upper = lane & d;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (i & d) continue;
            uint4 send = upper ? w[i] : w[i + d];
            send.x = __shfl_xor_sync(0xffffffffu, send.x, d);
            send.y = __shfl_xor_sync(0xffffffffu, send.y, d);
            send.z = __shfl_xor_sync(0xffffffffu, send.z, d);
            send.w = __shfl_xor_sync(0xffffffffu, send.w, d);
            if (upper) w[i] = send;
            else w[i + d] = send;
        }
    }
}

template <int DP, bool EIGHT, bool CARE>
__device__ __forceinline__ void softmax_rows(const Args& a, Smem<DP, EIGHT>& sm) {
    using C = Cfg<DP>;
    constexpr float kSlack = 8.0f;            // powers of two that a reference may lag behind where it is looked at
    const float most_sum = kSum * exp2f(-a.lower);      // what a tile's weights may sum to before it is
    Bars& bars = sm.bars;
    int* abort = &bars.abort;
    const int t = threadIdx.x >> 7, i = threadIdx.x & 127, lane = threadIdx.x & 31, item_row = t * 128 + i;
    const uint32_t lanes = bars.tmem + (static_cast<uint32_t>(i & ~31) << 16);
    const uint32_t o_addr = lanes + C::kO + t * DP;
    const float scale = fabsf(a.scale_log2);
    uint32_t tile = 0, used[kLanes] = {0, 0, 0};      // tiles so far; of the lanes of this stream
    bool alive = true;
    uint32_t k = 0;
    for (Piece p; alive && next_piece(sm, k, p);) {
        if (t < p.streams) {
            Row row = row_at<C::kRows>(a, p.r, p.kvh, p.rb, item_row);
            if (!row.there) row.sees = 0;
            const float limit = row.there ? most_sum : INFINITY - INFINITY;      // NaN: nothing is as large
            const int n = p.tiles(t);
            const int all_see = p.r.len - p.r.n + 1 + (p.rb * C::kRows + t * 128) / a.G;
            float m = -INFINITY, l = 0.0f;
            const auto await_sums = [&](int j) {      // of tile j, the last one that was counted in its lane
                const int b = p.lane(t, j);
                alive = warp_wait(&bars.pv_done[b], used[b] - 1, abort);
                tcgen05_fence_after_sync();
            };
            for (int j = 0; j < n && alive; ++j) {
                const int b = p.lane(t, j), p0 = (p.t0 + j) * kTile;
                alive = warp_wait(&bars.s_full[b], used[b], abort);
                if (!alive) break;
                tcgen05_fence_after_sync();
                const uint32_t s_addr = lanes + p.buffer(b) * 128, p_addr = lanes + C::kP + p.buffer(b) * C::kPStep;
                uint32_t there[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) there[c] = *const_cast<volatile const uint32_t*>(&sm.flags.there[(tile + j) % kFlags][c]);
                const bool masked = p0 + kTile > all_see || (there[0] & there[1] & there[2] & there[3]) != 0xffffffffu;
                uint32_t pk[4][16];
                // 32 scores at a time, the next on their way; mask: what the row does not see as -infinity (none: no row of the warp sees
                // any of them)
                const auto each = [&](auto mask, auto use) {
                    uint32_t sc[2][32];
                    tmem_ld_32x32(s_addr, sc[0]);
                    tmem_ld_wait_for(sc[0]);
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        if (c < 3) tmem_ld_32x32(s_addr + (c + 1) * 32, sc[(c + 1) & 1]);
                        bool none = false;
                        if (decltype(mask)::value) {
                            const int left = row.sees - p0 - c * 32;
                            const uint32_t in = left >= 32 ? there[c] : left <= 0 ? 0u : there[c] & ((1u << left) - 1u);
                            none = __all_sync(0xffffffffu, in == 0u);
                            if (!none && !__all_sync(0xffffffffu, in == 0xffffffffu)) {
#pragma unroll
                                for (int e = 0; e < 32; ++e)
                                    if (!(in >> e & 1u)) sc[c & 1][e] = 0xff800000u;
                            }
                        }
                        use(c, sc[c & 1], none);
                        if (c < 3) tmem_ld_wait_for(sc[(c + 1) & 1]);
                    }
                };
                const auto weights = [&](auto mask) {
                    const Pair times = twice(scale), minus = twice(fmaf(m == -INFINITY ? 0.0f : -m, scale, -a.lower));
                    Pair sum[2] = {0, 0};
                    each(mask, [&](int c, const uint32_t (&sc)[32], bool none) {
                        if (decltype(mask)::value && none) {
#pragma unroll
                            for (int e = 0; e < 16; ++e) pk[c][e] = 0u;
                            return;
                        }
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            const Pair x = fma2(pair_of(__uint_as_float(sc[2 * e]), __uint_as_float(sc[2 * e + 1])), times, minus);
                            float2 y = both(x);
                            y = make_float2(pow2(y.x), pow2(y.y));
                            sum[e & 1] = add2(sum[e & 1], pair_of(y.x, y.y));
                            pk[c][e] = pack_bf16(y.x, y.y);
                        }
                    });
                    const float2 s0 = both(sum[0]), s1 = both(sum[1]);
                    return (s0.x + s0.y) + (s1.x + s1.y);
                };
                // the first tile: relative to the score of its first key, which every row of it sees that sees anything
                if (j == 0) {
                    const float first_score = __uint_as_float(tmem_ld_word(s_addr));
                    if (row.sees > p0 && (there[0] & 1u) && fabsf(first_score) < INFINITY) m = first_score;
                }
                float more = masked ? weights(Const<1>()) : weights(Const<0>());
                // a new reference: from the scores again.  A row moves by what it sees alone, not by its neighbours, and not where its weights
                // are NaN, which no reference mends; what lies in rows of no sequence moves nothing.
                const bool anew = more >= limit || !(m > -INFINITY || row.sees <= p0);
                if (__any_sync(0xffffffffu, anew)) {
                    float mx = -INFINITY;
                    each(Const<1>(), [&](int, const uint32_t (&sc)[32], bool none) {
                        if (none) return;
                        float most[4];
#pragma unroll
                        for (int q = 0; q < 4; ++q) most[q] = max3(__uint_as_float(sc[q]), __uint_as_float(sc[q + 4]), __uint_as_float(sc[q + 8]));
#pragma unroll
                        for (int e = 12; e < 28; e += 8)
#pragma unroll
                            for (int q = 0; q < 4; ++q) most[q] = max3(most[q], __uint_as_float(sc[e + q]), __uint_as_float(sc[e + 4 + q]));
#pragma unroll
                        for (int q = 0; q < 4; ++q) most[q] = max2(most[q], __uint_as_float(sc[28 + q]));
                        mx = max3(max3(most[0], most[1], most[2]), most[3], mx);
                    });
                    const bool moves = anew && (mx - m) * scale > kSlack;      // not where it is NaN: all weights of the row are
                    if (__any_sync(0xffffffffu, moves)) {
                        const float to = moves ? fmaxf(m, mx) : m, f = !moves ? 1.0f : m == -INFINITY ? 0.0f : pow2((m - to) * scale);
                        if (j > 0) {
                            await_sums(j - 1);
                            if (!alive) break;
                            for (int c = 0; c < a.dh; c += 16) {
                                uint32_t o[16];
                                tmem_ld_32x16(o_addr + c, o);
                                tmem_ld_wait_for(o);
#pragma unroll
                                for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                                tmem_st_32x16(o_addr + c, o);
                            }
                        }
                        l *= f;
                        m = to;
                    }
                    more = weights(Const<1>());
                }
                l += more;
                if (C::kApart && j > (p.streams == 2 ? 0 : 1)) {      // the P before it in its place has been read
                    alive = warp_wait(&bars.pv_done[b], used[b] - 1, abort);
                    if (!alive) break;
                    tcgen05_fence_after_sync();
                }
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_st_32x16(p_addr + c * 16, pk[c]);
                tmem_st_wait();
                ++used[b];
                tcgen05_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(&bars.p_full[b]);
            }
            if (n > 0 && alive) await_sums(n - 1);
            if (CARE && alive)
                alive = add_odd<DP, EIGHT>(a, sm, p, k - 1, n, row.token, row.head, row.sees, (m == -INFINITY ? 0.0f : m * scale) + a.lower, o_addr);
            if (!alive) break;
            const bool some = l != 0.0f && row.kept;
            const long long at = static_cast<long long>(row.token) * a.H + row.head;
            const float f = some ? 1.0f / l : 0.0f;
            float* slot = p.slot(a) + 2ll * a.rows + static_cast<long long>(item_row) * 4;
            Pair zeros = 0;      // the sums times 0: NaN where one is infinite or NaN
            if (p.complete) {
                const long long mine = row.there ? at * a.dh : -1;
                long long rows[4];      // of the four lanes' rows of the output
#pragma unroll
                for (int q = 0; q < 4; ++q) rows[q] = __shfl_sync(0xffffffffu, mine, (lane & ~3) + q);
                for (int c = 0; c < a.dh; c += 32) {
                    uint32_t o[2][16] = {};
                    if (n > 0) {
                        tmem_ld_32x16(o_addr + c, o[0]);
                        if (c + 16 < a.dh) tmem_ld_32x16(o_addr + c + 16, o[1]);
                        tmem_ld_wait_for(o[0]);
                        tmem_ld_wait_for(o[1]);
                    }
                    uint4 y[4];
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        uint32_t v[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float x = __uint_as_float(o[q >> 1][(q & 1) * 8 + 2 * e]), z = __uint_as_float(o[q >> 1][(q & 1) * 8 + 2 * e + 1]);
                            zeros = fma2(pair_of(x, z), 0, zeros);
                            v[e] = some ? pack_bf16(x * f, z * f) : 0u;
                        }
                        y[q] = make_uint4(v[0], v[1], v[2], v[3]);
                    }
                    turn_words(y, lane);
                    const int col = c + (lane & 3) * 8;
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        if (rows[q] >= 0 && col < a.dh) *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(a.out) + rows[q] + col) = y[q];
                }
                if (row.there && a.lse) a.lse[at] = some ? fmaf(m, scale, log2f(l * a.raise)) * kLn2 : -INFINITY;
            } else {
                if (row.there) {
                    p.slot(a)[item_row] = m * scale;
                    p.slot(a)[a.rows + item_row] = l;
                }
                for (int c = 0; c < a.dh; c += 16) {
                    uint32_t o[16] = {};
                    if (n > 0) {
                        tmem_ld_32x16(o_addr + c, o);
                        tmem_ld_wait_for(o);
                    }
#pragma unroll
                    for (int e = 0; e < 16; e += 2) zeros = fma2(pair_of(__uint_as_float(o[e]), __uint_as_float(o[e + 1])), 0, zeros);
                    if (row.there) {
#pragma unroll
                        for (int q = 0; q < 4; ++q)
                            *reinterpret_cast<uint4*>(slot + (c / 4 + q) * 4ll * a.rows) = make_uint4(o[4 * q], o[4 * q + 1], o[4 * q + 2], o[4 * q + 3]);
                    }
                }
            }
            // a value that is infinite or NaN, and a tile that the row does not see all of
            const float2 z = both(zeros);
            if (!CARE && z.x + z.y != 0.0f && some && fabsf(l) < INFINITY && (p.t0 + n) * kTile > all_see) *const_cast<volatile int*>(&bars.again) = 1;
        }
        tile += p.n;
    }
}

template <int DP, bool EIGHT>
__device__ __forceinline__ void init_barriers(Bars& bars) {
    for (int i = 0; i < Cfg<DP, EIGHT>::kStages; ++i) {
        mbar_init(&bars.full[i], 4);      // the gathering warps
        mbar_init(&bars.empty[i], 1);
    }
    mbar_init(&bars.q_full, 4);
    mbar_init(&bars.q_empty, 1);
    for (int b = 0; b < kLanes; ++b) {
        mbar_init(&bars.s_full[b], 2);    // the products, and the thread that issues them
        mbar_init(&bars.p_full[b], 4);    // a stream's warps
        mbar_init(&bars.pv_done[b], 1);
    }
    for (int i = 0; i < 4; ++i) mbar_init(&bars.raw[i], 1);
    mbar_init(&bars.drained, 1);
    for (int i = 0; i < 2 * kPieces; ++i) mbar_init(&bars.looked[i], 4);
    for (int i = 0; i < kPieces; ++i) {
        mbar_init(&bars.piece_full[i], 1);
        mbar_init(&bars.piece_empty[i], kReaders);
    }
    bars.again = 0;
    mbar_fence_init();
}
// The thread block's part of the line, by all its threads; the first time they share registers out anew.
template <int DP, bool EIGHT, bool CARE>
__device__ __forceinline__ void take_part(const Args& a, const Maps& maps, Smem<DP, EIGHT>& sm) {
    using C = Cfg<DP, EIGHT>;
    const int warp = threadIdx.x >> 5;
    const Found<C::kRows, kTile, kOver> f = locate<C::kRows, kTile, kOver, kThreads>(a, sm.sh);      // threads meet in it
    tcgen05_fence_after_sync();
    if (f.walk.left <= 0) return;      // the same in every thread
    if (warp < 8) {
        if (!CARE) more_registers<kRowRegs>();
        softmax_rows<DP, EIGHT, CARE>(a, sm);
    } else if (warp < 12) {
        if (!CARE) fewer_registers<kCopyRegs>();
        Gather<DP, EIGHT, CARE>(a, maps, sm).run();
    } else {
        if (!CARE) fewer_registers<kIssueRegs>();
        if (warp == 12) Issue<DP, EIGHT>(a, sm).run();
        if (warp == 13) walk_line<DP, EIGHT>(a, sm, f.walk, f.total);
    }
    __syncwarp();
    tcgen05_fence_before_sync();
    __syncthreads();
    tcgen05_fence_after_sync();
}
// Behind a wait that ran out: every copy that the gathering warps have asked for lands before the thread block goes away.  Warps got to different
// stages; who lags arrives at the others' without copies, so that their phases end.  No warp lags a whole ring.
template <int DP, bool EIGHT>
__device__ __noinline__ void land(Smem<DP, EIGHT>& sm) {
    constexpr uint32_t S = Cfg<DP, EIGHT>::kStages;
    const int warp = static_cast<int>(threadIdx.x >> 5) - 8;
    if (warp >= 0 && warp < 4 && (threadIdx.x & 31) == 0) {
        uint32_t fills = 0, asked = 0;
        for (int w = 0; w < 4; ++w) {
            fills = max(fills, static_cast<uint32_t>(sm.sh[w]));
            asked = max(asked, static_cast<uint32_t>(sm.sh[4 + w]));
        }
        const uint32_t cleared = static_cast<uint32_t>(sm.sh[8 + warp]);
        int never = 0;
        for (uint32_t f = static_cast<uint32_t>(sm.sh[warp]); f < fills; ++f) mbar_arrive(&sm.bars.full[f % S]);
        for (uint32_t p = static_cast<uint32_t>(sm.sh[4 + warp]); p < asked; ++p) mbar_arrive(&sm.bars.q_full);
        if (cleared > 0) mbar_wait_bounded(&sm.bars.raw[warp], (cleared - 1) & 1u, &never);
        for (uint32_t f = fills > S ? fills - S : 0; f < fills; ++f) mbar_wait_bounded(&sm.bars.full[f % S], f / S & 1u, &never);
        if (asked > 0) mbar_wait_bounded(&sm.bars.q_full, (asked - 1) & 1u, &never);
    }
    __syncthreads();
}
// A second time, with the registers of the launch.  A function of its own, so that none of it is in the first time's way.
template <int DP, bool EIGHT>
__device__ __noinline__ void take_part_with_care(const Args& a, const Maps& maps, Smem<DP, EIGHT>& sm) {
    if (threadIdx.x == 0) {
        for (uint64_t* b = reinterpret_cast<uint64_t*>(&sm.bars); b < reinterpret_cast<uint64_t*>(&sm.bars.tmem); ++b) mbar_inval(b);
        init_barriers<DP, EIGHT>(sm.bars);
    }
    take_part<DP, EIGHT, true>(a, maps, sm);
}

template <int DP, bool EIGHT>
__global__ void __launch_bounds__(kThreads, 1) paged_prompt_mha_kernel(const __grid_constant__ Args a, const __grid_constant__ Maps maps) {
    extern __shared__ __align__(1024) unsigned char raw[];
    Smem<DP, EIGHT>& sm = *reinterpret_cast<Smem<DP, EIGHT>*>(raw);
    Bars& bars = sm.bars;
    const int tid = threadIdx.x, warp = tid >> 5;
    chain_wait();
    if (tid == 0) {
        init_barriers<DP, EIGHT>(bars);
        bars.abort = 0;
    }
    if (warp == 12) {
        tmem_alloc(&bars.tmem, 512);
        tmem_relinquish_alloc_permit();
    }
    tcgen05_fence_before_sync();
    take_part<DP, EIGHT, false>(a, maps, sm);
    if (bars.again && !bars.abort) {      // the same in every thread
        if (warp < 8) fewer_registers<128>();
        __syncthreads();
        if (warp >= 8) more_registers<128>();
        take_part_with_care<DP, EIGHT>(a, maps, sm);
    }
    if (bars.abort) land<DP, EIGHT>(sm);
    if (warp == 12) tmem_dealloc(bars.tmem, 512);
    if (tid == 0 && bars.abort) flag_status(a.status, HALO_DEV_TIMEOUT);
}

template <int DP>
int blocks_of(const halo_paged_shape& sh, int n_tok, int n_seq) {
    return line_blocks(sh, n_tok, n_seq, Cfg<DP>::kRows, kTile, kOver, kSmCount);
}
template <typename F>
auto by_width(const halo_paged_shape& sh, F f) {
    return sh.head_dim <= 64    ? f(std::integral_constant<int, 64>())
           : sh.head_dim <= 128 ? f(std::integral_constant<int, 128>())
                                : f(std::integral_constant<int, 256>());
}
size_t workspace(const halo_paged_shape& sh, int n_tok, int n_seq) {
    return by_width(sh, [&](auto dp) {
        constexpr int DP = decltype(dp)::value;
        return static_cast<size_t>(blocks_of<DP>(sh, n_tok, n_seq)) *
               (sizeof(Opening) + 2 * sizeof(float) * slot_floats(slot_rows(Cfg<DP>::kRows, n_tok, sh), sh.head_dim));
    });
}
halo_status launch(const Args& args, const halo_paged_shape& sh, void* ws, cudaStream_t st) {
    return by_width(sh, [&](auto dp) -> halo_status {
        constexpr int DP = decltype(dp)::value;
        Args a = args;
        a.blocks = blocks_of<DP>(sh, a.n_tok, a.n_seq);
        a.rows = slot_rows(Cfg<DP>::kRows, a.n_tok, sh);
        a.slot = slot_floats(a.rows, a.dh);
        a.openings = static_cast<Opening*>(ws);
        a.ws = reinterpret_cast<float*>(a.openings + a.blocks);
        const long long tiles = (static_cast<long long>(sh.max_pages) * sh.page_size + kTile - 1) / kTile;
        int lower = 21;
        while (1ll << (lower - 21) < tiles) ++lower;
        a.lower = static_cast<float>(lower);
        a.raise = ldexpf(1.0f, lower);
        Maps maps = {};
        const uint64_t wide = sh.head_dim, row = wide * 2;
        const int page_bits = sh.page_size & -sh.page_size;
        if (wide >= 64 && page_bits >= 8 && !a.K_scale) {
            maps.box_rows = page_bits < 32 ? page_bits : 32;
            const uint64_t dims[4] = {wide, static_cast<uint64_t>(sh.page_size), static_cast<uint64_t>(a.Hk), static_cast<uint64_t>(sh.n_pages)};
            const uint64_t strides[3] = {row, row * sh.page_size, static_cast<uint64_t>(a.page_stride) * 2};
            const uint32_t box[4] = {64, static_cast<uint32_t>(maps.box_rows), 1, 1};
            if (!make_bf16_map_nd(&maps.K, a.K, 4, dims, strides, box) || !make_bf16_map_nd(&maps.V, a.V, 4, dims, strides, box)) return HALO_ERR_CUDA;
        }
        if (wide >= 64 && 128 % a.G == 0 && a.n_tok >= 128 / a.G) {
            maps.whole_q = 1;
            const uint64_t dims[3] = {wide, static_cast<uint64_t>(a.H), static_cast<uint64_t>(a.n_tok)};
            const uint64_t strides[2] = {row, static_cast<uint64_t>(a.q_stride) * 2};
            const uint32_t box[3] = {64, static_cast<uint32_t>(a.G), static_cast<uint32_t>(128 / a.G)};
            if (!make_bf16_map_nd(&maps.q, a.q, 3, dims, strides, box)) return HALO_ERR_CUDA;
        }
        const auto run = [&](auto eight) -> halo_status {
            constexpr bool E = decltype(eight)::value;
            static_assert(sizeof(Smem<DP, E>) <= 227 * 1024, "shared memory of a thread block");
            static bool done[64];
            if (!ensure_dynamic_smem(paged_prompt_mha_kernel<DP, E>, sizeof(Smem<DP, E>), done)) return HALO_ERR_CUDA;
            return launch_chained(paged_prompt_mha_kernel<DP, E>, a.blocks, kThreads, sizeof(Smem<DP, E>), st, a, maps);
        };
        const halo_status rc = a.K_scale ? run(std::true_type()) : run(std::false_type());
        return rc != HALO_OK ? rc : launch_join<__nv_bfloat16, Cfg<DP>::kRows>(a, st);
    });
}

}  // namespace
}  // namespace prompt
}  // namespace halo

using namespace halo;

extern "C" size_t halo_paged_prompt_mha_workspace_bytes(const halo_paged_shape* shape, int n_tok, int n_seq) {
    if (check_paged_shape(shape) != HALO_OK || n_seq <= 0 || n_seq > HALO_MAX_SEQUENCES || n_tok <= 0 || n_tok > HALO_MAX_PROMPT_ROWS) return 0;
    return shape->dtype == HALO_F32 ? prompt::f32_workspace(*shape, n_tok, n_seq) : prompt::workspace(*shape, n_tok, n_seq);
}

extern "C" halo_status halo_paged_prompt_mha(const halo_paged_shape* shape, int n_tok, int n_seq, const void* q, long long q_stride,
                                             const int32_t* q_start, const void* K_cache, const void* V_cache, const uint8_t* K_scale,
                                             const uint8_t* V_scale, const int32_t* block_table, const int32_t* seq_len,
                                             const uint8_t* keep, float scale, void* out, float* lse, void* workspace,
                                             size_t workspace_bytes, uint32_t* dev_status, void* stream) {
    halo_status rc = check_paged_shape(shape);
    if (rc != HALO_OK) return rc;
    if (!q || !q_start || !K_cache || !V_cache || !block_table || !seq_len || !out || q == out) return HALO_ERR_ARG;
    if (!isfinite(scale)) return HALO_ERR_ARG;
    if (n_seq <= 0 || n_seq > HALO_MAX_SEQUENCES || n_tok <= 0 || n_tok > HALO_MAX_PROMPT_ROWS) return HALO_ERR_SHAPE;
    const int elem = shape->dtype == HALO_F32 ? 4 : 2;
    if (q_stride < static_cast<long long>(shape->n_heads) * shape->head_dim) return HALO_ERR_SHAPE;
    if (!aligned16(q) || !aligned16(K_cache) || !aligned16(V_cache) || !aligned16(out) || q_stride * elem % 16 != 0) return HALO_ERR_ALIGN;
    rc = check_eight(*shape, K_scale, V_scale);
    if (rc != HALO_OK) return rc;
    const size_t need = halo_paged_prompt_mha_workspace_bytes(shape, n_tok, n_seq);
    if (!workspace || workspace_bytes < need) return HALO_ERR_WORKSPACE;
    if (!aligned16(workspace)) return HALO_ERR_ALIGN;
    prompt::Args a = {};
    a.n_tok = n_tok;
    a.n_seq = n_seq;
    a.H = shape->n_heads;
    a.Hk = shape->n_kv_heads;
    a.G = a.H / a.Hk;
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
    if (a.scale_log2 == 0.0f) a.scale_log2 = 1.0e-45f;      // scores of zero, and -infinity for what is not seen
    a.q = q;
    a.K = K_cache;
    a.V = V_cache;
    a.K_scale = K_scale;
    a.V_scale = V_scale;
    a.q_start = q_start;
    a.table = block_table;
    a.seq_len = seq_len;
    a.keep = keep;
    a.out = out;
    a.lse = lse;
    a.status = dev_status;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    return shape->dtype == HALO_F32 ? prompt::f32_launch(a, *shape, workspace, st) : prompt::launch(a, *shape, workspace, st);
}
