// halo_product_mx4: y[t][r] = <x_t, w_r> of rows in microscaled 4-bit floating point, on the block-scaled tensor
// cores (tcgen05.mma kind::mxf4, products of 64 elements with a power of two per 32, fp32 accumulators in TMEM).
//
// The weight rows are the rows of A and the tokens the columns of B, so one token costs a tile of 16 columns and not
// one of 128 rows, and a lane of the epilogue is a weight row: 32 lanes store 32 neighbouring outputs.
// Stages of 256 elements: 128-byte rows of codes by tensor-map TMA (128-byte swizzle), the scales as 512-byte blocks
// by bulk copies, moved on to TMEM by tcgen05.cp in front of the products that use them.  Every stage of the ring has
// its own columns of scales: a stage is refilled only when the products that read its old scales have completed.
//
// Three kernels:
//   mx4_one_kernel   one token and some thousand rows: exact fp16 products on the ordinary pipe, described at the kernel.
//   mx4_line_kernel  up to 32 tokens, bound by HBM (0.53 bytes per weight element): the weight rows in groups of 32 form
//     a line that is cut into equal pieces, one thread block per SM; whole outputs per thread block, so nothing has to
//     be added up between thread blocks.  32000 x 4096: 16.1 us for up to 16 tokens, 4.3 TB/s of weights.
//   mx4_pair_kernel  more tokens, or fewer through many long rows: pairs of SMs (cta_group::2) on tiles of 256 rows x 256
//     tokens; each SM fetches half of either operand, 35 KB per 16.8 M products and SM where a single SM's 128 x 256
//     tile takes 51 KB.  Prompts are bound by the L2-to-SM traffic and the tensor pipe: 4096 x 11008 x 4096 70 us = 5.3
//     PFLOP/s, tensor pipe 68 % active; a stage takes 0.37 us and a tile 0.85 us beyond its stages (one accumulator: a
//     second one would leave no tensor memory for the scales at this tile, and smaller tiles fetch more per product).
//     A last round that fits twice is halved into 128 tokens a tile, as are tiles with no more tokens left: 300 x 4096 x
//     4096 9.5 -> 7.5 us, 512 x 11008 x 4096 15.9 -> 14.4.
//
// Every wait is bounded; when one runs out the block's roles leave their loops, the copies in flight are waited for,
// TMEM is freed and HALO_DEV_TIMEOUT is raised.
#include <cuda_fp16.h>

#include "common.cuh"
#include "umma.cuh"

namespace halo {

bool make_byte_map(CUtensorMap* map, const void* base, uint64_t rows, uint64_t row_bytes, uint32_t box_bytes, uint32_t box_rows);
bool make_scale_map(CUtensorMap* map, const void* base, uint64_t tiles, uint64_t blocks, uint32_t box_tiles, uint32_t box_blocks);

namespace {

constexpr int kThreads = 192;      // loader warp, MMA warp, four epilogue warps
constexpr int kRowsTile = 128;
constexpr int kStageK = 256;       // elements of a stage

__device__ __forceinline__ void umma_mxf4(uint32_t tmem_d, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t tmem_sfa,
                                          uint32_t tmem_sfb, bool accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(tmem_d),
        "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(tmem_sfa), "r"(tmem_sfb), "r"(static_cast<uint32_t>(accumulate))
        : "memory");
}
// Instruction descriptor of kind::mxf4: e2m1 x e2m1 -> fp32, scales powers of two; sf = 0 or 2 picks the bytes of the
// scale words that belong to these 64 elements.
__device__ __forceinline__ constexpr uint32_t idesc_mxf4(int m, int n, uint32_t sf) {
    return (sf << 4)                                // scale bytes of B
           | (1u << 7)                              // A: e2m1
           | (1u << 10)                             // B: e2m1
           | (static_cast<uint32_t>(n >> 3) << 17)  // N / 8
           | (1u << 23)                             // scales: powers of two
           | (static_cast<uint32_t>(m >> 7) << 27)
           | (sf << 29);                            // scale bytes of A
}
// 512 bytes of shared memory (32 rows of 16 bytes, no swizzle, 128 bytes per 8 rows) -> 4 columns, repeated in the four
// quarters of the lanes
__device__ __forceinline__ uint64_t scales_desc(uint32_t smem) {
    return static_cast<uint64_t>((smem & 0x3FFFFu) >> 4) | (static_cast<uint64_t>(128u >> 4) << 32) | (1ull << 46);
}
__device__ __forceinline__ void tmem_cp_scales(uint32_t taddr, uint64_t desc) {
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}

// ---- one token -----------------------------------------------------------------------------------------------------
// A run of 32 elements shares a scale on either side, so it is a sum of 32 products of plain 4-bit values, which fp16
// holds exactly: a product is a whole number of quarters of at most 36, and 8 of them (what one half of one accumulator
// takes here) stay below 2^11 quarters.  So a byte of codes is one conversion to two fp16 values and one packed
// multiply-add; the run's sum meets both scales in fp32.  The token sits in shared memory as fp16; a warp takes kRows
// rows at once, a lane the runs lane, lane + 32, ... of them, with kAhead 16-byte loads per row in flight.  A thread
// block's rows are neighbours: they share the lines of the scale blocks.  11008 x 4096: 7.3 us = 3.3 TB/s of weights, bound
// by issue and by the latency of a warp's few rounds (32000 x 4096: 16.7 us = 4.2 TB/s; 17.1 with integer products of
// bytes, dp4a and the byte permute as a table, which the wide multiplier bounds; loads of the next rows issued ahead of
// the products 19.5, half as many loads in flight 20).
constexpr int kOneThreads = 256;
constexpr size_t kOneSmem = 140 * 1024;   // the widest row
__device__ __forceinline__ float power(uint32_t byte) {   // 2^(byte - 127); 255 is NaN
    return __uint_as_float(byte == 0 ? 0x00400000u : byte == 255u ? 0x7fc00000u : byte << 23);
}
__device__ __forceinline__ void unpack(uint32_t w, __half2 (&h)[4]) {   // eight codes, exactly
    uint32_t r[4];
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\tmov.b32 {b0, b1, b2, b3}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, b0;\n\tcvt.rn.f16x2.e2m1x2 %1, b1;\n\tcvt.rn.f16x2.e2m1x2 %2, b2;\n\tcvt.rn.f16x2.e2m1x2 %3, b3;\n\t}"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(w));
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = *reinterpret_cast<const __half2*>(&r[i]);
}
template <typename T>
__global__ void __launch_bounds__(kOneThreads, 3)
mx4_one_kernel(int d, int n_rows, const uint8_t* __restrict__ Qx, const uint8_t* __restrict__ Sx,
               const uint8_t* __restrict__ Qw, const uint8_t* __restrict__ Sw, T* __restrict__ y) {
    constexpr int kRows = 2, kAhead = 4, kWarps = kOneThreads / 32;
    extern __shared__ __align__(16) unsigned char smem[];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int runs = d / 32;                       // of a row
    uint4* xs = reinterpret_cast<uint4*>(smem);    // [quarter of a run][run] 8 values, then [run] the token's scale
    float* sx = reinterpret_cast<float*>(xs + 4 * runs);
    chain_wait();
    bool large = false;
    for (int b = tid; b < runs; b += kOneThreads) {
        const uint4 code = ldg_stream16(Qx + b * 16);
        const uint32_t word[4] = {code.x, code.y, code.z, code.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            alignas(16) __half2 h[4];
            unpack(word[k], h);
            xs[k * runs + b] = *reinterpret_cast<uint4*>(h);
        }
        const uint32_t byte = ldg_waited(Sx + (b >> 2) * 512 + (b & 3));
        large |= byte > 240u;
        sx[b] = power(byte);
    }
    // A run's sum times a scale near 2^127 would leave the range before a small scale of w brings it back: a token with
    // such a scale is summed 2^-16 times its size (exact: scales are 2^-143 at least).
    const bool reduced = __syncthreads_or(large);
    if (reduced) {
        for (int b = tid; b < runs; b += kOneThreads) sx[b] *= 0x1p-16f;
        __syncthreads();
    }
    const float back = reduced ? 0x1p16f : 1.0f;
    const int first = static_cast<int>(static_cast<long long>(n_rows) * blockIdx.x / gridDim.x);
    const int end = static_cast<int>(static_cast<long long>(n_rows) * (blockIdx.x + 1) / gridDim.x);
    for (int r0 = first + warp * kRows; r0 < end; r0 += kWarps * kRows) {
        const uint8_t* q[kRows];
        const uint8_t* sc[kRows];
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            const int row = min(r0 + r, end - 1);
            q[r] = Qw + static_cast<size_t>(row) * (d / 2);
            sc[r] = Sw + static_cast<size_t>(row >> 7) * (d >> 7) * 512 + (row & 31) * 16 + ((row >> 5) & 3) * 4;
        }
        float sum[kRows] = {};
        for (int b0 = 0; b0 < runs; b0 += 32 * kAhead) {
            uint4 code[kAhead][kRows];
            uint32_t scale[kAhead][kRows];
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
#pragma unroll
                for (int r = 0; r < kRows; ++r) {
                    const int b = b0 + i * 32 + lane;
                    code[i][r] = b < runs ? ldg_stream16(q[r] + b * 16) : make_uint4(0, 0, 0, 0);
                    scale[i][r] = b < runs ? ldg_waited(sc[r] + (b >> 2) * 512 + (b & 3)) : 0u;
                }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int b = b0 + i * 32 + lane;
                if (b >= runs) break;
                __half2 acc[kRows][2];
#pragma unroll
                for (int r = 0; r < kRows; ++r) acc[r][0] = acc[r][1] = __float2half2_rn(0.0f);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const uint4 xv = xs[k * runs + b];
                    const __half2* xh = reinterpret_cast<const __half2*>(&xv);
#pragma unroll
                    for (int r = 0; r < kRows; ++r) {
                        const uint32_t w = k == 0 ? code[i][r].x : k == 1 ? code[i][r].y : k == 2 ? code[i][r].z : code[i][r].w;
                        __half2 h[4];
                        unpack(w, h);
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[r][k >> 1] = __hfma2(h[e], xh[e], acc[r][k >> 1]);
                    }
                }
#pragma unroll
                for (int r = 0; r < kRows; ++r) {
                    const float2 f0 = __half22float2(acc[r][0]), f1 = __half22float2(acc[r][1]);
                    // the plain sum x scale of x first: exact, and 0 stays 0 before a scale of 2^127
                    sum[r] = fmaf(((f0.x + f0.y) + (f1.x + f1.y)) * sx[b], power(scale[i][r]), sum[r]);
                }
            }
        }
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            const float v = warp_sum(sum[r]);
            if (lane == 0 && r0 + r < end) y[r0 + r] = from_float<T>(v * back);
        }
    }
}

// NT tokens (at most 128: one block of scales)
template <int NT, int STAGES>
struct Ring {
    static constexpr int kA = kRowsTile * (kStageK / 2);
    static constexpr int kB = NT * (kStageK / 2);
    static constexpr int kSf = 1024;
    static constexpr int kStage = kA + kB + 2 * kSf;
    static constexpr int kSfCols = 16;
    static constexpr int kAcc = 2;   // accumulators: one is read while the next fills
    static constexpr int kCols = kAcc * NT + STAGES * kSfCols;
    static constexpr int kTmem = kCols <= 256 ? 256 : 512;
    static constexpr size_t kSmem = static_cast<size_t>(STAGES) * kStage + 512;
    static_assert(kCols <= 512, "tensor memory");
    static_assert(kStage % 1024 == 0, "swizzled tiles start on 1024 bytes");
    static_assert(STAGES <= 12, "barriers");
};

struct LineBars {
    uint64_t full[12], empty[12], acc_full[2], acc_empty[2];
    uint32_t tmem;
    int abort_flag;
};

// The whole warp waits: the loops of the loader and MMA warps run in all lanes, so that addresses and descriptors stay
// in uniform registers, and one elected lane issues.  (With one lane in the loops a stage of six scale copies and four
// products took 510 ns to issue, more than the products themselves.)
__device__ __forceinline__ bool wait_or_abort(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
    const bool ok = mbar_wait_bounded(bar, parity, abort_flag);
    if (!ok) *abort_flag = 1;
    return __all_sync(0xffffffffu, ok);
}
__device__ __forceinline__ bool elect_one() {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0;
}
__device__ __forceinline__ int warp_index() { return __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x >> 5), 0); }
// stage of a ring and the parity of its current phase
template <int STAGES>
struct Slot {
    uint32_t stage = 0, parity = 0;
    __device__ __forceinline__ void advance() {
        if (++stage == STAGES) { stage = 0; parity ^= 1u; }
    }
};

// The line: the row groups of 32 in order.  A piece is a run of groups inside one block of 128 rows, so the rows of a
// group stand where the block's scales expect them.
struct Piece {
    int block, g0, g1;   // groups of the block, 0..4
};
struct Line {
    int at, end;
    __device__ __forceinline__ bool next(Piece& p) {
        if (at >= end) return false;
        p.block = at >> 2;
        p.g0 = at & 3;
        p.g1 = min(4, end - p.block * 4);
        at += p.g1 - p.g0;
        return true;
    }
};

template <typename T, int NT, int STAGES>
__global__ void __launch_bounds__(kThreads, 1)
mx4_line_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_g,
                const __grid_constant__ CUtensorMap map_x, int d, int n_tok,
                int n_rows, const uint8_t* __restrict__ Sw, const uint8_t* __restrict__ Sx, T* __restrict__ y,
                uint32_t* status) {
    using R = Ring<NT, STAGES>;
    extern __shared__ __align__(1024) unsigned char smem[];
    LineBars& bars = *reinterpret_cast<LineBars*>(smem + static_cast<size_t>(STAGES) * R::kStage);
    const int tid = threadIdx.x, warp = warp_index(), lane = tid & 31;
    const int atoms = d / 128;                       // 512-byte blocks of scales along a row
    const int nk = (d + kStageK - 1) / kStageK;
    Line line;
    const long long groups = (n_rows + 31) / 32;
    line.at = static_cast<int>(groups * blockIdx.x / gridDim.x);
    line.end = static_cast<int>(groups * (blockIdx.x + 1) / gridDim.x);

    if (tid == 0) {
        for (int s = 0; s < STAGES; ++s) { mbar_init(&bars.full[s], 1); mbar_init(&bars.empty[s], 1); }
        for (int b = 0; b < R::kAcc; ++b) { mbar_init(&bars.acc_full[b], 1); mbar_init(&bars.acc_empty[b], 4); }
        bars.abort_flag = 0;
        mbar_fence_init();
        tma_prefetch_descriptor(&map_w);
        tma_prefetch_descriptor(&map_x);
    }
    if (warp == 1) { tmem_alloc(&bars.tmem, R::kTmem); tmem_relinquish_alloc_permit(); }
    tcgen05_fence_before_sync();
    __syncthreads();
    tcgen05_fence_after_sync();
    chain_wait();
    volatile int* abort_flag = &bars.abort_flag;
    const uint32_t tmem = bars.tmem;
    Piece p;

    if (warp == 0) {
        const bool leader = elect_one();
        Slot<STAGES> slot;
        int it = 0;
        bool alive = true;
        while (alive && line.next(p)) {
            const uint8_t* sw = Sw + static_cast<size_t>(p.block) * atoms * 512;
            for (int k = 0; k < nk; ++k, ++it, slot.advance()) {
                uint64_t* full = &bars.full[slot.stage];
                if (it >= STAGES && !wait_or_abort(&bars.empty[slot.stage], slot.parity ^ 1u, abort_flag)) { alive = false; break; }
                unsigned char* st = smem + slot.stage * R::kStage;
                unsigned char* sc = st + R::kA + R::kB;
                const uint32_t bytes = min(2, atoms - k * 2) * 512u;
                if (leader) {
                    mbar_arrive_expect_tx(full, (p.g1 - p.g0) * 32 * (kStageK / 2) + R::kB + 2 * bytes);
                    if (p.g1 - p.g0 == 4)
                        tma_load_2d(st, &map_w, k * (kStageK / 2), p.block * kRowsTile, full);
                    else
                        for (int g = p.g0; g < p.g1; ++g)
                            tma_load_2d(st + g * 32 * (kStageK / 2), &map_g, k * (kStageK / 2), p.block * kRowsTile + g * 32, full);
                    tma_load_2d(st + R::kA, &map_x, k * (kStageK / 2), 0, full);
                    bulk_copy_g2s(sc, sw + k * 1024, bytes, full);
                    bulk_copy_g2s(sc + R::kSf, Sx + k * 1024, bytes, full);
                }
                __syncwarp();
            }
        }
        if (*abort_flag && leader) {
            int never = 0;
            for (int i = max(0, it - STAGES); i < it; ++i) mbar_wait_bounded(&bars.full[i % STAGES], (i / STAGES) & 1, &never);
        }
    } else if (warp == 1) {
        const bool leader = elect_one();
        Slot<STAGES> slot;
        int n = 0;
        bool alive = true;
        while (alive && line.next(p)) {
            const int acc = n % R::kAcc;
            if (n >= R::kAcc && !wait_or_abort(&bars.acc_empty[acc], ((n / R::kAcc) - 1) & 1, abort_flag)) break;
            tcgen05_fence_after_sync();
            const uint32_t tmem_d = tmem + acc * NT;
            for (int k = 0; k < nk; ++k, slot.advance()) {
                if (!wait_or_abort(&bars.full[slot.stage], slot.parity, abort_flag)) { alive = false; break; }
                tcgen05_fence_after_sync();
                const uint32_t st = smem_u32(smem) + slot.stage * R::kStage, sc = st + R::kA + R::kB;
                const uint32_t sfa = tmem + R::kAcc * NT + slot.stage * R::kSfCols, sfb = sfa + 8;
                const uint64_t da = umma_smem_desc(st, 0, 1024), db = umma_smem_desc(st + R::kA, 0, 1024);
                const uint64_t dsa = scales_desc(sc), dsb = scales_desc(sc + R::kSf);
                if (leader) {
#pragma unroll
                    for (int at = 0; at < 2; ++at) {
                        if (at == 1 && atoms - k * 2 < 2) break;   // an odd number of runs of 128: half a stage
                        tmem_cp_scales(sfa + at * 4, dsa + at * 32);
                        tmem_cp_scales(sfb + at * 4, dsb + at * 32);
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        if (j == 2 && atoms - k * 2 < 2) break;
                        umma_mxf4(tmem_d, da + j * 2, db + j * 2, idesc_mxf4(kRowsTile, NT, (j & 1) * 2), sfa + (j >> 1) * 4,
                                  sfb + (j >> 1) * 4, j > 0 || k > 0);
                    }
                    umma_commit(&bars.empty[slot.stage]);
                }
                __syncwarp();
            }
            if (leader) umma_commit(&bars.acc_full[acc]);
            __syncwarp();
            ++n;
        }
    } else {
        int n = 0;
        const int quad = warp & 3;
        while (line.next(p)) {
            const int acc = n % R::kAcc;
            if (!wait_or_abort(&bars.acc_full[acc], (n / R::kAcc) & 1, abort_flag)) break;
            tcgen05_fence_after_sync();
            const int row = p.block * kRowsTile + quad * 32 + lane;
            const bool mine = quad >= p.g0 && quad < p.g1 && row < n_rows;
            const uint32_t base = tmem + acc * NT + (static_cast<uint32_t>(quad * 32) << 16);
            T* out = y + row;
            for (int c0 = 0; c0 < n_tok; c0 += 16) {
                uint32_t v[16];
                tmem_ld_32x16(base + c0, v);
                tmem_ld_wait();
                if (c0 + 16 >= n_tok) {   // the accumulator has been read
                    tcgen05_fence_before_sync();
                    if (lane == 0) mbar_arrive(&bars.acc_empty[acc]);
                }
#pragma unroll
                for (int c = 0; c < 16; ++c)
                    if (mine && c0 + c < n_tok) out[static_cast<long long>(c0 + c) * n_rows] = from_float<T>(__uint_as_float(v[c]));
            }
            ++n;
        }
    }
    __syncwarp();
    tcgen05_fence_before_sync();
    __syncthreads();
    if (warp == 1) { tcgen05_fence_after_sync(); tmem_dealloc(tmem, R::kTmem); }
    if (tid == 0 && *abort_flag) flag_status(status, HALO_DEV_TIMEOUT);
}

// ---- pairs of SMs -----------------------------------------------------------------------------------------------
constexpr int kPairThreads = 320;      // loader warp, MMA warp, eight epilogue warps
constexpr int kPairStages = 6;
constexpr int kPairTile = 256;         // rows and tokens of a pair's tile; an SM fetches 128 of either
struct PairRing {
    static constexpr int kOp = 128 * (kStageK / 2);
    static constexpr int kSfa = 1024, kSfb = 2048;     // the scales of all 256 tokens go to both SMs
    static constexpr int kStage = 2 * kOp + kSfa + kSfb;
    static constexpr int kSfCols = 24;
    static constexpr size_t kSmem = static_cast<size_t>(kPairStages) * kStage + 512;
};
static_assert(PairRing::kStage % 1024 == 0 && kPairTile + kPairStages * PairRing::kSfCols <= 512, "layout");

struct PairBars {
    uint64_t full[kPairStages];        // first SM only: the copies of both have landed
    uint64_t empty[kPairStages];       // the products that read the stage have completed
    uint64_t acc_full, acc_empty;      // acc_empty: first SM only, all sixteen epilogue warps have read
    uint32_t tmem;
    int abort_flag;
};

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync_all() {
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}
__device__ __forceinline__ uint32_t in_block_of(uint32_t rank, const void* p) {
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(rank));
    return a;
}
// Relaxed: what it announces are finished reads of tensor memory (tcgen05.wait::ld and the fence in front of it); a
// release would wait for the outstanding stores of the tile before as well (4096 x 11008 x 4096: 74 instead of 69 us).
__device__ __forceinline__ void arrive_at(uint32_t cluster_addr) {
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
// a phase that threads or products of the other SM complete; the whole warp waits
__device__ __forceinline__ bool wait_cluster(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
    const long long t0 = clock64();
    uint32_t spins = 0;
    while (true) {
        uint32_t ok;
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(ok)
            : "r"(smem_u32(bar)), "r"(parity)
            : "memory");
        if (__all_sync(0xffffffffu, ok != 0)) return true;
        if ((++spins & 255u) == 0u && __any_sync(0xffffffffu, *abort_flag || clock64() - t0 > kWaitLimitCycles)) {
            *abort_flag = 1;
            return false;
        }
    }
}
// Tensor-map copies into this SM's shared memory that count at a barrier of either SM of the pair (an address in the
// cluster's shared memory).
__device__ __forceinline__ void tma_pair_2d(void* dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(
            smem_u32(dst)),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(bar)
        : "memory");
}
__device__ __forceinline__ void tma_pair_3d(void* dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(
            smem_u32(dst)),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(bar)
        : "memory");
}
__device__ __forceinline__ void umma_mxf4_pair(uint32_t tmem_d, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t tmem_sfa,
                                               uint32_t tmem_sfb, bool accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(tmem_d),
        "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(tmem_sfa), "r"(tmem_sfb), "r"(static_cast<uint32_t>(accumulate))
        : "memory");
}
__device__ __forceinline__ void tmem_cp_scales_pair(uint32_t taddr, uint64_t desc) {
    asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}
// arrives at the same barrier of both SMs once the products issued so far have completed
__device__ __forceinline__ void umma_commit_pair(uint64_t* bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(
                     smem_u32(bar)),
                 "h"(static_cast<uint16_t>(3))
                 : "memory");
}

// The tiles of a product, 256 rows each, in the order of the pairs: whole rounds of 256 tokens, then the tiles of the
// last round, in halves of 128 tokens where these fit one round.  A tile that has at most 128 tokens left takes 128.
struct PairTiles {
    int row_tiles, whole, items;   // whole: tiles that are not halved; items: those and the halves
    int halves;                    // 0 or 1
};
struct PairTile {
    int row, tok, n;               // first row, first token, tokens (128 or 256; 0: nothing is left)
};
__device__ __forceinline__ PairTile tile_at(const PairTiles& t, int u, int n_tok) {
    const int half = u < t.whole ? 0 : (u - t.whole) & t.halves;
    const int tile = u < t.whole ? u : t.whole + ((u - t.whole) >> t.halves);
    PairTile p;
    p.row = tile % t.row_tiles * kPairTile;
    p.tok = tile / t.row_tiles * kPairTile + half * 128;
    p.n = p.tok >= n_tok ? 0 : n_tok - p.tok <= 128 || (u >= t.whole && t.halves) ? 128 : kPairTile;
    return p;
}

template <typename T>
__global__ void __launch_bounds__(kPairThreads, 1)
mx4_pair_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x,
                const __grid_constant__ CUtensorMap map_x64, const __grid_constant__ CUtensorMap map_sw, const __grid_constant__ CUtensorMap map_sx, PairTiles list,
                int d, int n_tok, int n_rows, T* __restrict__ y, uint32_t* status) {
    using R = PairRing;
    extern __shared__ __align__(1024) unsigned char smem[];
    PairBars& bars = *reinterpret_cast<PairBars*>(smem + static_cast<size_t>(kPairStages) * R::kStage);
    const int tid = threadIdx.x, warp = warp_index(), lane = tid & 31;
    const uint32_t rank = cluster_rank();
    const int atoms = d / 128, nk = (d + kStageK - 1) / kStageK;
    const int pairs = gridDim.x / 2, pair = blockIdx.x / 2;

    if (tid == 0) {
        for (int s = 0; s < kPairStages; ++s) {
            mbar_init(&bars.full[s], 1);
            mbar_init(&bars.empty[s], 1);
        }
        mbar_init(&bars.acc_full, 1);
        mbar_init(&bars.acc_empty, 16);
        bars.abort_flag = 0;
        mbar_fence_init();
        tma_prefetch_descriptor(&map_w);
        tma_prefetch_descriptor(&map_x);
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&bars.tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    __syncwarp();
    tcgen05_fence_before_sync();
    __syncthreads();
    cluster_sync_all();
    tcgen05_fence_after_sync();
    chain_wait();
    volatile int* abort_flag = &bars.abort_flag;
    const uint32_t tmem = bars.tmem;

    if (warp == 0) {
        const bool leader = elect_one();
        const uint32_t full0 = in_block_of(0, &bars.full[0]);
        Slot<kPairStages> slot;
        int it = 0;
        bool alive = true;
        for (int u = pair; u < list.items && alive; u += pairs) {
            const PairTile tile = tile_at(list, u, n_tok);
            if (tile.n == 0) continue;
            const int rb = tile.row / 128 + static_cast<int>(rank);            // this SM's block of 128 rows
            const int tb0 = tile.tok / 128;                                    // the pair's blocks of 128 tokens
            const bool wide = tile.n == kPairTile;
            for (int k = 0; k < nk; ++k, ++it, slot.advance()) {
                if (it >= kPairStages && !wait_or_abort(&bars.empty[slot.stage], slot.parity ^ 1u, abort_flag)) { alive = false; break; }
                unsigned char* st = smem + slot.stage * R::kStage;
                unsigned char* sc = st + 2 * R::kOp;
                const uint32_t full = full0 + slot.stage * 8;
                if (leader) {
                    // what lies outside a matrix arrives as zeros and counts: both SMs' bytes, the same for every stage
                    if (rank == 0) mbar_arrive_expect_tx(&bars.full[slot.stage], 2 * (wide ? R::kStage : R::kStage - R::kOp / 2));
                    tma_pair_2d(st, &map_w, k * (kStageK / 2), rb * 128, full);
                    if (wide)
                        tma_pair_2d(st + R::kOp, &map_x, k * (kStageK / 2), tile.tok + static_cast<int>(rank) * 128, full);
                    else
                        tma_pair_2d(st + R::kOp, &map_x64, k * (kStageK / 2), tile.tok + static_cast<int>(rank) * 64, full);
                    tma_pair_3d(sc, &map_sw, 0, k * 2, rb, full);
                    tma_pair_3d(sc + R::kSfa, &map_sx, 0, k * 2, tb0, full);
                }
                __syncwarp();
            }
        }
        if (*abort_flag && leader && rank == 0) {   // the copies of both SMs; neither leaves before the other
            int never = 0;
            for (int i = max(0, it - kPairStages); i < it; ++i)
                mbar_wait_bounded(&bars.full[i % kPairStages], (i / kPairStages) & 1, &never);
        }
    } else if (warp == 1) {
        const bool leader = elect_one();
        Slot<kPairStages> slot;
        int n = 0;
        bool alive = true;
        for (int u = pair; u < list.items && alive && rank == 0; u += pairs) {
            const PairTile tile = tile_at(list, u, n_tok);
            if (tile.n == 0) continue;
            if (n > 0 && !wait_cluster(&bars.acc_empty, (n - 1) & 1, abort_flag)) break;
            tcgen05_fence_after_sync();
            for (int k = 0; k < nk; ++k, slot.advance()) {
                if (!wait_cluster(&bars.full[slot.stage], slot.parity, abort_flag)) { alive = false; break; }
                tcgen05_fence_after_sync();
                const uint32_t st = smem_u32(smem) + slot.stage * R::kStage, sc = st + 2 * R::kOp;
                const uint32_t sfa = tmem + kPairTile + slot.stage * R::kSfCols, sfb = sfa + 8;
                const uint64_t da = umma_smem_desc(st, 0, 1024), db = umma_smem_desc(st + R::kOp, 0, 1024);
                const uint64_t dsa = scales_desc(sc), dsb = scales_desc(sc + R::kSfa);
                if (leader) {
#pragma unroll
                    for (int at = 0; at < 2; ++at) {
                        if (at == 1 && atoms - k * 2 < 2) break;
                        tmem_cp_scales_pair(sfa + at * 4, dsa + at * 32);
                        tmem_cp_scales_pair(sfb + at * 8, dsb + at * 32);
                        tmem_cp_scales_pair(sfb + at * 8 + 4, dsb + 64 + at * 32);
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        if (j == 2 && atoms - k * 2 < 2) break;
                        umma_mxf4_pair(tmem, da + j * 2, db + j * 2, idesc_mxf4(kPairTile, tile.n, (j & 1) * 2), sfa + (j >> 1) * 4,
                                       sfb + (j >> 1) * 8, j > 0 || k > 0);
                    }
                    umma_commit_pair(&bars.empty[slot.stage]);
                }
                __syncwarp();
            }
            if (leader) umma_commit_pair(&bars.acc_full);
            __syncwarp();
            ++n;
        }
    } else {
        // a warp reads 32 rows x 128 tokens into registers and lets the accumulator go before it stores
        const int quad = warp & 3, half = (warp - 2) >> 2;
        const uint32_t base = tmem + half * 128 + (static_cast<uint32_t>(quad * 32) << 16);
        const uint32_t acc_empty = in_block_of(0, &bars.acc_empty);
        int n = 0;
        for (int u = pair; u < list.items; u += pairs) {
            const PairTile tile = tile_at(list, u, n_tok);
            if (tile.n == 0) continue;
            if (!wait_cluster(&bars.acc_full, n++ & 1, abort_flag)) break;
            tcgen05_fence_after_sync();
            if (half * 128 >= tile.n) {
                if (lane == 0) arrive_at(acc_empty);
                continue;
            }
            uint32_t v[4][32];
#pragma unroll
            for (int c = 0; c < 4; ++c) tmem_ld_32x32(base + c * 32, v[c]);
            tmem_ld_wait();
            tcgen05_fence_before_sync();
            if (lane == 0) arrive_at(acc_empty);
            const int row = tile.row + static_cast<int>(rank) * 128 + quad * 32 + lane;
            const int tok0 = tile.tok + half * 128;
            if constexpr (sizeof(T) == 2) {
                if ((n_rows & 1) == 0) {
                    // two rows per word: lanes 2i and 2i + 1 exchange one token each of a pair of tokens
                    T* p = y + static_cast<long long>(tok0 + (lane & 1)) * n_rows + (row & ~1);
#pragma unroll
                    for (int i = 0; i < 64; ++i) {
                        const float a0 = __uint_as_float(v[i >> 4][(i & 15) * 2]), a1 = __uint_as_float(v[i >> 4][(i & 15) * 2 + 1]);
                        const float other = __shfl_xor_sync(0xffffffffu, lane & 1 ? a0 : a1, 1);
                        const __nv_bfloat162 two = lane & 1 ? __floats2bfloat162_rn(other, a1) : __floats2bfloat162_rn(a0, other);
                        if (row < n_rows && tok0 + 2 * i + (lane & 1) < n_tok) *reinterpret_cast<__nv_bfloat162*>(p) = two;
                        p += 2ll * n_rows;
                    }
                    continue;
                }
            }
            if (row < n_rows) {
                T* p = y + static_cast<long long>(tok0) * n_rows + row;
#pragma unroll
                for (int i = 0; i < 128; ++i) {
                    if (tok0 + i < n_tok) *p = from_float<T>(__uint_as_float(v[i >> 5][i & 31]));
                    p += n_rows;
                }
            }
        }
    }
    __syncwarp();
    tcgen05_fence_before_sync();
    __syncthreads();
    cluster_sync_all();   // neither SM leaves while the other may still read its memory or signal its barriers
    if (warp == 1) {
        tcgen05_fence_after_sync();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
    }
    if (tid == 0 && *abort_flag) flag_status(status, HALO_DEV_TIMEOUT);
}

struct Operands {
    int d, n_tok, n_rows;
    const void *Qx, *Sx, *Qw, *Sw;
    uint32_t* status;
    cudaStream_t st;
};

template <typename T>
halo_status launch_one(const Operands& o, T* y) {
    static bool done[64];
    if (!ensure_dynamic_smem(mx4_one_kernel<T>, kOneSmem, done)) return HALO_ERR_CUDA;
    static_assert(2 * HALO_MX4_MAX_WIDTH + HALO_MX4_MAX_WIDTH / 8 <= kOneSmem, "the widest row fits");
    const int most = 3 * kSmCount, want = (o.n_rows + 15) / 16;   // a pair of rows per warp at least
    return launch_chained(mx4_one_kernel<T>, want < most ? want : most, kOneThreads, 2 * o.d + o.d / 8, o.st, o.d, o.n_rows,
                          static_cast<const uint8_t*>(o.Qx), static_cast<const uint8_t*>(o.Sx), static_cast<const uint8_t*>(o.Qw),
                          static_cast<const uint8_t*>(o.Sw), y);
}

template <typename T, int NT, int STAGES>
halo_status launch_line(const Operands& o, T* y) {
    using R = Ring<NT, STAGES>;
    static bool done[64];
    if (!ensure_dynamic_smem(mx4_line_kernel<T, NT, STAGES>, R::kSmem, done)) return HALO_ERR_CUDA;
    CUtensorMap map_w, map_g, map_x;   // whole blocks of rows, groups of rows, tokens
    if (!make_byte_map(&map_w, o.Qw, o.n_rows, o.d / 2, kStageK / 2, kRowsTile) ||
        !make_byte_map(&map_g, o.Qw, o.n_rows, o.d / 2, kStageK / 2, 32) ||
        !make_byte_map(&map_x, o.Qx, o.n_tok, o.d / 2, kStageK / 2, NT))
        return HALO_ERR_CUDA;
    const int groups = (o.n_rows + 31) / 32, blocks = groups < kSmCount ? groups : kSmCount;
    return launch_chained(mx4_line_kernel<T, NT, STAGES>, blocks, kThreads, R::kSmem, o.st, map_w, map_g, map_x, o.d, o.n_tok, o.n_rows,
                          static_cast<const uint8_t*>(o.Sw), static_cast<const uint8_t*>(o.Sx), y, o.status);
}

template <typename T>
halo_status launch_pair(const Operands& o, T* y) {
    static bool done[64];
    if (!ensure_dynamic_smem(mx4_pair_kernel<T>, PairRing::kSmem, done)) return HALO_ERR_CUDA;
    CUtensorMap map_w, map_x, map_x64, map_sw, map_sx;
    if (!make_byte_map(&map_w, o.Qw, o.n_rows, o.d / 2, kStageK / 2, 128) ||
        !make_byte_map(&map_x, o.Qx, o.n_tok, o.d / 2, kStageK / 2, 128) ||
        !make_byte_map(&map_x64, o.Qx, o.n_tok, o.d / 2, kStageK / 2, 64) ||
        !make_scale_map(&map_sw, o.Sw, (o.n_rows + 127) / 128, o.d / 128, 1, 2) ||
        !make_scale_map(&map_sx, o.Sx, (o.n_tok + 127) / 128, o.d / 128, 2, 2))
        return HALO_ERR_CUDA;
    constexpr int kPairs = kSmCount / 2;
    PairTiles list;
    list.row_tiles = (o.n_rows + kPairTile - 1) / kPairTile;
    const int tiles = list.row_tiles * ((o.n_tok + kPairTile - 1) / kPairTile);   // at most 2^28
    const int rest = tiles % kPairs;
    list.halves = 2 * rest <= kPairs;
    list.whole = tiles - rest;
    list.items = tiles + (list.halves ? rest : 0);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2 * (list.items < kPairs ? list.items : kPairs));
    cfg.blockDim = dim3(kPairThreads);
    cfg.dynamicSmemBytes = PairRing::kSmem;
    cfg.stream = o.st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = 2;
    at[0].val.clusterDim.y = 1;
    at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;   // as in launch_chained
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    return cuda_status(cudaLaunchKernelEx(&cfg, mx4_pair_kernel<T>, map_w, map_x, map_x64, map_sw, map_sx, list, o.d, o.n_tok, o.n_rows, y,
                                          o.status));
}

template <typename T>
halo_status by_tokens(const Operands& o, void* y) {
    T* out = static_cast<T*>(y);
    // us, rows x d, the same weights call after call: up to some 100 MB come from L2 (11008 x 4096 for 8 to 64 tokens 7.4 to 7.6
    // so, 9.4 to 9.6 from HBM).  One token (one / line / pair): 4096 x 4096 4.2 / 5.6 / 7.0, 11008 x 4096 7.2 / 8.9 / 9.0, 24576 x 4096
    // 13.1 / 13.7 / 15.4, 4096 x 11008 8.0 / 10.9 / 12.5, 32000 x 8192 27.8 / 28.1 / 30.0; with more rows, or rows so short
    // that lanes of the one-token kernel stay idle, the line: 16384 x 2048 6.6 / 5.9 / 7.3, 32000 x 256 7.9 / 3.9 / 5.4,
    // 64000 x 5120 37.9 / 31.6 / 36.2.
    const long long rows = o.n_rows;
    if (o.n_tok == 1 && (rows <= 8192 || (rows <= 7ll * o.d && rows <= 32768))) return launch_one<T>(o, out);
    // 8 tokens (line / pair): 4096 x 4096 5.6 / 7.0, 11008 x 2048 5.8 / 6.0, 32000 x 2048 8.4 / 10.9, 24576 x 4096 13.8 / 14.9.
    // A second group of rows per SM costs the line as much as the first, the pairs take 256 x 74 rows at once: 6144 x 4096
    // 8.6 / 7.2, 11008 x 4096 9.0 / 7.9, 8192 x 11008 19.5 / 14.5, 32000 x 11008 37.2 / 34.2.  64 tokens in a line of their
    // own: 4096 x 4096 7.4 / 7.2, 11008 x 4096 10.8 / 7.6.
    const bool line = rows <= 32 * kSmCount || o.d <= 2048 || (rows > kPairTile * (kSmCount / 2) && o.d <= 4096);
    if ((line && o.n_tok <= 16) || o.n_tok == 1) return launch_line<T, 16, 10>(o, out);
    if (line && o.n_tok <= 32) return launch_line<T, 32, 9>(o, out);
    return launch_pair<T>(o, out);
}

}  // namespace
}  // namespace halo

using namespace halo;

extern "C" halo_status halo_product_mx4(int d_model, int n_tok, int n_rows, const void* Qx, const void* Sx, const void* Qw,
                                        const void* Sw, halo_dtype ydtype, void* y, uint32_t* dev_status, void* stream) {
    if (ydtype != HALO_F32 && ydtype != HALO_BF16) return HALO_ERR_DTYPE;
    if (d_model <= 0 || d_model % 128 != 0 || d_model > HALO_MX4_MAX_WIDTH || n_tok <= 0 || n_tok > HALO_MX4_MAX_TOKENS ||
        n_rows <= 0 || n_rows > HALO_MX4_MAX_ROWS)
        return HALO_ERR_SHAPE;
    if (!Qx || !Sx || !Qw || !Sw || !y) return HALO_ERR_ARG;
    if (!aligned16(Qx) || !aligned16(Sx) || !aligned16(Qw) || !aligned16(Sw) || !aligned16(y)) return HALO_ERR_ALIGN;
    const Operands o = {d_model, n_tok, n_rows, Qx, Sx, Qw, Sw, dev_status, static_cast<cudaStream_t>(stream)};
    return ydtype == HALO_F32 ? by_tokens<float>(o, y) : by_tokens<__nv_bfloat16>(o, y);
}
