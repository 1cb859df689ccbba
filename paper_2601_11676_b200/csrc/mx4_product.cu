// halo_product_mx4: y[t][r] = <x_t, w_r> of rows in microscaled 4-bit floating point, on the block-scaled tensor
// cores (tcgen05.mma kind::mxf4, products of 64 elements with a power of two per 32, fp32 accumulators in TMEM).
//
// The weight rows are the 128 rows of A and the tokens the columns of B, so one token costs a tile of 16 columns and
// not one of 128 rows, and a lane of the epilogue is a weight row: 32 lanes store 32 neighbouring outputs.
// Stages of 256 elements: 128-byte rows of codes by tensor-map TMA (128-byte swizzle), the scales as 512-byte blocks
// by bulk copies, moved on to TMEM by tcgen05.cp in front of the products that use them.  Every stage of the ring has
// its own columns of scales: a stage is refilled only when the products that read its old scales have completed.
//
// Bounds: few tokens HBM (0.53 bytes per weight element), prompts the tensor pipe.  With few tokens a cluster of up to
// 8 thread blocks shares a tile's elements and adds its parts through distributed shared memory in rank order.
//
// Every wait is bounded; when one runs out the block's roles leave their loops, the copies in flight are waited for,
// TMEM is freed and HALO_DEV_TIMEOUT is raised.
#include <cooperative_groups.h>

#include "common.cuh"
#include "umma.cuh"

namespace halo {

bool make_byte_map(CUtensorMap* map, const void* base, uint64_t rows, uint64_t row_bytes, uint32_t box_bytes, uint32_t box_rows);

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
__device__ __forceinline__ constexpr uint32_t idesc_mxf4(int n, uint32_t sf) {
    return (sf << 4)                                // scale bytes of B
           | (1u << 7)                              // A: e2m1
           | (1u << 10)                             // B: e2m1
           | (static_cast<uint32_t>(n >> 3) << 17)  // N / 8
           | (1u << 23)                             // scales: powers of two
           | (static_cast<uint32_t>(kRowsTile >> 7) << 27)
           | (sf << 29);                            // scale bytes of A
}
// 512 bytes of shared memory (32 rows of 16 bytes) -> 4 columns, repeated in the four quarters of the lanes
__device__ __forceinline__ void tmem_cp_scales(uint32_t taddr, uint32_t smem) {
    const uint64_t desc = static_cast<uint64_t>((smem & 0x3FFFFu) >> 4) | (static_cast<uint64_t>(128u >> 4) << 32) | (1ull << 46);
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}

template <int NT, int STAGES>
struct Ring {
    static constexpr int kA = kRowsTile * (kStageK / 2);
    static constexpr int kB = NT * (kStageK / 2);
    static constexpr int kTokTiles = (NT + 127) / 128;
    static constexpr int kSfa = 1024, kSfb = 1024 * kTokTiles;
    static constexpr int kStage = kA + kB + kSfa + kSfb;
    static constexpr int kSfCols = 8 + 8 * kTokTiles;
    static constexpr int kCols = NT + STAGES * kSfCols;
    static constexpr int kTmem = kCols <= 32 ? 32 : kCols <= 64 ? 64 : kCols <= 128 ? 128 : kCols <= 256 ? 256 : 512;
    static constexpr size_t kBars = 256;
    static constexpr size_t kSmem = static_cast<size_t>(STAGES) * kStage + kBars;
    static_assert(kCols <= 512, "tensor memory");
    static_assert(kStage % 1024 == 0, "swizzled tiles start on 1024 bytes");
};

struct Bars {
    uint64_t full[8], empty[8], done;
    uint32_t tmem;
    int abort_flag;
};

template <typename T, int NT, int STAGES>
__global__ void __launch_bounds__(kThreads)
mx4_product_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x, int d, int n_tok,
                   int n_rows, const uint8_t* __restrict__ Sw, const uint8_t* __restrict__ Sx, T* __restrict__ y, int split,
                   uint32_t* status) {
    using R = Ring<NT, STAGES>;
    extern __shared__ __align__(1024) unsigned char smem[];
    Bars& bars = *reinterpret_cast<Bars*>(smem + static_cast<size_t>(STAGES) * R::kStage);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int rank = blockIdx.x % split;
    const int rt = blockIdx.x / split, tt = blockIdx.y;
    const int row0 = rt * kRowsTile, tok0 = tt * NT;
    const int atoms = d / 128;                       // 512-byte blocks of scales along a row
    const int nk = (d + kStageK - 1) / kStageK;
    const int k0 = nk * rank / split, k1 = nk * (rank + 1) / split;

    if (tid == 0) {
        for (int s = 0; s < STAGES; ++s) { mbar_init(&bars.full[s], 1); mbar_init(&bars.empty[s], 1); }
        mbar_init(&bars.done, 1);
        bars.abort_flag = 0;
        mbar_fence_init();
        tma_prefetch_descriptor(&map_w);
        tma_prefetch_descriptor(&map_x);
    }
    if (warp == 1) { tmem_alloc(&bars.tmem, R::kTmem); tmem_relinquish_alloc_permit(); }
    tcgen05_fence_before_sync();
    __syncthreads();
    tcgen05_fence_after_sync();
    volatile int* abort_flag = &bars.abort_flag;
    const uint32_t tmem = bars.tmem;

    if (warp == 0) {
        if (lane == 0) {
            int it = 0;
            for (int k = k0; k < k1; ++k, ++it) {
                const int s = it % STAGES;
                if (it >= STAGES && !mbar_wait_bounded(&bars.empty[s], ((it / STAGES) - 1) & 1, abort_flag)) {
                    *abort_flag = 1;
                    break;
                }
                unsigned char* st = smem + static_cast<size_t>(s) * R::kStage;
                const uint32_t n_at = min(2, atoms - k * 2);
                const int tiles = min(R::kTokTiles, (n_tok - tok0 + 127) / 128);
                mbar_arrive_expect_tx(&bars.full[s], R::kA + R::kB + n_at * 512u * (1 + tiles));
                tma_load_2d(st, &map_w, k * (kStageK / 2), row0, &bars.full[s]);
                tma_load_2d(st + R::kA, &map_x, k * (kStageK / 2), tok0, &bars.full[s]);
                bulk_copy_g2s(st + R::kA + R::kB, Sw + (static_cast<size_t>(rt) * atoms + k * 2) * 512, n_at * 512u, &bars.full[s]);
                for (int t = 0; t < tiles; ++t)
                    bulk_copy_g2s(st + R::kA + R::kB + R::kSfa + t * 1024,
                                  Sx + (static_cast<size_t>(tok0 / 128 + t) * atoms + k * 2) * 512, n_at * 512u, &bars.full[s]);
            }
            if (*abort_flag) {
                int never = 0;
                for (int i = max(0, it - STAGES); i < it; ++i) mbar_wait_bounded(&bars.full[i % STAGES], (i / STAGES) & 1, &never);
            }
        }
    } else if (warp == 1) {
        if (lane == 0) {
            int it = 0;
            for (int k = k0; k < k1; ++k, ++it) {
                const int s = it % STAGES;
                if (!mbar_wait_bounded(&bars.full[s], (it / STAGES) & 1, abort_flag)) { *abort_flag = 1; break; }
                tcgen05_fence_after_sync();
                const uint32_t st = smem_u32(smem + static_cast<size_t>(s) * R::kStage);
                const uint32_t sfa = tmem + NT + s * R::kSfCols, sfb = sfa + 8;
                const int n_at = min(2, atoms - k * 2);
                for (int at = 0; at < n_at; ++at) {
                    tmem_cp_scales(sfa + at * 4, st + R::kA + R::kB + at * 512);
#pragma unroll
                    for (int t = 0; t < R::kTokTiles; ++t)
                        tmem_cp_scales(sfb + (at * R::kTokTiles + t) * 4, st + R::kA + R::kB + R::kSfa + t * 1024 + at * 512);
                }
                for (int j = 0; j < n_at * 2; ++j) {
                    const uint32_t sf = (j & 1) * 2;
                    umma_mxf4(tmem, umma_smem_desc(st + j * 32, 0, 1024), umma_smem_desc(st + R::kA + j * 32, 0, 1024),
                              idesc_mxf4(NT, sf), sfa + (j >> 1) * 4, sfb + (j >> 1) * 4 * R::kTokTiles, it > 0 || j > 0);
                }
                umma_commit(&bars.empty[s]);
            }
            umma_commit(&bars.done);
        }
    }
    if (warp >= 2) {
        const bool ok = __all_sync(0xffffffffu, mbar_wait_bounded(&bars.done, 0, abort_flag));
        if (!ok) *abort_flag = 1;
        tcgen05_fence_after_sync();
        const int quad = warp & 3, row = row0 + quad * 32 + lane;
        const uint32_t base = tmem + (static_cast<uint32_t>(quad * 32) << 16);
        const int cols = min(NT, n_tok - tok0);
        float* part = reinterpret_cast<float*>(smem);   // [cols][128]: the ring is drained
        for (int c0 = 0; c0 < cols; c0 += 16) {
            uint32_t v[16];
            tmem_ld_32x16(base + c0, v);
            tmem_ld_wait();
            if (!ok) continue;
#pragma unroll
            for (int c = 0; c < 16; ++c) {
                if (c0 + c >= cols) break;
                const float f = k1 > k0 ? __uint_as_float(v[c]) : 0.0f;
                if (split > 1)
                    part[(c0 + c) * kRowsTile + quad * 32 + lane] = f;
                else if (row < n_rows)
                    y[static_cast<long long>(tok0 + c0 + c) * n_rows + row] = from_float<T>(f);
            }
        }
    }
    __syncwarp();   // warps 0 and 1 worked with one lane
    tcgen05_fence_before_sync();
    if (split > 1) {
        namespace cg = cooperative_groups;
        cg::cluster_group cl = cg::this_cluster();
        cl.sync();
        // rank r adds up its share of the outputs over the thread blocks, in rank order
        const int cols = min(NT, n_tok - tok0);
        const float* part = reinterpret_cast<const float*>(smem);
        for (int i = tid + rank * kThreads; i < cols * kRowsTile; i += kThreads * split) {
            const int row = row0 + i % kRowsTile;
            float sum = 0.0f;
            for (int r = 0; r < split; ++r) sum += *cl.map_shared_rank(part + i, r);
            if (row < n_rows) y[static_cast<long long>(tok0 + i / kRowsTile) * n_rows + row] = from_float<T>(sum);
        }
        cl.sync();
    } else {
        __syncthreads();
    }
    if (warp == 1) { tcgen05_fence_after_sync(); tmem_dealloc(tmem, R::kTmem); }
    if (tid == 0 && *abort_flag) flag_status(status, HALO_DEV_TIMEOUT);
}

template <typename T, int NT, int STAGES>
halo_status launch(int d, int n_tok, int n_rows, const void* Qx, const void* Sx, const void* Qw, const void* Sw, T* y,
                   uint32_t* status, cudaStream_t st) {
    using R = Ring<NT, STAGES>;
    static bool done[64];
    if (!ensure_dynamic_smem(mx4_product_kernel<T, NT, STAGES>, R::kSmem, done)) return HALO_ERR_CUDA;
    CUtensorMap map_w, map_x;
    if (!make_byte_map(&map_w, Qw, n_rows, d / 2, kStageK / 2, kRowsTile) ||
        !make_byte_map(&map_x, Qx, n_tok, d / 2, kStageK / 2, NT))
        return HALO_ERR_CUDA;
    const int tiles = (n_rows + kRowsTile - 1) / kRowsTile, tok_tiles = (n_tok + NT - 1) / NT;
    const int nk = (d + kStageK - 1) / kStageK;
    int split = 1;
    if (NT <= 64)
        while (split < 8 && split * 2 <= nk && tiles * tok_tiles * split < 4 * kSmCount) split *= 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(tiles * split, tok_tiles);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = R::kSmem;
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = split;
    at[0].val.clusterDim.y = 1;
    at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cuda_status(cudaLaunchKernelEx(&cfg, mx4_product_kernel<T, NT, STAGES>, map_w, map_x, d, n_tok, n_rows,
                                          static_cast<const uint8_t*>(Sw), static_cast<const uint8_t*>(Sx), y, split, status));
}

template <typename T>
halo_status by_tokens(int d, int n_tok, int n_rows, const void* Qx, const void* Sx, const void* Qw, const void* Sw, void* y,
                      uint32_t* status, cudaStream_t st) {
    T* out = static_cast<T*>(y);
    if (n_tok <= 16) return launch<T, 16, 5>(d, n_tok, n_rows, Qx, Sx, Qw, Sw, out, status, st);
    if (n_tok <= 64) return launch<T, 64, 4>(d, n_tok, n_rows, Qx, Sx, Qw, Sw, out, status, st);
    return launch<T, 256, 4>(d, n_tok, n_rows, Qx, Sx, Qw, Sw, out, status, st);
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
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    return ydtype == HALO_F32 ? by_tokens<float>(d_model, n_tok, n_rows, Qx, Sx, Qw, Sw, y, dev_status, st)
                              : by_tokens<__nv_bfloat16>(d_model, n_tok, n_rows, Qx, Sx, Qw, Sw, y, dev_status, st);
}
