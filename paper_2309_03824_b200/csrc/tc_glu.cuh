// Tensor-core kernel (sm_100a) of gated feed-forward blocks and of products in 8-bit integers.
//   gated:  out[M x N] = act(G) * U,  [G | U] = P = X W^T + bias, W[2N x K]; P kept on request
//   plain:  out[M x N] = X W^T + bias, W[N x K]                                       (8-bit operands only)
// bf16 operands accumulate in fp32.  8-bit operands accumulate exactly in 32-bit integers; sum, row scale of X and row scale of W are
// multiplied in fp32 in the epilogue, so the result is off by three roundings of 2^-24 before its own.
//
// The gate costs no traffic: a tile's B operand is made of BN / 2 rows of W's upper half (gate) and the same rows of its lower half,
// so that one accumulator holds G in its first BN / 2 columns and U in the others, and a thread that reads its row of
// tensor memory has both factors of every H in hand.  On pairs of SMs (CG = 2, 256-row MMAs) each block loads half of B: the even
// one the gate's rows, the odd one the others.  A k-block is 128 bytes of a row (64 bf16 or 128 8-bit values) and four MMAs
// either way, and the swizzled layouts are the same, so both operand types share everything but the MMA and the epilogue's
// conversion.  There W's scale comes first: weights are of moderate size, so sum times scale is, and times the row's scale it passes
// fp32's range only where the result does (rows of 1e35 times the other way round: infinity).
//
// One block per SM walks over the tiles (tile_at: blocks working at the same time share X and W in L2); accumulators are double-buffered
// in tensor memory and the epilogue of a tile overlaps the MMAs of the next.
//
// ONE: tiles of any width, for calls of at most 128 rows of X (and split ones).  Such a call moves little but W, so its tiles are as
// wide as spreads W evenly over the SMs (any multiple of 16 columns of the output: p.hc), and a stage holds only the rows of X there
// are (p.a_rows), which leaves the rest of shared memory to W in flight.  The MMAs still read 128 rows -- what stands behind X's in shared memory, within the block's own
// -- and the rows past M are never looked at (a row of the product depends on its own row of X alone).
//
// SPLIT: a tile's reduction over the blocks of a cluster, one tile a cluster, for calls of few tiles over a long reduction.  A narrow tile's
// MMA takes as long as one four times as wide, so wide tiles over a part of K each beat narrow ones over all of it.  When all
// MMAs of the cluster are done, each block owns some 32-column pieces, gets the others' sums of them into the shared memory that the ring
// had (its own rows only), adds them in rank order and goes on as ever: the same bits every time.
//
// Warp 0: TMA producer.  Warp 1: tensor memory + MMA issue.  Warps 2-9: epilogue, two to each quarter of tensor memory's rows (with four,
// 4096 x 1024 -> 2816 gated in bf16 took 36.7 us instead of 33.9).  Every wait for a
// barrier in shared memory is bounded; a cluster's own barriers are met by all its warps, those that gave up too.
#pragma once
#include "glu.cuh"
#include "ptx_pair.cuh"
#include "tc.cuh"
#include "tma.cuh"

namespace lrd {
namespace glu {

using namespace ptx;

constexpr int BM = 128;
constexpr uint32_t kRow = 128;                               // bytes of K per k-block
constexpr int kEpilogueWarps = 8, kShare = kEpilogueWarps / 4, kThreads = 64 + 32 * kEpilogueWarps;
constexpr uint32_t kTableBytes = 1024;                       // one epilogue warp's per-column values of a tile
constexpr int kMaxStages = 16;
constexpr uint32_t kAllSmem = 232448 - 1024;                 // of a block, beside its static variables

// GK: k-blocks per stage (the issue loop's cost is per stage)
template <bool GATED, typename OUT, int BN, int CG, int GK, bool ONE> struct Cfg {
    static_assert(!ONE || (CG == 1 && BN == 256), "tiles of any width: single blocks, up to 256 accumulator columns");
    static constexpr int BNH = BN / CG;                      // rows of W this block loads
    static constexpr int HC = GATED ? BN / 2 : BN;           // columns of the output in a tile
    static constexpr int PW = 32;                            // an epilogue step: 32 rows x 32 columns of the output
    static constexpr int PIECES = (HC + PW - 1) / PW, PER_WARP = (PIECES + kShare - 1) / kShare;
    static constexpr int TABLES = GATED ? 4 : 2;             // bias and scale of each column
    static_assert(PER_WARP * TABLES * 32 * 4 <= (int)kTableBytes, "per-column values");
    static constexpr int G = GK;
    static constexpr uint32_t A_TILE = BM * kRow, B_TILE = BNH * kRow;                 // ONE: p.a_rows and p.hc rows in their place
    static constexpr uint32_t STAGE_BYTES = G * (A_TILE + B_TILE);
    static constexpr uint32_t SLAB_BYTES = 32 * PW * sizeof(OUT);
    static constexpr int SLABS = 2;
    static constexpr uint32_t STAGING = kEpilogueWarps * SLABS * SLAB_BYTES, FIXED = STAGING + kEpilogueWarps * kTableBytes + 1024;
    static constexpr uint32_t RING_MAX = kAllSmem - FIXED;
    static constexpr int STAGES_RAW = RING_MAX / STAGE_BYTES;
    static constexpr int STAGES = STAGES_RAW > 8 ? 8 : STAGES_RAW;
    static_assert(ONE || STAGES >= 3, "ring");
    static constexpr uint32_t SMEM_BYTES = FIXED + STAGES * STAGE_BYTES;
    static constexpr uint32_t TMEM_COLS = 2 * BN <= 128 ? 128 : 2 * BN <= 256 ? 256 : 512;
    static constexpr uint32_t BUF_COLS = TMEM_COLS / 2;
};

// ordinary stores of single elements or of 16 bytes, or TMA
enum { kByElements, kByPieces, kByTma };

struct Params {
    int64_t M, N;
    int kb_total, m_tiles, n_tiles, m_group, tiles;
    const void* bias;
    const float *x_scale, *w_scale;
    void* out; int64_t ldo;
    void* p_save; int64_t ldp;
    int out_by, p_by;         // how these leave (kByElements, kByPieces, kByTma)
    int act;
    int hc, a_rows, stages;   // ONE: columns of the output in a tile, rows of X in a stage, stages
    int split, kb_share, own_pieces;      // SPLIT: blocks of a cluster, k-blocks of each, 32-column pieces each owns at most
    unsigned int* timeout_flag;
};

// 8-bit x 8-bit -> 32-bit integers, 32 deep
__device__ __forceinline__ void mma_i8_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(acc) : "memory");
}
__device__ __forceinline__ void mma_i8_ss_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(acc) : "memory");
}
// both operands signed 8-bit and K-major, 32-bit integer sums, M = 128 CG rows, N = n
__host__ __device__ constexpr uint32_t idesc_i8(int n, int cg) {
    return (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(128 * cg >> 4) << 24);
}

template <typename OUT> __device__ __forceinline__ float out_to_f32(OUT x) { return (float)x; }

// A warp's 32 x PW values (lane = row) -> its slab, in the layout of a swizzled TMA box of that width
template <typename OUT, int PW> __device__ __forceinline__ uint32_t slab_xor(uint32_t row) {
    constexpr uint32_t bytes = PW * sizeof(OUT);
    return bytes == 128 ? row & 7u : bytes == 64 ? (row >> 1) & 3u : (row >> 2) & 1u;
}
template <typename OUT, int PW> __device__ __forceinline__ void put_slab(uint32_t slab, const uint64_t (&v)[PW / 2]) {
    const uint32_t lane = threadIdx.x & 31u, at = slab + lane * (PW * sizeof(OUT)), x = slab_xor<OUT, PW>(lane);
    if constexpr (sizeof(OUT) == 2) {
        auto two = [](uint64_t p) {
            float a, b;
            pair_split(p, a, b);
            return pack_bf16(a, b);
        };
#pragma unroll
        for (uint32_t c = 0; c < PW / 8; ++c) st_shared_v4(at + ((c ^ x) << 4), two(v[4 * c]), two(v[4 * c + 1]), two(v[4 * c + 2]), two(v[4 * c + 3]));
    } else {
#pragma unroll
        for (uint32_t c = 0; c < PW / 4; ++c)
            st_shared_v4(at + ((c ^ x) << 4), (uint32_t)v[2 * c], (uint32_t)(v[2 * c] >> 32), (uint32_t)v[2 * c + 1], (uint32_t)(v[2 * c + 1] >> 32));
    }
}
// The slab's rows and columns that exist, by ordinary stores: to rows of any stride and alignment a lane a column, or (by 16 bytes) to
// such whose 16-byte pieces lie on boundaries and exist as a whole
template <typename OUT, int PW> __device__ __forceinline__ void store_slab(uint32_t slab, OUT* dst, int64_t ld, int64_t rows, int64_t cols, bool pieces) {
    constexpr uint32_t ROW = PW * sizeof(OUT), PER = ROW / 16, STEP = 32 / PER;        // pieces of a row, rows an instruction covers
    const uint32_t lane = threadIdx.x & 31u;
    if (pieces) {
        const uint32_t c = lane % PER;
#pragma unroll
        for (uint32_t r = lane / PER; r < 32; r += STEP) {
            uint4 v;
            asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(slab + r * ROW + ((c ^ slab_xor<OUT, PW>(r)) << 4)));
            if (r < rows && c * (16 / sizeof(OUT)) < cols) *reinterpret_cast<uint4*>(dst + r * ld + c * (16 / sizeof(OUT))) = v;
        }
        return;
    }
    const uint32_t byte = lane * sizeof(OUT);
#pragma unroll 8
    for (uint32_t r = 0; r < 32; ++r) {
        if (r >= rows) break;                                // (uniform)
        const uint32_t at = slab + r * ROW + (((byte >> 4) ^ slab_xor<OUT, PW>(r)) << 4) + (byte & 15u);
        if constexpr (sizeof(OUT) == 2) {
            uint16_t v;
            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(at));
            if (lane < cols) dst[r * ld + lane] = __ushort_as_bfloat16(v);
        } else {
            float v;
            asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(at));
            if (lane < cols) dst[r * ld + lane] = v;
        }
    }
}
// 16 bytes into the shared memory of block `rank` of the cluster, at this block's address of the place
__device__ __forceinline__ void st_cluster_v4(uint32_t addr, uint32_t rank, const uint32_t* v) {
    asm volatile("st.shared::cluster.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(map_to_cta(addr, rank)), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
}

template <bool I8, bool GATED, typename OUT, int BN, int CG, int GK, bool ONE, bool SPLIT>
__global__ void __launch_bounds__(kThreads, 1)
tc_glu_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const __grid_constant__ CUtensorMap tmO,
              const __grid_constant__ CUtensorMap tmG, const __grid_constant__ CUtensorMap tmU, const Params p) {
    using C = Cfg<GATED, OUT, BN, CG, GK, ONE>;
    constexpr int G = C::G, PW = C::PW;
    constexpr bool EXACT = sizeof(OUT) == 4;
    static_assert(ONE || !SPLIT, "a split reduction has tiles of any width");
    const int STAGES = ONE ? p.stages : C::STAGES, HC = ONE ? p.hc : C::HC;
    const uint32_t A_TILE = ONE ? (uint32_t)p.a_rows * kRow : C::A_TILE, B_TILE = ONE ? (uint32_t)(GATED ? 2 * p.hc : p.hc) * kRow : C::B_TILE;
    const uint32_t STAGE_BYTES = G * (A_TILE + B_TILE);
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t full_bar[kMaxStages], empty_bar[kMaxStages], out_full[2], out_empty[2];
    __shared__ uint32_t tmem_base_slot;
    __shared__ int abort_flag;

    const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t staging_base = smem_base, ring_base = smem_base + C::STAGING + kEpilogueWarps * kTableBytes;
    float* const tables = reinterpret_cast<float*>(smem_raw + (smem_base - smem_u32(smem_raw)) + C::STAGING);
    const AbortCtx ab{&abort_flag, p.timeout_flag};
    const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x / 32, 0), lane = threadIdx.x % 32;
    const int h = CG == 2 ? (int)cluster_ctarank() : 0;      // this block's half of the pair
    const int blocks = SPLIT ? p.split : CG, unit = (int)blockIdx.x / blocks, n_units = (int)gridDim.x / blocks;
    const int rank = SPLIT ? (int)cluster_ctarank() : 0;     // this block's share of the reduction
    const int kb_first = SPLIT ? rank * p.kb_share : 0, kb_end = SPLIT ? min(p.kb_total, kb_first + p.kb_share) : p.kb_total;

    if (threadIdx.x == 0) {
        abort_flag = 0;
        prefetch_tmap(&tmA);
        prefetch_tmap(&tmB);
        if (p.out_by == kByTma) prefetch_tmap(&tmO);
        if (GATED && p.p_by == kByTma) {
            prefetch_tmap(&tmG);
            prefetch_tmap(&tmU);
        }
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(smem_u32(&full_bar[s]), 1);
            mbar_init(smem_u32(&empty_bar[s]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&out_full[i]), 1);
            mbar_init(smem_u32(&out_empty[i]), kEpilogueWarps * CG);     // the epilogue warps of every block of the pair
        }
        fence_mbar_init();
    }
    if (warp == 1) {
        if (CG == 2) {
            tmem_alloc_pair(smem_u32(&tmem_base_slot), C::TMEM_COLS);
            tmem_relinquish_pair();
        } else {
            tmem_alloc(smem_u32(&tmem_base_slot), C::TMEM_COLS);
            tmem_relinquish();
        }
    }
    tc_fence_before();
    if (CG == 2) {                   // the other block's barriers exist before anything signals them
        cluster_arrive();
        cluster_wait();
    } else {
        __syncthreads();
    }
    tc_fence_after();
    const uint32_t tmem_base = tmem_base_slot;
    griddep_wait();                  // what stands above touched only this block's own shared and tensor memory
    if (warp != 0) griddep_launch_dependents();

    if (warp == 0) {
        // ------------------------------------------------------------------ TMA producer
        int s = 0;
        uint32_t ph = 1;
        bool ok = true;
        auto load = [&](uint32_t dst, const CUtensorMap* m, uint32_t bar, int x, int y) {
            if (CG == 2) tma_load_2d_pair(dst, m, bar, x, y);
            else tma_load_2d(dst, m, bar, x, y);
        };
        constexpr int KE = I8 ? 128 : 64;                    // elements of a k-block
        for (int t = unit; t < p.tiles && ok; t += n_units) {
            int mt, nt;
            tile_at(t, p.m_tiles, p.n_tiles, p.m_group, mt, nt);
            const int m0 = mt * (BM * CG) + h * BM, n0 = nt * HC;
            for (int kb = kb_first; kb < kb_end; kb += G) {     // k-blocks past the last read as zeros
                ok = mbar_wait_uniform(smem_u32(&empty_bar[s]), ph, ab);
                if (!ok) break;
                const uint32_t fb = CG == 2 ? map_to_cta(smem_u32(&full_bar[s]), 0) : smem_u32(&full_bar[s]);
                const uint32_t a_dst = ring_base + s * STAGE_BYTES, b_dst = a_dst + G * A_TILE;
                if (elect_one()) {
                    if (h == 0) mbar_expect_tx(smem_u32(&full_bar[s]), CG * STAGE_BYTES);
#pragma unroll
                    for (int g = 0; g < G; ++g) {
                        load(a_dst + g * A_TILE, &tmA, fb, (kb + g) * KE, m0);
                        const uint32_t b = b_dst + g * B_TILE;
                        if (!GATED) {
                            load(b, &tmB, fb, (kb + g) * KE, n0 + h * C::BNH);
                        } else if (CG == 2) {
                            load(b, &tmB, fb, (kb + g) * KE, n0 + (h ? (int)p.N : 0));
                        } else {
                            load(b, &tmB, fb, (kb + g) * KE, n0);
                            load(b + HC * kRow, &tmB, fb, (kb + g) * KE, n0 + (int)p.N);
                        }
                    }
                }
                __syncwarp();
                if (++s == STAGES) { s = 0; ph ^= 1; }
            }
        }
    } else if (warp == 1 && h == 0) {
        // ------------------------------------------------------------------ MMA issuer (the even block of a pair)
        const int cols = ONE ? (GATED ? 2 * HC : HC) : BN;
        const uint32_t idesc = I8 ? idesc_i8(cols, CG) : CG == 2 ? idesc_bf16_pair(cols, false, false) : idesc_bf16(cols, false, false);
        const uint64_t a_desc0 = smem_desc_sw128(ring_base, 0, 1024), b_desc0 = smem_desc_sw128(ring_base + G * A_TILE, 0, 1024);
        int s = 0, i = 0;
        uint32_t ph = 0;
        bool ok = true;
        for (int t = unit; t < p.tiles && ok; t += n_units, ++i) {
            const int buf = i & 1;
            const uint32_t d_tmem = tmem_base + (uint32_t)buf * C::BUF_COLS;
            ok = mbar_wait_uniform(smem_u32(&out_empty[buf]), ((i >> 1) & 1) ^ 1, ab);      // accumulator buffer drained
            tc_fence_after();
            uint32_t ready = mbar_test_wait(smem_u32(&full_bar[s]), ph);
            for (int kb = kb_first; kb < kb_end && ok; kb += G) {
                ok = mbar_wait_peeked(ready, smem_u32(&full_bar[s]), ph, ab);
                if (!ok) break;
                tc_fence_after();
                const uint64_t ad = a_desc0 + (uint32_t)s * (STAGE_BYTES >> 4), bd = b_desc0 + (uint32_t)s * (STAGE_BYTES >> 4);
                const uint32_t eb = smem_u32(&empty_bar[s]);
                const bool last = kb + G >= kb_end;
                if (++s == STAGES) { s = 0; ph ^= 1; }
                ready = last ? 0u : mbar_test_wait(smem_u32(&full_bar[s]), ph);
                if (elect_one()) {
#pragma unroll
                    for (int g = 0; g < G; ++g) {
                        if (g > 0 && kb + g >= kb_end) break;
#pragma unroll
                        for (int kk = 0; kk < 4; ++kk) {     // 32 bytes of K each
                            const uint64_t a = ad + (g * (A_TILE >> 4) + kk * 2u), b = bd + (g * (B_TILE >> 4) + kk * 2u);
                            const uint32_t acc = g > 0 || kk > 0 ? 1u : (kb > kb_first ? 1u : 0u);
                            if (I8) {
                                if (CG == 2) mma_i8_ss_pair(d_tmem, a, b, idesc, acc);
                                else mma_i8_ss(d_tmem, a, b, idesc, acc);
                            } else {
                                if (CG == 2) mma_bf16_ss_pair(d_tmem, a, b, idesc, acc);
                                else mma_bf16_ss(d_tmem, a, b, idesc, acc);
                            }
                        }
                    }
                    if (CG == 2) {       // both blocks' stages are free, both blocks' accumulators are ready
                        mma_commit_pair(eb, 3);
                        if (last) mma_commit_pair(smem_u32(&out_full[buf]), 3);
                    } else {
                        mma_commit(eb);
                        if (last) mma_commit(smem_u32(&out_full[buf]));
                    }
                }
                __syncwarp();
            }
        }
    } else if (warp >= 2) {
        // ------------------------------------------------------------------ epilogue
        const int q = warp % 4;                              // tensor-memory lanes [32 q, 32 q + 32)
        const int hw = (warp - 2) / 4;                       // the warps of a quarter take its pieces in turn
        const uint32_t lane_addr = tmem_base + ((uint32_t)(q * 32) << 16);
        const uint32_t slab0 = staging_base + (uint32_t)(warp - 2) * C::SLABS * C::SLAB_BYTES;
        float* const table = tables + (warp - 2) * (kTableBytes / 4);
        const OUT* const bias = (const OUT*)p.bias;
        // this warp's piece j of a tile (SPLIT: of those that the block owns; past the last: a piece that no tile has)
        auto piece = [&](int j) {
            const int own = hw + kShare * j;
            return !SPLIT ? own : own < p.own_pieces ? rank * p.own_pieces + own : BN;
        };
        // bias and scale of this warp's columns, and the scale of this lane's row, fetched a tile ahead
        float ahead[C::PER_WARP][C::TABLES], x_ahead = 0.0f;
        auto fetch = [&](int t) {
            int mt, nt;
            tile_at(t, p.m_tiles, p.n_tiles, p.m_group, mt, nt);
            const int64_t row = (int64_t)mt * (BM * CG) + h * BM + q * 32 + lane, n0 = (int64_t)nt * HC;
#pragma unroll
            for (int j = 0; j < C::PER_WARP; ++j) {
                const int64_t col = n0 + piece(j) * PW + lane;
                const bool in = t < p.tiles && col < p.N;
#pragma unroll
                for (int half = 0; half < (GATED ? 2 : 1); ++half) {
                    ahead[j][2 * half] = bias && in ? out_to_f32(bias[half * p.N + col]) : 0.0f;
                    ahead[j][2 * half + 1] = I8 && in ? p.w_scale[half * p.N + col] : 0.0f;
                }
            }
            if (I8) x_ahead = t < p.tiles && row < p.M ? p.x_scale[row] : 0.0f;
        };
        fetch(unit);
        int i = 0, sb = 0;
        bool ok = true;
        for (int t = unit; t < p.tiles && ok; t += n_units, ++i) {
            const int buf = i & 1;
            int mt, nt;
            tile_at(t, p.m_tiles, p.n_tiles, p.m_group, mt, nt);
            const int64_t m0 = (int64_t)mt * (BM * CG) + h * BM + q * 32, n0 = (int64_t)nt * HC;
            const bool rows_inside = m0 < p.M;               // (uniform) a tile may hang over the last row
            const int64_t n_end = ONE && n0 + HC < p.N ? n0 + HC : p.N;      // (ONE: the last piece may pass the tile's columns)
            __syncwarp();
#pragma unroll
            for (int j = 0; j < C::PER_WARP; ++j)
#pragma unroll
                for (int e = 0; e < C::TABLES; ++e) table[(j * C::TABLES + e) * 32 + lane] = ahead[j][e];
            const float x_scale = x_ahead;
            __syncwarp();
            fetch(t + n_units);
            ok = mbar_wait_uniform(smem_u32(&out_full[buf]), (i >> 1) & 1, ab);
            if (!ok) break;
            tc_fence_after();
            const uint32_t d_tmem = lane_addr + (uint32_t)buf * C::BUF_COLS;
            // SPLIT: where block `from`'s sums of this lane's row stand in the block that owns them (piece `own` of its, G or U)
            const uint32_t row_cap = SPLIT ? ((uint32_t)p.a_rows + 31u) & ~31u : 0u, tile_row = (uint32_t)(q * 32 + lane);
            auto sums_at = [&](int from, int own, int half) {
                return ring_base + ((uint32_t)((from * p.own_pieces + own) * (GATED ? 2 : 1) + half) * row_cap + tile_row) * 128u;
            };
            if constexpr (SPLIT) {
                cluster_arrive();                            // every block's ring is dead: its own MMAs have read it, and nothing more is loaded
                cluster_wait();
                for (int c = hw; c * PW < HC && rows_inside; c += kShare) {
                    const int owner = c / p.own_pieces, own = c - owner * p.own_pieces;
                    if (owner == rank) continue;             // (uniform)
#pragma unroll
                    for (int half = 0; half < (GATED ? 2 : 1); ++half) {
                        uint32_t v[PW];
                        tmem_ld_32x32(d_tmem + half * HC + c * PW, v);
                        tmem_ld_wait();
                        if (m0 + lane < p.M)
#pragma unroll
                            for (uint32_t e = 0; e < 8; ++e) st_cluster_v4(sums_at(rank, own, half) + ((e ^ (tile_row & 7u)) << 4), (uint32_t)owner, v + 4 * e);
                        __syncwarp();                        // (lanes past the last row stood aside; the next load is the whole warp's)
                    }
                }
                cluster_arrive();                            // (release / acquire: every block's sums have landed)
                cluster_wait();
            }
            // accumulators of piece c
            auto take = [&](int c, int half, uint32_t (&v)[PW]) {
                tmem_ld_32x32(d_tmem + half * HC + c * PW, v);
                if constexpr (SPLIT) {
                    tmem_ld_wait();
                    uint32_t sum[PW] = {};
                    for (int from = 0; from < p.split; ++from) {
                        const uint32_t at = sums_at(from, c - rank * p.own_pieces, half);
#pragma unroll
                        for (uint32_t e = 0; e < 8; ++e) {
                            uint32_t w[4] = {v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]};
                            if (from != rank)
                                asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at + ((e ^ (tile_row & 7u)) << 4)));
#pragma unroll
                            for (int x = 0; x < 4; ++x)
                                sum[4 * e + x] = I8 ? sum[4 * e + x] + w[x] : __float_as_uint(__uint_as_float(sum[4 * e + x]) + __uint_as_float(w[x]));
                        }
                    }
#pragma unroll
                    for (int e = 0; e < PW; ++e) v[e] = sum[e];
                }
            };
            // 32 x 32 values out: slab, then TMA or the rows themselves.  Before a slab is written again, the store that last read
            // it has.
            auto emit = [&](const uint64_t (&v)[PW / 2], const CUtensorMap* m, int by, OUT* base, int64_t ld, int64_t col) {
                const bool tma = !ONE && by == kByTma;
                const uint32_t slab = slab0 + (C::SLABS == 2 ? (uint32_t)(sb & 1) * C::SLAB_BYTES : 0u);
                if (sb >= C::SLABS) tma_store_wait_read<C::SLABS - 1>();
                ++sb;
                __syncwarp();
                put_slab<OUT, PW>(slab, v);
                if (tma) fence_proxy_async_smem();
                __syncwarp();
                if (!tma) store_slab<OUT, PW>(slab, base + m0 * ld + col, ld, p.M - m0, n_end - col, by != kByElements);
                if (elect_one()) {                           // (a group each time, an empty one behind ordinary stores)
                    if (tma) tma_store_2d(m, slab, (int)col, (int)m0);
                    tma_store_commit();
                }
                __syncwarp();
            };
            // accumulators -> the projection's 32 columns, a pair at a time; at: their bias, their scales 32 further on
            const uint64_t x_scale2 = pair_both(x_scale);
            auto project = [&](uint64_t (&v)[PW / 2], const uint32_t (&acc)[PW], const float* at) {
                const ulonglong2* b2 = reinterpret_cast<const ulonglong2*>(at);
                const ulonglong2* s2 = reinterpret_cast<const ulonglong2*>(at + 32);
#pragma unroll
                for (int e = 0; e < PW / 4; ++e) {
                    const ulonglong2 b = b2[e];
                    if constexpr (I8) {
                        const ulonglong2 sc = s2[e];
                        v[2 * e] = pair_fma(pair_mul(pair_of((float)(int)acc[4 * e], (float)(int)acc[4 * e + 1]), sc.x), x_scale2, b.x);
                        v[2 * e + 1] = pair_fma(pair_mul(pair_of((float)(int)acc[4 * e + 2], (float)(int)acc[4 * e + 3]), sc.y), x_scale2, b.y);
                    } else {
                        v[2 * e] = pair_add(pair_of(__uint_as_float(acc[4 * e]), __uint_as_float(acc[4 * e + 1])), b.x);
                        v[2 * e + 1] = pair_add(pair_of(__uint_as_float(acc[4 * e + 2]), __uint_as_float(acc[4 * e + 3])), b.y);
                    }
                }
            };
#pragma unroll 1
            for (int j = 0; j < C::PER_WARP && rows_inside; ++j) {
                const int c = piece(j);
                const int64_t col = n0 + c * PW;
                if (c * PW >= HC || col >= n_end) break;     // (uniform) nothing of this piece is inside
                const float* at = table + j * C::TABLES * 32;
                uint32_t a[PW];
                uint64_t o[PW / 2];
                take(c, 0, a);
                if constexpr (GATED) {
                    uint32_t b[PW];
                    take(c, 1, b);
                    tmem_ld_wait();
                    uint64_t u[PW / 2];
                    project(o, a, at);
                    project(u, b, at + 64);
                    if (p.p_save) {
                        emit(o, &tmG, p.p_by, (OUT*)p.p_save, p.ldp, col);
                        emit(u, &tmU, p.p_by, (OUT*)p.p_save + p.N, p.ldp, col);
                    }
                    with_act(p.act, [&](auto tag) {
#pragma unroll
                        for (int e = 0; e < PW / 2; ++e) o[e] = pair_gate<decltype(tag)::value, EXACT>(o[e], u[e]);
                    });
                } else {
                    tmem_ld_wait();
                    project(o, a, at);
                }
                emit(o, &tmO, p.out_by, (OUT*)p.out, p.ldo, col);
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if (CG == 2) mbar_arrive_remote(smem_u32(&out_empty[buf]), 0);
                else mbar_arrive(smem_u32(&out_empty[buf]));
            }
        }
        tma_store_wait_read<0>();                            // shared memory may go once the stores have read it
        __syncwarp();
        if (SPLIT && !ok) {          // gave up: the others of the cluster still meet this warp
            cluster_arrive();
            cluster_wait();
            cluster_arrive();
            cluster_wait();
        }
    }
    if (SPLIT && warp < 2) {         // the two meetings of the exchange
        __syncwarp();
        cluster_arrive();
        cluster_wait();
        cluster_arrive();
        cluster_wait();
    }

    tc_fence_before();
    if (CG == 2) {
        // neither block leaves (or frees tensor memory) while the other may still signal one of its barriers, read its shared memory
        // with an MMA or write its accumulators: every thread of the pair is past all of that when it arrives here
        cluster_arrive();
        cluster_wait();
    } else {
        __syncthreads();
    }
    if (warp == 1) {
        if (abort_flag) {            // give copies and MMAs still in flight time to land before freeing
            for (int i = 0; i < 256; ++i) __nanosleep(1000);
        }
        tc_fence_after();
        if (CG == 2) tmem_dealloc_pair(tmem_base, C::TMEM_COLS);
        else tmem_dealloc(tmem_base, C::TMEM_COLS);
    }
}

// What a stage of the ring takes where its layout goes by the call (ONE), and what the exchange of a split reduction takes in its place
template <bool GATED, int GK> struct OneLayout {
    int a_rows, own_pieces;
    uint32_t stage, tail, exchange;
    OneLayout(int64_t M, int hc, int split) {
        a_rows = M >= BM ? BM : (int)((M + 7) / 8 * 8);
        stage = GK * ((uint32_t)a_rows + (uint32_t)(GATED ? 2 * hc : hc)) * kRow;
        tail = (uint32_t)(BM - a_rows) * kRow;               // what the MMAs of the last stage read past its rows of X
        own_pieces = ((hc + 31) / 32 + split - 1) / split;
        exchange = split > 1 ? (uint32_t)(split * own_pieces * (GATED ? 2 : 1)) * (((uint32_t)a_rows + 31u) / 32u * 32u) * 128u : 0u;
    }
};

// hc: columns of the output in a tile (ONE); split: blocks that share its reduction (SPLIT)
template <bool I8, bool GATED, typename OUT, int BN, int CG, int GK, bool ONE, bool SPLIT = false>
lrd_status_t launch(const GluArgs& g, int hc, int split, cudaStream_t stream) {
    using C = Cfg<GATED, OUT, BN, CG, GK, ONE>;
    constexpr int out_type = sizeof(OUT) == 2 ? kTmaBf16 : kTmaF32, in_type = I8 ? kTmaU8 : kTmaBf16;
    constexpr int64_t vec = 16 / (int64_t)sizeof(OUT);
    if (!ONE) hc = C::HC;
    if (!SPLIT) split = 1;
    Params p;
    p.M = g.M; p.N = g.N;
    p.kb_total = (int)((g.K + (I8 ? 127 : 63)) / (I8 ? 128 : 64));
    p.m_tiles = (int)((g.M + BM * CG - 1) / (BM * CG));
    p.n_tiles = (int)((g.N + hc - 1) / hc);
    if ((int64_t)p.m_tiles * p.n_tiles > 0x7FFFFFFF - 2 * kNumSms) return LRD_ERR_TOO_LARGE;       // (over 10^13 elements)
    p.tiles = p.m_tiles * p.n_tiles;
    const int64_t row_bytes = (int64_t)p.kb_total * kRow;
    p.m_group = tile_group(p.m_tiles, p.n_tiles, kNumSms / CG, BM * CG * row_bytes, BN * row_bytes);
    uint32_t smem = C::SMEM_BYTES;
    p.hc = hc; p.a_rows = BM; p.stages = C::STAGES;
    p.split = split; p.kb_share = p.kb_total; p.own_pieces = 0;
    if (ONE) {
        const OneLayout<GATED, GK> o(g.M, hc, split);
        p.kb_share = ((p.kb_total + split - 1) / split + GK - 1) / GK * GK;
        if ((split - 1) * p.kb_share >= p.kb_total || o.exchange > C::RING_MAX) return LRD_ERR_UNSUPPORTED;      // (a block without a share)
        const uint32_t fit = (C::RING_MAX - o.tail) / o.stage;
        const uint32_t need = (uint32_t)((p.kb_share + GK - 1) / GK) * (uint32_t)((p.tiles * split + kNumSms - 1) / kNumSms);
        p.a_rows = o.a_rows;
        p.own_pieces = o.own_pieces;
        p.stages = (int)(fit < (uint32_t)kMaxStages ? fit : (uint32_t)kMaxStages);
        if (need < (uint32_t)p.stages) p.stages = (int)need;
        const uint32_t ring = (uint32_t)p.stages * o.stage + o.tail;
        smem = C::FIXED + (ring > o.exchange ? ring : o.exchange);
        // Blocks of a cluster wait for one another while they hold tensor memory, so no two such blocks may share an SM, of one launch or of
        // two: each could hold what the other's peer waits for.  With all of shared memory a block has its SM to itself.
        if (SPLIT) smem = kAllSmem;
    }
    p.bias = g.bias; p.x_scale = g.x_scale; p.w_scale = g.w_scale;
    p.out = g.out; p.ldo = g.ldo; p.p_save = g.p_save; p.ldp = g.ldp; p.act = g.act;
    p.timeout_flag = device_timeout_flag();
    // a result leaves by TMA where TMA can address its rows (and, of the two halves of P, both) and they end with a whole 16 bytes: it
    // writes those whole, past the last column too
    auto leave = [&](const void* base, int64_t ld) {
        return g.N % vec || ld % vec || ((uintptr_t)base & 15u) ? kByElements : ONE ? kByPieces : kByTma;
    };
    p.out_by = leave(g.out, g.ldo);
    p.p_by = g.p_save ? leave(g.p_save, g.ldp) : kByElements;
    CUtensorMap tA, tB, tO = {}, tG = {}, tU = {};
    const uint64_t rows_w = (uint64_t)(GATED ? 2 * g.N : g.N);
    const uint32_t kbox = I8 ? 128 : 64;
    bool ok = make_tmap_2d(&tA, in_type, g.X, (uint64_t)g.M, (uint64_t)g.K, (uint64_t)g.ldx, (uint32_t)p.a_rows, kbox);
    ok = ok && make_tmap_2d(&tB, in_type, g.W, rows_w, (uint64_t)g.K, (uint64_t)g.ldw, (uint32_t)(GATED || ONE ? hc : C::BNH), kbox);
    if (p.out_by == kByTma) ok = ok && make_tmap_2d(&tO, out_type, g.out, (uint64_t)g.M, (uint64_t)g.N, (uint64_t)g.ldo, 32, C::PW);
    if (p.p_by == kByTma) {
        ok = ok && make_tmap_2d(&tG, out_type, g.p_save, (uint64_t)g.M, (uint64_t)g.N, (uint64_t)g.ldp, 32, C::PW);
        ok = ok && make_tmap_2d(&tU, out_type, (const OUT*)g.p_save + g.N, (uint64_t)g.M, (uint64_t)g.N, (uint64_t)g.ldp, 32, C::PW);
    }
    if (!ok) return LRD_ERR_CUDA;
    auto kern = tc_glu_kernel<I8, GATED, OUT, BN, CG, GK, ONE, SPLIT>;
    static bool configured_on[kMaxDevices] = {};     // per instantiation; the attribute is sticky per function
    bool& configured = configured_on[device_slot()];
    if (!configured) {
        if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, ONE ? kAllSmem : C::SMEM_BYTES) != cudaSuccess) return LRD_ERR_CUDA;
        configured = true;
    }
    // every unit (block or pair) gets the same number of tiles (+-1)
    const int units_max = kNumSms / CG, waves = (p.tiles + units_max - 1) / units_max;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(SPLIT ? (unsigned)(p.tiles * split) : (unsigned)((p.tiles + waves - 1) / waves) * CG, 1, 1);
    cfg.blockDim = dim3(kThreads, 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;   // the kernel waits (griddepcontrol.wait)
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = SPLIT ? (unsigned)split : CG;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = CG == 2 || SPLIT ? 2 : 1;
    if (!cuda_ok(cudaLaunchKernelEx(&cfg, kern, tA, tB, tO, tG, tU, p), "cudaLaunchKernelEx(glu)")) return LRD_ERR_CUDA;
    count_launch();
    return LRD_OK;
}

// Tile shape beyond 128 rows: microseconds by what each shape's k-block and epilogue took where that bounded it (8192 x 4096 -> 4096 and
// 4093 x 1024 -> 2816 gated, both 8-bit to bf16); the epilogue of a tile runs beside the next tile's k-blocks.  One table for all operands: k-blocks are
// 128 bytes deep and four MMAs for either type; epilogues of fp32 results, which take longer, were not fitted.
struct Shape { int bn, cg; double k_block, epilogue, us; };
// bn = 0: no shape takes the form asked for by the test hook (columns and blocks per MMA of GluForm; 0: any)
inline Shape pick_shape(const GluArgs& g, int k_elems) {
    static const Shape cands[] = {{256, 2, 0.37, 4.3, 0}, {128, 2, 0.23, 3.0, 0}, {256, 1, 0.45, 4.0, 0}, {128, 1, 0.27, 2.4, 0}, {64, 1, 0.20, 1.7, 0}};
    const GluForm form = glu_form();
    Shape best = {0, 1, 0, 0, 1e300};
    const int64_t kb = (g.K + k_elems - 1) / k_elems;
    for (const Shape& c : cands) {
        if ((form.columns && c.bn != form.columns) || (form.blocks && c.cg != form.blocks)) continue;
        const int hc = g.gated ? c.bn / 2 : c.bn;
        const int64_t units = kNumSms / c.cg, tiles = ((g.M + BM * c.cg - 1) / (BM * c.cg)) * ((g.N + hc - 1) / hc), waves = (tiles + units - 1) / units;
        const double main = (double)kb * c.k_block, us = main + (double)(waves - 1) * (main > c.epilogue ? main : c.epilogue) + c.epilogue;
        if (us < best.us) { best = c; best.us = us; }
    }
    return best;
}
// Columns of the output in a tile (any multiple of 16) and blocks that share its reduction, for up to 128 rows, or, split, for a few tiles of
// more: microseconds of the rounds that all SMs make over the tiles.  A k-block costs its issue and its bytes at 120 GB/s a block; an exchange
// costs two meetings of the cluster and, with many rows, what crosses.  So columns are dealt out evenly over the SMs (16 x 4096 ->
// 2 x 10752 in 8 bits: 17.6 us in 135 tiles of 80, 19.7 of 64, 19.0 of 128), and a reduction is shared where the tiles leave SMs idle (16 x 4096
// -> 1024 in 8 bits: 6.8 us unsplit, 5.2 by four; 16 x 4096 -> 2 x 1024 in bf16 12.4 and 9.5; 512 x 8192 -> 1024 15.7 and 11.8).
struct OneShape { int hc, split; double us; };
inline OneShape pick_one(const GluArgs& g, int k_elems) {
    const int64_t kb = (g.K + k_elems - 1) / k_elems, m_tiles = (g.M + BM - 1) / BM;
    const int rows = g.M >= BM ? BM : (int)((g.M + 7) / 8 * 8), most = g.gated ? 128 : 256;
    OneShape best = {0, 1, 1e300};
    // A reduction is shared only where narrow tiles (32 accumulator columns, 64 beyond 128 rows) leave a third or a fifth of the SMs idle.  The
    // fastest shared form against the fastest unshared one, over 522 calls of 16 to 512 rows, 1024 to 8192 deep: up to 128 rows it is the
    // faster in 124 of 243 calls below the limit and in 60 of 135 above it, where what it saves is larger only for long reductions (16 x 8192
    // -> 2 x 1600 in bf16 12.8 us by four, 21.2 unshared; 128 x 4096 -> 2 x 1760 in 8 bits 9.2 / 7.6); beyond 128 rows in 44 of 111 and
    // in 3 of 33.  The forms chosen take 2.8 % longer on average than the fastest ones measured.
    const int64_t narrow = (g.M <= BM ? 32 : 64) / (g.gated ? 2 : 1);
    const int most_split = m_tiles * ((g.N + narrow - 1) / narrow) >= (g.M <= BM ? 100 : 120) ? 1 : g.M <= BM ? 4 : 2;
    for (int hc = 16; hc <= most; hc += 16) {
        const int bn = g.gated ? 2 * hc : hc;
        const int64_t tiles = m_tiles * ((g.N + hc - 1) / hc), group = bn <= 96 ? 2 : 1;
        const double k_block = (bn <= 96 ? 0.025 : 0.04) + (rows + bn) * (double)kRow * 8.3e-6, epilogue = 0.3 + 0.004 * bn;
        for (int split = g.M > BM ? 2 : 1; split <= most_split; split *= 2) {
            const int64_t share = ((kb + split - 1) / split + group - 1) / group * group, rounds = (tiles + kNumSms - 1) / kNumSms;
            // (not all SMs are in clusters of four at one time: 37 of them, 148 blocks, ran in two rounds)
            if (split > 1 && (tiles * split > (split == 2 ? kNumSms : 128) || (split - 1) * share >= kb)) continue;
            const double us = 2.7 + (double)rounds * ((double)share * k_block + epilogue) + (split > 1 ? 0.6 + 0.016 * rows * (split > 2 ? 1.5 : 1.0) : 0.0);
            if (us < best.us) best = {hc, split, us};
        }
    }
    return best;
}

template <bool I8, bool GATED, typename OUT> lrd_status_t launch_one(const GluArgs& g, int hc, int split, cudaStream_t s) {
    // two k-blocks a stage where a tile's rows are few
    if ((GATED ? 2 * hc : hc) <= 96)
        return split > 1 ? launch<I8, GATED, OUT, 256, 1, 2, true, true>(g, hc, split, s) : launch<I8, GATED, OUT, 256, 1, 2, true>(g, hc, 1, s);
    return split > 1 ? launch<I8, GATED, OUT, 256, 1, 1, true, true>(g, hc, split, s) : launch<I8, GATED, OUT, 256, 1, 1, true>(g, hc, 1, s);
}

template <bool I8, bool GATED, typename OUT> lrd_status_t launch_shape(const GluArgs& g, cudaStream_t s) {
    const GluForm form = glu_form();
    const int columns = GATED ? form.columns / 2 : form.columns;
    if (form.split > 1 || g.M <= BM) {
        if (form.blocks == 2) return LRD_ERR_UNSUPPORTED;
        if (form.columns) return launch_one<I8, GATED, OUT>(g, columns, form.split > 1 ? form.split : 1, s);
    }
    const bool any = form.columns == 0 && form.blocks == 0;
    const OneShape one = any || g.M <= BM ? pick_one(g, I8 ? 128 : 64) : OneShape{0, 1, 1e300};
    if (g.M <= BM) return launch_one<I8, GATED, OUT>(g, one.hc, one.split, s);
    const Shape c = pick_shape(g, I8 ? 128 : 64);
    // (2.3: pick_one counts a launch and a call's first loads, some 2.7 us, pick_shape does not.  Over 144 calls of 300 and 512 rows the choice
    // between the two takes 0.2 % longer on average than the faster one, 19 % at worst.)
    if (any && one.hc && one.us < c.us + 2.3) return launch_one<I8, GATED, OUT>(g, one.hc, one.split, s);
    if (c.bn == 0) return LRD_ERR_UNSUPPORTED;
    if (c.cg == 2) return c.bn == 256 ? launch<I8, GATED, OUT, 256, 2, 1, false>(g, 0, 1, s) : launch<I8, GATED, OUT, 128, 2, 1, false>(g, 0, 1, s);
    if (c.bn == 256) return launch<I8, GATED, OUT, 256, 1, 1, false>(g, 0, 1, s);
    return c.bn == 128 ? launch<I8, GATED, OUT, 128, 1, 1, false>(g, 0, 1, s) : launch<I8, GATED, OUT, 64, 1, 2, false>(g, 0, 1, s);
}

}  // namespace glu
}  // namespace lrd
