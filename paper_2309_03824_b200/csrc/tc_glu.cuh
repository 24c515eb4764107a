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
// conversion.
//
// One block per SM walks over the tiles (tile t -> row tile t % m_tiles, so that blocks working at the same time share W in L2);
// accumulators are double-buffered in tensor memory and the epilogue of a tile overlaps the MMAs of the next.
// AR: rows of X a stage holds.  With 32 rows or fewer (AR = 32) a stage takes a quarter of the shared memory, and the rest holds more of
// W in flight, which is all such a call moves; the MMAs still read 128 rows -- what stands behind the 32 in shared memory, within
// the block's own -- and the rows past M are never looked at (a row of the product depends on its own row of X alone).
//
// Warp 0: TMA producer.  Warp 1: tensor memory + MMA issue.  Warps 2-9: epilogue.  Every wait is bounded.
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
constexpr int kThreads = 320;
constexpr uint32_t kTableBytes = 1024;                       // one epilogue warp's per-column values of a tile

template <bool GATED, typename OUT, int BN, int CG, int AR> struct Cfg {
    static_assert(AR == BM || (AR == 32 && CG == 1), "rows of X in a stage");
    static constexpr int BNH = BN / CG;                      // rows of W this block loads
    static constexpr int HC = GATED ? BN / 2 : BN;           // columns of the output in a tile
    static constexpr int PW = HC < 32 ? HC : 32;             // an epilogue step: 32 rows x PW columns of the output
    static constexpr int PIECES = HC / PW, PER_WARP = (PIECES + 1) / 2;
    static constexpr int TABLES = GATED ? 4 : 2;             // bias and scale of each column
    static_assert(PER_WARP * TABLES * 32 * 4 <= (int)kTableBytes, "per-column values");
    static constexpr int G = CG == 1 && (BN <= 64 || AR == 32) ? 2 : 1;    // k-blocks per stage: the issue loop's cost is per stage
    static constexpr uint32_t A_TILE = AR * kRow, B_TILE = BNH * kRow;
    static constexpr uint32_t STAGE_BYTES = G * (A_TILE + B_TILE);
    static constexpr uint32_t SLAB_BYTES = 32 * PW * sizeof(OUT);
    static constexpr uint32_t STAGING = 8 * 2 * SLAB_BYTES;
    static constexpr uint32_t TAIL = (BM - AR) * kRow;       // what the MMAs of the last stage read past its rows of X
    static constexpr uint32_t RING_MAX = 232448 - 1024 - 2048 - STAGING - 8 * kTableBytes - TAIL;       // 2048: static shared memory
    static constexpr int STAGES_RAW = RING_MAX / STAGE_BYTES;
    static constexpr int STAGES = STAGES_RAW > 12 ? 12 : STAGES_RAW;
    static_assert(STAGES >= 3, "ring");
    static constexpr uint32_t SMEM_BYTES = STAGING + STAGES * STAGE_BYTES + TAIL + 8 * kTableBytes + 1024;
    static constexpr uint32_t TMEM_COLS = 2 * BN <= 64 ? 64 : 2 * BN <= 128 ? 128 : 2 * BN <= 256 ? 256 : 512;
    static constexpr uint32_t BUF_COLS = TMEM_COLS / 2;
};

struct Params {
    int64_t M, N;
    int kb_total, m_tiles;
    int64_t tiles;
    const void* bias;
    const float *x_scale, *w_scale;
    void* out; int64_t ldo;
    void* p_save; int64_t ldp;
    int out_tma, p_tma;       // these leave by TMA; else by ordinary stores
    int act;
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

template <int PW> __device__ __forceinline__ void tmem_piece(uint32_t at, uint32_t (&v)[PW]) {
    if constexpr (PW == 32) tmem_ld_32x32(at, v);
    else tmem_ld_32x16(at, v);
}
template <typename OUT> __device__ __forceinline__ float out_to_f32(OUT x) { return (float)x; }

// A warp's 32 x PW values (lane = row) -> its slab, in the layout of a swizzled TMA box of that width
template <typename OUT, int PW> __device__ __forceinline__ uint32_t slab_xor(uint32_t row) {
    constexpr uint32_t bytes = PW * sizeof(OUT);
    return bytes == 128 ? row & 7u : bytes == 64 ? (row >> 1) & 3u : (row >> 2) & 1u;
}
template <typename OUT, int PW> __device__ __forceinline__ void put_slab(uint32_t slab, const float (&v)[PW]) {
    const uint32_t lane = threadIdx.x & 31u, at = slab + lane * (PW * sizeof(OUT)), x = slab_xor<OUT, PW>(lane);
    if constexpr (sizeof(OUT) == 2) {
#pragma unroll
        for (uint32_t c = 0; c < PW / 8; ++c)
            st_shared_v4(at + ((c ^ x) << 4), pack_bf16(v[8 * c], v[8 * c + 1]), pack_bf16(v[8 * c + 2], v[8 * c + 3]), pack_bf16(v[8 * c + 4], v[8 * c + 5]),
                         pack_bf16(v[8 * c + 6], v[8 * c + 7]));
    } else {
#pragma unroll
        for (uint32_t c = 0; c < PW / 4; ++c)
            st_shared_v4(at + ((c ^ x) << 4), __float_as_uint(v[4 * c]), __float_as_uint(v[4 * c + 1]), __float_as_uint(v[4 * c + 2]), __float_as_uint(v[4 * c + 3]));
    }
}
// The slab's rows and columns that exist, to rows of any stride and alignment: a lane a column
template <typename OUT, int PW> __device__ __forceinline__ void store_slab(uint32_t slab, OUT* dst, int64_t ld, int64_t rows, int64_t cols) {
    constexpr uint32_t STEP = 32 / PW;                       // rows an instruction covers
    const uint32_t lane = threadIdx.x & 31u, c = lane % PW, r0 = lane / PW, byte = c * sizeof(OUT);
#pragma unroll 8
    for (uint32_t r = r0; r < 32; r += STEP) {
        const uint32_t at = slab + r * (PW * sizeof(OUT)) + (((byte >> 4) ^ slab_xor<OUT, PW>(r)) << 4) + (byte & 15u);
        if constexpr (sizeof(OUT) == 2) {
            uint16_t v;
            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(at));
            if (r < rows && c < cols) dst[r * ld + c] = __ushort_as_bfloat16(v);
        } else {
            float v;
            asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(at));
            if (r < rows && c < cols) dst[r * ld + c] = v;
        }
    }
}

template <bool I8, bool GATED, typename OUT, int BN, int CG, int AR>
__global__ void __launch_bounds__(kThreads, 1)
tc_glu_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const __grid_constant__ CUtensorMap tmO,
              const __grid_constant__ CUtensorMap tmG, const __grid_constant__ CUtensorMap tmU, const Params p) {
    using C = Cfg<GATED, OUT, BN, CG, AR>;
    constexpr int STAGES = C::STAGES, G = C::G, HC = C::HC, PW = C::PW;
    constexpr bool EXACT = sizeof(OUT) == 4;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t full_bar[STAGES], empty_bar[STAGES], out_full[2], out_empty[2];
    __shared__ uint32_t tmem_base_slot;
    __shared__ int abort_flag;

    const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t staging_base = smem_base, ring_base = smem_base + C::STAGING;
    float* const tables = reinterpret_cast<float*>(smem_raw + (smem_base - smem_u32(smem_raw)) + C::STAGING + STAGES * C::STAGE_BYTES + C::TAIL);
    const AbortCtx ab{&abort_flag, p.timeout_flag};
    const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x / 32, 0), lane = threadIdx.x % 32;
    const int h = CG == 2 ? (int)cluster_ctarank() : 0;      // this block's half of the pair
    const int64_t unit = (int64_t)(blockIdx.x / CG), n_units = (int64_t)(gridDim.x / CG);

    if (threadIdx.x == 0) {
        abort_flag = 0;
        prefetch_tmap(&tmA);
        prefetch_tmap(&tmB);
        if (p.out_tma) prefetch_tmap(&tmO);
        if (GATED && p.p_tma) {
            prefetch_tmap(&tmG);
            prefetch_tmap(&tmU);
        }
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(smem_u32(&full_bar[s]), 1);
            mbar_init(smem_u32(&empty_bar[s]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&out_full[i]), 1);
            mbar_init(smem_u32(&out_empty[i]), 8 * CG);      // the epilogue warps of every block of the pair
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
        for (int64_t t = unit; t < p.tiles && ok; t += n_units) {
            const int m0 = (int)(t % p.m_tiles) * (BM * CG) + h * BM, n0 = (int)(t / p.m_tiles) * HC;
            for (int kb = 0; kb < p.kb_total; kb += G) {     // k-blocks past the last read as zeros
                ok = mbar_wait_uniform(smem_u32(&empty_bar[s]), ph, ab);
                if (!ok) break;
                const uint32_t fb = CG == 2 ? map_to_cta(smem_u32(&full_bar[s]), 0) : smem_u32(&full_bar[s]);
                const uint32_t a_dst = ring_base + s * C::STAGE_BYTES, b_dst = a_dst + G * C::A_TILE;
                if (elect_one()) {
                    if (h == 0) mbar_expect_tx(smem_u32(&full_bar[s]), CG * C::STAGE_BYTES);
#pragma unroll
                    for (int g = 0; g < G; ++g) {
                        load(a_dst + g * C::A_TILE, &tmA, fb, (kb + g) * KE, m0);
                        const uint32_t b = b_dst + g * C::B_TILE;
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
        constexpr uint32_t idesc = I8 ? idesc_i8(BN, CG) : CG == 2 ? idesc_bf16_pair(BN, false, false) : idesc_bf16(BN, false, false);
        const uint64_t a_desc0 = smem_desc_sw128(ring_base, 0, 1024), b_desc0 = smem_desc_sw128(ring_base + G * C::A_TILE, 0, 1024);
        int s = 0, i = 0;
        uint32_t ph = 0;
        bool ok = true;
        for (int64_t t = unit; t < p.tiles && ok; t += n_units, ++i) {
            const int buf = i & 1;
            const uint32_t d_tmem = tmem_base + (uint32_t)buf * C::BUF_COLS;
            ok = mbar_wait_uniform(smem_u32(&out_empty[buf]), ((i >> 1) & 1) ^ 1, ab);      // accumulator buffer drained
            tc_fence_after();
            uint32_t ready = mbar_test_wait(smem_u32(&full_bar[s]), ph);
            for (int kb = 0; kb < p.kb_total && ok; kb += G) {
                ok = mbar_wait_peeked(ready, smem_u32(&full_bar[s]), ph, ab);
                if (!ok) break;
                tc_fence_after();
                const uint64_t ad = a_desc0 + (uint32_t)s * (C::STAGE_BYTES >> 4), bd = b_desc0 + (uint32_t)s * (C::STAGE_BYTES >> 4);
                const uint32_t eb = smem_u32(&empty_bar[s]);
                const bool last = kb + G >= p.kb_total;
                if (++s == STAGES) { s = 0; ph ^= 1; }
                ready = last ? 0u : mbar_test_wait(smem_u32(&full_bar[s]), ph);
                if (elect_one()) {
#pragma unroll
                    for (int g = 0; g < G; ++g) {
                        if (g > 0 && kb + g >= p.kb_total) break;
#pragma unroll
                        for (int kk = 0; kk < 4; ++kk) {     // 32 bytes of K each
                            const uint64_t a = ad + (g * (C::A_TILE >> 4) + kk * 2u), b = bd + (g * (C::B_TILE >> 4) + kk * 2u);
                            const uint32_t acc = g > 0 || kk > 0 ? 1u : (kb > 0 ? 1u : 0u);
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
        const int hw = (warp - 2) / 4;                       // two warps share a quarter: they take alternate pieces
        const uint32_t lane_addr = tmem_base + ((uint32_t)(q * 32) << 16);
        const uint32_t slab0 = staging_base + (uint32_t)(warp - 2) * 2u * C::SLAB_BYTES;
        float* const table = tables + (warp - 2) * (kTableBytes / 4);
        const OUT* const bias = (const OUT*)p.bias;
        int i = 0, sb = 0;
        bool ok = true;
        for (int64_t t = unit; t < p.tiles && ok; t += n_units, ++i) {
            const int buf = i & 1;
            const int64_t m0 = (t % p.m_tiles) * (BM * CG) + h * BM + q * 32, n0 = (t / p.m_tiles) * HC;
            const bool rows_inside = m0 < p.M;               // (uniform) a tile may hang over the last row
            // bias and scale of this warp's columns, into a table of its own while the MMAs run
            if (rows_inside) {
                __syncwarp();
#pragma unroll
                for (int j = 0; j < C::PER_WARP; ++j) {
                    const int64_t col = n0 + (hw + 2 * j) * PW + lane;
                    const bool in = lane < PW && col < p.N;
                    float* at = table + j * C::TABLES * 32 + lane;
                    at[0] = bias && in ? out_to_f32(bias[col]) : 0.0f;
                    if (I8) at[32] = in ? p.w_scale[col] : 0.0f;
                    if (GATED) {
                        at[64] = bias && in ? out_to_f32(bias[p.N + col]) : 0.0f;
                        if (I8) at[96] = in ? p.w_scale[p.N + col] : 0.0f;
                    }
                }
                __syncwarp();
            }
            const float x_scale = I8 && m0 + lane < p.M ? p.x_scale[m0 + lane] : 0.0f;
            ok = mbar_wait_uniform(smem_u32(&out_full[buf]), (i >> 1) & 1, ab);
            if (!ok) break;
            tc_fence_after();
            const uint32_t d_tmem = lane_addr + (uint32_t)buf * C::BUF_COLS;
            // 32 x PW values out: slab, then TMA or the rows themselves.  Two slabs a warp: before one is written again, the store
            // that last read it (two groups ago) has.
            auto emit = [&](const float (&v)[PW], const CUtensorMap* m, bool tma, OUT* base, int64_t ld, int64_t col) {
                const uint32_t slab = slab0 + (uint32_t)(sb & 1) * C::SLAB_BYTES;
                if (sb >= 2) tma_store_wait_read<1>();
                ++sb;
                __syncwarp();
                put_slab<OUT, PW>(slab, v);
                if (tma) fence_proxy_async_smem();
                __syncwarp();
                if (!tma) store_slab<OUT, PW>(slab, base + m0 * ld + col, ld, p.M - m0, p.N - col);
                if (elect_one()) {                           // (a group each time, an empty one behind ordinary stores)
                    if (tma) tma_store_2d(m, slab, (int)col, (int)m0);
                    tma_store_commit();
                }
                __syncwarp();
            };
            auto value = [&](uint32_t acc, const float* at, int c) {     // accumulator -> the projection
                return I8 ? fmaf((float)(int)acc * x_scale, at[32 + c], at[c]) : __uint_as_float(acc) + at[c];
            };
#pragma unroll 1
            for (int j = 0; j < C::PER_WARP && rows_inside; ++j) {
                const int c = hw + 2 * j;
                const int64_t col = n0 + c * PW;
                if (c >= C::PIECES || col >= p.N) break;     // (uniform) nothing of this piece is inside
                const float* at = table + j * C::TABLES * 32;
                uint32_t a[PW];
                float o[PW];
                tmem_piece<PW>(d_tmem + c * PW, a);
                if constexpr (GATED) {
                    uint32_t b[PW];
                    tmem_piece<PW>(d_tmem + HC + c * PW, b);
                    tmem_ld_wait();
                    float g[PW], u[PW];
#pragma unroll
                    for (int e = 0; e < PW; ++e) {
                        g[e] = value(a[e], at, e);
                        u[e] = value(b[e], at + 64, e);
                    }
                    with_act(p.act, [&](auto tag) {
#pragma unroll
                        for (int e = 0; e < PW; ++e) o[e] = act_value<decltype(tag)::value, EXACT>(g[e]) * u[e];
                    });
                    if (p.p_save) {
                        emit(g, &tmG, p.p_tma, (OUT*)p.p_save, p.ldp, col);
                        emit(u, &tmU, p.p_tma, (OUT*)p.p_save + p.N, p.ldp, col);
                    }
                } else {
                    tmem_ld_wait();
#pragma unroll
                    for (int e = 0; e < PW; ++e) o[e] = value(a[e], at, e);
                }
                emit(o, &tmO, p.out_tma, (OUT*)p.out, p.ldo, col);
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

template <bool I8, bool GATED, typename OUT, int BN, int CG, int AR>
lrd_status_t launch(const GluArgs& g, cudaStream_t stream) {
    using C = Cfg<GATED, OUT, BN, CG, AR>;
    constexpr int out_type = sizeof(OUT) == 2 ? kTmaBf16 : kTmaF32, in_type = I8 ? kTmaU8 : kTmaBf16;
    constexpr int64_t vec = 16 / (int64_t)sizeof(OUT);
    Params p;
    p.M = g.M; p.N = g.N;
    p.kb_total = (int)((g.K + (I8 ? 127 : 63)) / (I8 ? 128 : 64));
    p.m_tiles = (int)((g.M + BM * CG - 1) / (BM * CG));
    p.tiles = (int64_t)p.m_tiles * ((g.N + C::HC - 1) / C::HC);
    p.bias = g.bias; p.x_scale = g.x_scale; p.w_scale = g.w_scale;
    p.out = g.out; p.ldo = g.ldo; p.p_save = g.p_save; p.ldp = g.ldp; p.act = g.act;
    p.timeout_flag = device_timeout_flag();
    // a result leaves by TMA where TMA can address its rows (and, of the two halves of P, both) and they end with a whole 16 bytes: it
    // writes those whole, past the last column too
    auto tma_rows = [&](const void* base, int64_t ld) { return C::PW == 32 && g.N % vec == 0 && ld % vec == 0 && ((uintptr_t)base & 15u) == 0; };
    p.out_tma = tma_rows(g.out, g.ldo);
    p.p_tma = g.p_save && tma_rows(g.p_save, g.ldp);
    CUtensorMap tA, tB, tO = {}, tG = {}, tU = {};
    const uint64_t rows_w = (uint64_t)(GATED ? 2 * g.N : g.N);
    const uint32_t kbox = I8 ? 128 : 64;
    bool ok = make_tmap_2d(&tA, in_type, g.X, (uint64_t)g.M, (uint64_t)g.K, (uint64_t)g.ldx, AR, kbox);
    ok = ok && make_tmap_2d(&tB, in_type, g.W, rows_w, (uint64_t)g.K, (uint64_t)g.ldw, GATED ? C::HC : C::BNH, kbox);
    if (p.out_tma) ok = ok && make_tmap_2d(&tO, out_type, g.out, (uint64_t)g.M, (uint64_t)g.N, (uint64_t)g.ldo, 32, C::PW);
    if (p.p_tma) {
        ok = ok && make_tmap_2d(&tG, out_type, g.p_save, (uint64_t)g.M, (uint64_t)g.N, (uint64_t)g.ldp, 32, C::PW);
        ok = ok && make_tmap_2d(&tU, out_type, (const OUT*)g.p_save + g.N, (uint64_t)g.M, (uint64_t)g.N, (uint64_t)g.ldp, 32, C::PW);
    }
    if (!ok) return LRD_ERR_CUDA;
    auto kern = tc_glu_kernel<I8, GATED, OUT, BN, CG, AR>;
    static bool configured_on[kMaxDevices] = {};     // per instantiation; the attribute is sticky per function
    bool& configured = configured_on[device_slot()];
    if (!configured) {
        if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM_BYTES) != cudaSuccess) return LRD_ERR_CUDA;
        configured = true;
    }
    // every unit (block or pair) gets the same number of tiles (+-1)
    const int64_t units_max = kNumSms / CG, waves = (p.tiles + units_max - 1) / units_max;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((p.tiles + waves - 1) / waves) * CG, 1, 1);
    cfg.blockDim = dim3(kThreads, 1, 1);
    cfg.dynamicSmemBytes = C::SMEM_BYTES;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;   // the kernel waits (griddepcontrol.wait)
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = CG;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = CG == 2 ? 2 : 1;
    if (!cuda_ok(cudaLaunchKernelEx(&cfg, kern, tA, tB, tO, tG, tU, p), "cudaLaunchKernelEx(glu)")) return LRD_ERR_CUDA;
    count_launch();
    return LRD_OK;
}

// Tile shape: estimated microseconds as of the persistent product (tc_gemm_persistent_estimate): the k-blocks of a tile at the issue
// loop's, the tensor pipe's or the loads' pace, whichever is slowest, the epilogue of a tile beside the next tile's k-blocks.
struct Shape { int bn, cg, ar; };
// bn = 0: no shape takes the form asked for by the test hook (columns and blocks per MMA of GluForm; 0: any)
inline Shape pick_shape(const GluArgs& g, int k_elems) {
    const GluForm form = glu_form();
    static const Shape cands[] = {{256, 2, 128}, {128, 2, 128}, {256, 1, 128}, {128, 1, 128}, {64, 1, 128}, {128, 1, 32}, {64, 1, 32}, {32, 1, 32}};
    Shape best = {0, 1, 128};
    double best_us = 1e300;
    const int64_t kb = (g.K + k_elems - 1) / k_elems;
    for (const Shape& c : cands) {
        if ((c.ar == 32) != (g.M <= 32)) continue;
        if (c.cg == 2 && g.M <= BM) continue;
        if ((form.columns && c.bn != form.columns) || (form.blocks && c.cg != form.blocks)) continue;
        const int hc = g.gated ? c.bn / 2 : c.bn;
        const int64_t units = kNumSms / c.cg, tiles = ((g.M + BM * c.cg - 1) / (BM * c.cg)) * ((g.N + hc - 1) / hc), waves = (tiles + units - 1) / units;
        const double mma = 4.0 * (c.bn / 2.0 > 32 + c.bn / 4.0 ? c.bn / 2.0 : 32 + c.bn / 4.0) / 1965.0;
        const double load = (double)(c.ar + c.bn / c.cg) * kRow * 6.6e-6, issue = c.cg == 1 && (c.bn <= 64 || c.ar == 32) ? 0.16 : 0.19;
        const double main = (double)kb * (mma > load ? (mma > issue ? mma : issue) : (load > issue ? load : issue)), epilogue = 0.0195 * c.bn;
        const double us = main + (double)(waves - 1) * (main > epilogue ? main : epilogue) + epilogue;
        if (us < best_us) { best_us = us; best = c; }
    }
    return best;
}

template <bool I8, bool GATED, typename OUT> lrd_status_t launch_shape(const GluArgs& g, cudaStream_t s) {
    const Shape c = pick_shape(g, I8 ? 128 : 64);
    if (c.bn == 0) return LRD_ERR_UNSUPPORTED;
    if (c.cg == 2) return c.bn == 256 ? launch<I8, GATED, OUT, 256, 2, 128>(g, s) : launch<I8, GATED, OUT, 128, 2, 128>(g, s);
    if (c.ar == 32) {
        if (c.bn == 128) return launch<I8, GATED, OUT, 128, 1, 32>(g, s);
        return c.bn == 64 ? launch<I8, GATED, OUT, 64, 1, 32>(g, s) : launch<I8, GATED, OUT, 32, 1, 32>(g, s);
    }
    if (c.bn == 256) return launch<I8, GATED, OUT, 256, 1, 128>(g, s);
    return c.bn == 128 ? launch<I8, GATED, OUT, 128, 1, 128>(g, s) : launch<I8, GATED, OUT, 64, 1, 128>(g, s);
}

}  // namespace glu
}  // namespace lrd
