// Both products of a layer's backward pass in one launch (sm_100a):  dX[M x K] = D W  and  dW[N x K] = D^T X,  from D[M x N], W[N x K] and
// X[M x K].  Neither reads what the other writes, and their tiles take different times: one walk of all pairs of SMs over the tiles of
// both, the longer ones first, wastes one unfinished round where two launches waste two, and a launch boundary less.
//
// The walk is the persistent product's (tc_gemm_persistent.cu) on pairs of SMs, 256 rows a tile: TMA producer, MMA issuer, eight epilogue
// warps, accumulators double-buffered.  B is MN-major in both (W and X as they lie); A is D, K-major for dX and MN-major for dW.  What
// differs from tile to tile -- maps, majorness, columns (256, 192 or 128) -- is looked up by which product the tile belongs to.
#include <algorithm>

#include "common.cuh"
#include "ptx_pair.cuh"
#include "tc.cuh"
#include "tma.cuh"

namespace lrd {
namespace {

using namespace ptx;

constexpr int BM = 128, BK = 64, kThreads = 320, kStages = 6;
constexpr uint32_t kTile = BM * BK * 2;                      // A's, and most of B's: 16 KB
constexpr uint32_t kStageBytes = 2 * kTile, kSlabBytes = 32 * 32 * 2, kStagingBytes = 8 * 2 * kSlabBytes;
constexpr uint32_t kSmemBytes = kStages * kStageBytes + kStagingBytes + 1024;

struct Product {
    int64_t M, N;
    int kb_total, m_tiles, n_tiles, m_group, tiles;
    int bn, a_mn;             // columns of a tile; A stored [K x M] (else [M x K])
};
struct Products {
    Product p[2];
    unsigned int* timeout_flag;
};

__global__ void __launch_bounds__(kThreads, 1)
two_products_kernel(const __grid_constant__ CUtensorMap tA0, const __grid_constant__ CUtensorMap tB0, const __grid_constant__ CUtensorMap tC0,
                    const __grid_constant__ CUtensorMap tA1, const __grid_constant__ CUtensorMap tB1, const __grid_constant__ CUtensorMap tC1,
                    const __grid_constant__ Products ps) {
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t full_bar[kStages], empty_bar[kStages], out_full[2], out_empty[2];
    __shared__ uint32_t tmem_base_slot;
    __shared__ int abort_flag;

    const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t staging_base = smem_base, ring_base = smem_base + kStagingBytes;
    const AbortCtx ab{&abort_flag, ps.timeout_flag};
    const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x / 32, 0), lane = threadIdx.x % 32;
    const int h = (int)cluster_ctarank();                    // this block's half of the pair
    const int unit = (int)blockIdx.x / 2, n_units = (int)gridDim.x / 2, total = ps.p[0].tiles + ps.p[1].tiles;

    if (threadIdx.x == 0) {
        abort_flag = 0;
        prefetch_tmap(&tA0);
        prefetch_tmap(&tB0);
        prefetch_tmap(&tC0);
        prefetch_tmap(&tA1);
        prefetch_tmap(&tB1);
        prefetch_tmap(&tC1);
        for (int s = 0; s < kStages; ++s) {
            mbar_init(smem_u32(&full_bar[s]), 1);
            mbar_init(smem_u32(&empty_bar[s]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&out_full[i]), 1);
            mbar_init(smem_u32(&out_empty[i]), 16);          // the epilogue warps of both blocks
        }
        fence_mbar_init();
    }
    if (warp == 1) {
        tmem_alloc_pair(smem_u32(&tmem_base_slot), 512);
        tmem_relinquish_pair();
    }
    tc_fence_before();
    cluster_arrive();                // the other block's barriers exist before anything signals them
    cluster_wait();
    tc_fence_after();
    const uint32_t tmem_base = tmem_base_slot;
    griddep_wait();                  // what stands above touched only this block's own shared and tensor memory
    if (warp != 0) griddep_launch_dependents();

    if (warp == 0) {
        // ------------------------------------------------------------------ TMA producer
        int s = 0;
        uint32_t ph = 1;
        bool ok = true;
        for (int t = unit; t < total && ok; t += n_units) {
            const bool second = t >= ps.p[0].tiles;
            const Product& p = ps.p[second];
            const CUtensorMap *mA = second ? &tA1 : &tA0, *mB = second ? &tB1 : &tB0;
            int mt, nt;
            tile_at(second ? t - ps.p[0].tiles : t, p.m_tiles, p.n_tiles, p.m_group, mt, nt);
            const int m0 = mt * 256 + h * BM, half = p.bn / 2, n0 = nt * p.bn + h * half, boxes = (half + 63) / 64;      // (the last box may be loaded past the half)
            for (int kb = 0; kb < p.kb_total; ++kb) {
                ok = mbar_wait_uniform(smem_u32(&empty_bar[s]), ph, ab);
                if (!ok) break;
                const uint32_t fb = map_to_cta(smem_u32(&full_bar[s]), 0), a_dst = ring_base + s * kStageBytes, b_dst = a_dst + kTile;
                if (elect_one()) {
                    if (h == 0) mbar_expect_tx(smem_u32(&full_bar[s]), 2 * (kTile + boxes * 8192));
                    if (p.a_mn) {
                        tma_load_2d_pair(a_dst, mA, fb, m0, kb * BK);
                        tma_load_2d_pair(a_dst + 8192, mA, fb, m0 + 64, kb * BK);
                    } else {
                        tma_load_2d_pair(a_dst, mA, fb, kb * BK, m0);
                    }
                    tma_load_2d_pair(b_dst, mB, fb, n0, kb * BK);
                    if (boxes == 2) tma_load_2d_pair(b_dst + 8192, mB, fb, n0 + 64, kb * BK);
                }
                __syncwarp();
                if (++s == kStages) { s = 0; ph ^= 1; }
            }
        }
    } else if (warp == 1 && h == 0) {
        // ------------------------------------------------------------------ MMA issuer (the even block of a pair)
        const uint64_t a_mn0 = smem_desc_sw128(ring_base, 8192, 1024), a_k0 = smem_desc_sw128(ring_base, 0, 1024);
        const uint64_t b_desc0 = smem_desc_sw128(ring_base + kTile, 8192, 1024);
        int s = 0, i = 0;
        uint32_t ph = 0;
        bool ok = true;
        for (int t = unit; t < total && ok; t += n_units, ++i) {
            const Product& p = ps.p[t >= ps.p[0].tiles];
            const int buf = i & 1, kb_total = p.kb_total;
            const uint32_t d_tmem = tmem_base + (uint32_t)buf * 256u, idesc = p.a_mn ? idesc_bf16_pair(p.bn, true, true) : idesc_bf16_pair(p.bn, false, true);
            const uint64_t a0 = p.a_mn ? a_mn0 : a_k0;
            const uint32_t a_step = p.a_mn ? 128u : 2u;      // of 16 rows of K, in 16 bytes
            ok = mbar_wait_uniform(smem_u32(&out_empty[buf]), ((i >> 1) & 1) ^ 1, ab);      // accumulator buffer drained
            tc_fence_after();
            uint32_t ready = mbar_test_wait(smem_u32(&full_bar[s]), ph);
            for (int kb = 0; kb < kb_total && ok; ++kb) {
                ok = mbar_wait_peeked(ready, smem_u32(&full_bar[s]), ph, ab);
                if (!ok) break;
                tc_fence_after();
                const uint64_t ad = a0 + (uint32_t)s * (kStageBytes >> 4), bd = b_desc0 + (uint32_t)s * (kStageBytes >> 4);
                const uint32_t eb = smem_u32(&empty_bar[s]);
                const bool last = kb + 1 == kb_total;
                if (++s == kStages) { s = 0; ph ^= 1; }
                ready = last ? 0u : mbar_test_wait(smem_u32(&full_bar[s]), ph);
                if (elect_one()) {
#pragma unroll
                    for (uint32_t kk = 0; kk < BK / 16; ++kk) mma_bf16_ss_pair(d_tmem, ad + kk * a_step, bd + kk * 128u, idesc, kb > 0 || kk > 0 ? 1u : 0u);
                    mma_commit_pair(eb, 3);                  // both blocks' stages are free, both blocks' accumulators are ready
                    if (last) mma_commit_pair(smem_u32(&out_full[buf]), 3);
                }
                __syncwarp();
            }
        }
    } else if (warp >= 2) {
        // ------------------------------------------------------------------ epilogue
        const int q = warp % 4;                              // tensor-memory lanes [32 q, 32 q + 32)
        const int hw = (warp - 2) / 4;                       // two warps share a quarter: they take alternate 32-column pieces
        const uint32_t lane_addr = tmem_base + ((uint32_t)(q * 32) << 16);
        const uint32_t slab0 = staging_base + (uint32_t)(warp - 2) * 2u * kSlabBytes;
        const uint32_t row_off = (uint32_t)lane * 64u, row_xor = ((uint32_t)lane >> 1) & 3u;
        int i = 0, sb = 0;
        bool ok = true;
        for (int t = unit; t < total && ok; t += n_units, ++i) {
            const bool second = t >= ps.p[0].tiles;
            const Product& p = ps.p[second];
            const CUtensorMap* mC = second ? &tC1 : &tC0;
            const int buf = i & 1;
            int mt, nt;
            tile_at(second ? t - ps.p[0].tiles : t, p.m_tiles, p.n_tiles, p.m_group, mt, nt);
            const int m0 = mt * 256 + h * BM + q * 32, n0 = nt * p.bn;
            const bool rows_inside = m0 < p.M;               // (uniform) the odd block may hang over the last row tile
            ok = mbar_wait_uniform(smem_u32(&out_full[buf]), (i >> 1) & 1, ab);
            if (!ok) break;
            tc_fence_after();
            const uint32_t d_tmem = lane_addr + (uint32_t)buf * 256u;
#pragma unroll 1
            for (int c0 = hw; c0 < p.bn / 32; c0 += 4) {     // this warp's pieces, two at a time
                if (n0 + c0 * 32 >= p.N) break;              // (uniform) nothing of this piece is inside
                const bool both = c0 + 2 < p.bn / 32 && n0 + c0 * 32 + 64 < p.N;
                uint32_t v2[2][32];
                tmem_ld_32x32(d_tmem + c0 * 32, v2[0]);
                if (both) tmem_ld_32x32(d_tmem + c0 * 32 + 64, v2[1]);
                tmem_ld_wait();
#pragma unroll
                for (int h2 = 0; h2 < 2; ++h2, ++sb) {
                    if (h2 == 1 && !both) break;             // (uniform)
                    const uint32_t(&v)[32] = v2[h2];
                    const uint32_t slab = slab0 + (uint32_t)(sb & 1) * kSlabBytes;
                    if (sb >= 2) {                           // the store that last read this slab has finished reading
                        tma_store_wait_read<1>();
                        __syncwarp();
                    }
#pragma unroll
                    for (int cc = 0; cc < 4; ++cc)
                        st_shared_v4(slab + row_off + ((((uint32_t)cc) ^ row_xor) << 4),
                                     pack_bf16(__uint_as_float(v[8 * cc]), __uint_as_float(v[8 * cc + 1])),
                                     pack_bf16(__uint_as_float(v[8 * cc + 2]), __uint_as_float(v[8 * cc + 3])),
                                     pack_bf16(__uint_as_float(v[8 * cc + 4]), __uint_as_float(v[8 * cc + 5])),
                                     pack_bf16(__uint_as_float(v[8 * cc + 6]), __uint_as_float(v[8 * cc + 7])));
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (elect_one()) {
                        if (rows_inside) tma_store_2d(mC, slab, n0 + (c0 + 2 * h2) * 32, m0);
                        tma_store_commit();
                    }
                    __syncwarp();
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_remote(smem_u32(&out_empty[buf]), 0);
        }
        tma_store_wait_read<0>();                            // shared memory may go once the stores have read it
        __syncwarp();
    }

    tc_fence_before();
    cluster_arrive();                // (as in the persistent product: neither block leaves while the other may still reach it)
    cluster_wait();
    if (warp == 1) {
        if (abort_flag) {            // give copies and MMAs still in flight time to land before freeing
            for (int i = 0; i < 256; ++i) __nanosleep(1000);
        }
        tc_fence_after();
        tmem_dealloc_pair(tmem_base, 512);
    }
}

constexpr int64_t kUnits = kNumSms / 2;
// microseconds of a k-block of a tile on a pair
double k_block_us(int bn) { return bn == 256 ? 0.37 : bn == 192 ? 0.32 : 0.26; }
int64_t tiles_of(const GemmArgs& g, int bn) { return (g.M + 255) / 256 * ((g.N + bn - 1) / bn); }
double tile_us(const GemmArgs& g, int bn) { return (double)((g.K + BK - 1) / BK) * k_block_us(bn) + 0.3; }
// A walk over one product's tiles on all pairs, at its best width
double alone_us(const GemmArgs& g) {
    double best = 1e300;
    for (int bn : {256, 192, 128}) best = std::min(best, (double)((tiles_of(g, bn) + kUnits - 1) / kUnits) * tile_us(g, bn));
    return best;
}
// Both in one walk, the tiles of `a` first: unit u takes every kUnits-th of the row of all tiles.  The longest unit is among those at which
// one of the two counts changes.
double together_us(const GemmArgs& a, int bn_a, const GemmArgs& b, int bn_b) {
    const int64_t ta = tiles_of(a, bn_a), all = ta + tiles_of(b, bn_b);
    double longest = 0;
    for (int64_t u : {(int64_t)0, ta % kUnits, all % kUnits}) {
        const int64_t na = ta > u ? (ta - u + kUnits - 1) / kUnits : 0, n = all > u ? (all - u + kUnits - 1) / kUnits : 0;
        longest = std::max(longest, (double)na * tile_us(a, bn_a) + (double)(n - na) * tile_us(b, bn_b));
    }
    return longest;
}

}  // namespace

bool tc_two_products_best(const GemmArgs& dx, const GemmArgs& dw, bool dw_walks, double more_us) {
    if (!tc_gemm_eligible(dx) || !tc_gemm_eligible(dw) || dx.a_mn_major || !dx.b_mn_major || !dw.a_mn_major || !dw.b_mn_major) return false;
    if (dx.N % 8 || dw.N % 8) return false;                  // (results leave by TMA, in whole 16 bytes)
    if (dx.M < 256 || dw.M < 256 || dw.a_colsum || dw.add || dw.any_rows || dx.bias || dw.bias) return false;
    int bx, bw;
    bool first;
    // a launch by itself has some 3 us before its first and behind its last MMAs; the estimates of the kernels that split a reduction go by the
    // tensor pipe's undisturbed pace, a third above the one here
    const double dx_us = tc_splits_data_product(dx.M, dx.N, dx.K) ? 1.3 * tc_gemm_estimate(dx.M, dx.N, dx.K) : alone_us(dx) + 3.0;
    const double dw_us = dw_walks ? alone_us(dw) + 3.0 : std::min(1.3 * tc_wgrad_pair_estimate(&dw, 1), alone_us(dw) + 3.0);
    // (by 2 %: where many rounds leave less than that to gain, one product's strips of operands push the other's out of L2.  Backward passes, one
    // launch for the two / one each: 4096 x 1024 -> 2 x 2816 with a bias 89 / 95 us, 3655 x 1176 -> 2 x 640 30 / 39, 2048 x 2048 -> 2 x 5632 146 / 155,
    // 1336 x 256 -> 2 x 768 with a bias 17.2 / 19.7, 8192 x 4096 -> 2 x 10752 2330 to 2580 / 2370 to 2430.)
    return tc_two_products_plan(dx, dw, &bx, &bw, &first) + 3.0 + more_us < 0.98 * (dx_us + dw_us);
}

double tc_two_products_plan(const GemmArgs& dx, const GemmArgs& dw, int* bx, int* bw, bool* dw_first) {
    double best = 1e300;
    for (int x : {256, 192, 128})
        for (int w : {256, 192, 128}) {
            const bool first = tile_us(dw, w) >= tile_us(dx, x);         // the longer tiles
            const double us = first ? together_us(dw, w, dx, x) : together_us(dx, x, dw, w);
            if (us < best) { best = us; *bx = x; *bw = w; *dw_first = first; }
        }
    return best;
}

lrd_status_t tc_two_products(const GemmArgs& dx, const GemmArgs& dw, cudaStream_t stream) {
    int bx, bw;
    bool dw_first;
    tc_two_products_plan(dx, dw, &bx, &bw, &dw_first);
    const GemmArgs* g[2] = {dw_first ? &dw : &dx, dw_first ? &dx : &dw};
    const int bn[2] = {dw_first ? bw : bx, dw_first ? bx : bw};
    CUtensorMap tA[2], tB[2], tC[2];
    Products ps;
    bool ok = true;
    for (int i = 0; i < 2; ++i) {
        const GemmArgs& a = *g[i];
        Product& p = ps.p[i];
        p.M = a.M; p.N = a.N;
        p.kb_total = (int)((a.K + BK - 1) / BK);
        p.m_tiles = (int)((a.M + 255) / 256);
        p.n_tiles = (int)((a.N + bn[i] - 1) / bn[i]);
        if (tiles_of(a, bn[i]) > 0x3FFFFFFF) return LRD_ERR_TOO_LARGE;
        p.tiles = p.m_tiles * p.n_tiles;
        p.m_group = tile_group(p.m_tiles, p.n_tiles, kUnits, (int64_t)256 * a.K * 2, (int64_t)bn[i] * a.K * 2);
        p.bn = bn[i]; p.a_mn = a.a_mn_major;
        ok = ok && (a.a_mn_major ? make_tmap_2d_bf16(&tA[i], a.A, (uint64_t)a.K, (uint64_t)a.M, (uint64_t)a.lda, BK, 64)
                                 : make_tmap_2d_bf16(&tA[i], a.A, (uint64_t)a.M, (uint64_t)a.K, (uint64_t)a.lda, BM, BK));
        ok = ok && make_tmap_2d_bf16(&tB[i], a.B, (uint64_t)a.K, (uint64_t)a.N, (uint64_t)a.ldb, BK, 64);
        ok = ok && make_tmap_2d_bf16(&tC[i], a.C, (uint64_t)a.M, (uint64_t)a.N, (uint64_t)a.ldc, 32, 32);
    }
    if (!ok) return LRD_ERR_CUDA;
    ps.timeout_flag = device_timeout_flag();
    static bool configured_on[kMaxDevices] = {};     // (the attribute is sticky per function)
    bool& configured = configured_on[device_slot()];
    if (!configured) {
        if (cudaFuncSetAttribute(two_products_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes) != cudaSuccess) return LRD_ERR_CUDA;
        configured = true;
    }
    const int64_t total = (int64_t)ps.p[0].tiles + ps.p[1].tiles;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(total < kUnits ? total : kUnits) * 2, 1, 1);
    cfg.blockDim = dim3(kThreads, 1, 1);
    cfg.dynamicSmemBytes = kSmemBytes;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;   // the kernel waits (griddepcontrol.wait)
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 2;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    if (!cuda_ok(cudaLaunchKernelEx(&cfg, two_products_kernel, tA[0], tB[0], tC[0], tA[1], tB[1], tC[1], ps), "cudaLaunchKernelEx(two products)")) return LRD_ERR_CUDA;
    count_launch();
    return LRD_OK;
}

}  // namespace lrd
