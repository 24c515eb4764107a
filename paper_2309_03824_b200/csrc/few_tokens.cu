// Gated blocks and 8-bit products of a few tokens (decoding): out = act(G) * U or X W^T + bias with at most four rows of X.
//
// Such a call reads W once and computes next to nothing, so the floor is W's bytes over the memory's rate, and what counts is how
// little stands before the first load and how many bytes are on their way.  A warp takes R columns of the output: the R rows of W (2 R
// gated) stream through its registers in 16-byte pieces, 512 consecutive bytes an instruction and several of them in flight; the
// tokens' pieces come from L1, where the block's other warps find them too.  Sums are fp32 (or exact 32-bit integers, four products
// an instruction), added over the lanes at the end; one lane per result applies scales, bias and gate.  Where the columns are too few to
// give every SM warps enough, 2, 4 or 8 warps of a block share a row's pieces and add up through shared memory, in their order.  No
// tensor memory or descriptors to set up.
#include "glu.cuh"
#include "ptx.cuh"
#include "tc.cuh"

namespace lrd {
namespace {

template <typename T> __device__ __forceinline__ float element(T x) { return (float)x; }

// 16 bytes of W: used once, not kept in L1.  (Not ld.global.nc: the launch in front, still at work when this kernel starts, may have written W.)
__device__ __forceinline__ uint4 load_stream(const void* p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
// acc += sum of the products of two 16-byte pieces
__device__ __forceinline__ void piece_products(float& acc, const uint4& a, const uint4& b, const __nv_bfloat16*) {
    const uint32_t x[4] = {a.x, a.y, a.z, a.w}, y[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        acc = fmaf(__uint_as_float(x[i] << 16), __uint_as_float(y[i] << 16), acc);
        acc = fmaf(__uint_as_float(x[i] & 0xFFFF0000u), __uint_as_float(y[i] & 0xFFFF0000u), acc);
    }
}
__device__ __forceinline__ void piece_products(float& acc, const uint4& a, const uint4& b, const float*) {
    acc = fmaf(__uint_as_float(a.x), __uint_as_float(b.x), acc);
    acc = fmaf(__uint_as_float(a.y), __uint_as_float(b.y), acc);
    acc = fmaf(__uint_as_float(a.z), __uint_as_float(b.z), acc);
    acc = fmaf(__uint_as_float(a.w), __uint_as_float(b.w), acc);
}
__device__ __forceinline__ void piece_products(int& acc, const uint4& a, const uint4& b, const int8_t*) {
    acc = __dp4a((int)a.x, (int)b.x, acc);
    acc = __dp4a((int)a.y, (int)b.y, acc);
    acc = __dp4a((int)a.z, (int)b.z, acc);
    acc = __dp4a((int)a.w, (int)b.w, acc);
}
__device__ __forceinline__ void warp_sum(float& v) {
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
}
__device__ __forceinline__ void warp_sum(int& v) { v = __reduce_add_sync(0xffffffffu, v); }

// The 16 bytes from byte `shift` (below 16, the same in all lanes) of two neighbouring pieces on
__device__ __forceinline__ uint4 window(const uint4& a, const uint4& b, uint32_t shift) {
    uint32_t v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 6; ++i) v[i] = shift & 8 ? v[i + 2] : v[i];
#pragma unroll
    for (int i = 0; i < 5; ++i) v[i] = shift & 4 ? v[i + 1] : v[i];
    const uint32_t bits = 8 * (shift & 3);
    return make_uint4(__funnelshift_r(v[0], v[1], bits), __funnelshift_r(v[1], v[2], bits), __funnelshift_r(v[2], v[3], bits),
                      __funnelshift_r(v[3], v[4], bits));
}

template <typename T> struct Sum { using type = float; };
template <> struct Sum<int8_t> { using type = int; };

// pieces of a row in flight
__host__ __device__ constexpr int depth_of(int rows) { return rows >= 4 ? 2 : rows == 2 ? 4 : 8; }

// MT: tokens, rounded up (those past M repeat the last and are dropped).  WIDE: rows on 16-byte boundaries.  Others are read in the
// pieces that lie on boundaries of W, each against the window of X that belongs to it, put together from X's two pieces there; both
// ends of a row, so far in that all those pieces lie inside the rows, go element by element.  (All of it element by element, us:
// 8-bit, one token, 4096 rows of 10751 bytes 34.7, so 17.0; four, 2 x 896 of 6190 25.5 / 9.6; fp32, one, 2 x 700 of 11007 51 / 16.8.)
template <typename T, bool GATED, typename OUT, int MT, int R, bool WIDE, bool SHARED>
__global__ void __launch_bounds__(256) few_tokens_kernel(const GluArgs a, int warps_a_row) {
    const int share = SHARED ? warps_a_row : 1;              // (a constant 1 is worth 0.3 to 0.5 us a call)
    using S = typename Sum<T>::type;
    constexpr bool I8 = sizeof(T) == 1, EXACT = sizeof(OUT) == 4;
    constexpr int ROWS = GATED ? 2 * R : R;                  // rows of W: R of the gate, then R of the other half
    constexpr int E = 16 / sizeof(T);
    constexpr int DEPTH = depth_of(ROWS);
    static_assert(MT * R <= 32, "a lane per result");
    ptx::griddep_wait();
    ptx::griddep_launch_dependents();
    __shared__ S handed[SHARED ? 8 : 1][32][2];
    const int lane = threadIdx.x & 31, warp = threadIdx.x / 32, slice = warp % share;      // `share` warps to a row
    const int64_t n0 = ((int64_t)blockIdx.x * (8 / share) + warp / share) * R;
    if (!SHARED && n0 >= a.N) return;                     // (else the block meets below; such warps read the last column)
    const T *w[ROWS], *x[MT];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const int64_t n = n0 + r % R < a.N ? n0 + r % R : a.N - 1;
        w[r] = (const T*)a.W + (n + (r < R ? 0 : a.N)) * a.ldw;
    }
#pragma unroll
    for (int m = 0; m < MT; ++m) x[m] = (const T*)a.X + (m < a.M ? m : a.M - 1) * a.ldx;
    S acc[MT][ROWS] = {};
    int64_t done = 0;                                        // elements of the rows that whole pieces cover
    if (WIDE) {
        const int64_t pieces = a.K / E;
        done = pieces * E;
        const int step = 32 * share;
        for (int64_t p0 = 32 * slice + lane; p0 < pieces; p0 += step * DEPTH) {
            uint4 wv[DEPTH][ROWS];
#pragma unroll
            for (int d = 0; d < DEPTH; ++d)
#pragma unroll
                for (int r = 0; r < ROWS; ++r)
                    wv[d][r] = p0 + step * d < pieces ? load_stream(w[r] + (p0 + step * d) * E) : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int d = 0; d < DEPTH; ++d) {
                if (p0 + step * d >= pieces) break;
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    const uint4 xv = *reinterpret_cast<const uint4*>(x[m] + (p0 + step * d) * E);
#pragma unroll
                    for (int r = 0; r < ROWS; ++r) piece_products(acc[m][r], xv, wv[d][r], (const T*)nullptr);
                }
            }
        }
    }
    if (WIDE) {
        for (int64_t k = done + 32 * slice + lane; k < a.K; k += 32 * share) {
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                const T wv = w[r][k];
#pragma unroll
                for (int m = 0; m < MT; ++m) acc[m][r] += (S)x[m][k] * (S)wv;
            }
        }
    } else {
        int head[ROWS];                                      // first element of the pieces: the second boundary of W's row
        int64_t pieces[ROWS], most = 0;
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            head[r] = (int)((-(uintptr_t)w[r] & 15) + 16) / (int)sizeof(T);
            pieces[r] = a.K >= head[r] + 2 * E ? (a.K - head[r] - E) / E : 0;      // X's last piece ends at most E further on
            if (pieces[r] == 0) head[r] = 0;
            most = max(most, pieces[r]);
        }
        const int step = 32 * share;
        for (int64_t p0 = 32 * slice + lane; p0 < most; p0 += step * DEPTH) {
            uint4 wv[DEPTH][ROWS];
#pragma unroll
            for (int d = 0; d < DEPTH; ++d)
#pragma unroll
                for (int r = 0; r < ROWS; ++r)
                    wv[d][r] = p0 + step * d < pieces[r] ? load_stream(w[r] + head[r] + (p0 + step * d) * E) : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int d = 0; d < DEPTH; ++d)
#pragma unroll
                for (int r = 0; r < ROWS; ++r) {
                    if (p0 + step * d >= pieces[r]) continue;
#pragma unroll
                    for (int m = 0; m < MT; ++m) {
                        const uintptr_t at = (uintptr_t)(x[m] + head[r] + (p0 + step * d) * E);
                        const uint4* pair = reinterpret_cast<const uint4*>(at & ~(uintptr_t)15);
                        piece_products(acc[m][r], window(pair[0], pair[1], (uint32_t)at & 15), wv[d][r], (const T*)nullptr);
                    }
                }
        }
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {                     // what stands before and behind the pieces
            const int64_t skipped = pieces[r] * E, singles = a.K - skipped;
            for (int64_t i = 32 * slice + lane; i < singles; i += step) {
                const int64_t k = i < head[r] ? i : i + skipped;
                const T wv = w[r][k];
#pragma unroll
                for (int m = 0; m < MT; ++m) acc[m][r] += (S)x[m][k] * (S)wv;
            }
        }
    }
    S g = 0, u = 0;                                          // lane m R + r: token m, column n0 + r
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int r = 0; r < R; ++r) {
            warp_sum(acc[m][r]);
            if (GATED) warp_sum(acc[m][R + r]);
            if (lane == m * R + r) {
                g = acc[m][r];
                if (GATED) u = acc[m][R + r];
            }
        }
    if (SHARED) {
        handed[warp][lane][0] = g;
        handed[warp][lane][1] = u;
        __syncthreads();
        if (slice) return;
        for (int i = 1; i < share; ++i) {
            g += handed[warp + i][lane][0];
            u += handed[warp + i][lane][1];
        }
    }
    const int64_t m = lane / R, n = n0 + lane % R;
    if (m >= a.M || m >= MT || n >= a.N) return;
    auto projection = [&](S sum, int64_t col) {
        const float bias = a.bias ? element(((const OUT*)a.bias)[col]) : 0.0f;
        return I8 ? fmaf((float)sum * a.w_scale[col], a.x_scale[m], bias) : (float)sum + bias;
    };
    const float gv = projection(g, n);
    OUT* out = (OUT*)a.out + m * a.ldo + n;
    if (!GATED) {
        *out = (OUT)gv;
        return;
    }
    const float uv = projection(u, a.N + n);
    with_act(a.act, [&](auto tag) { *out = (OUT)(act_value<decltype(tag)::value, EXACT>(gv) * uv); });
    if (a.p_save) {
        OUT* p = (OUT*)a.p_save + m * a.ldp + n;
        p[0] = (OUT)gv;
        p[a.N] = (OUT)uv;
    }
}

// Whole 16-byte pieces a row, on such boundaries
bool wide_rows(const GluArgs& g) {
    const int64_t e = g.x_scale ? 16 : 16 / (int64_t)elem_size(g.dtype);
    return g.ldx % e == 0 && g.ldw % e == 0 && (((uintptr_t)g.X | (uintptr_t)g.W) & 15u) == 0;
}

template <typename T, bool GATED, typename OUT, int MT, int R> lrd_status_t launch(const GluArgs& g, cudaStream_t s) {
    // As many warps to a row as give the SMs 24 each, while each has more of the row than it keeps in flight at once.  One warp a row and
    // so, us: one token, bf16, 2 x 512 rows of 8 KB 6.7 / 3.4, two, 2 x 1024 of 4 KB 4.4 / 3.7; 8-bit, three, 512 of 8 KB 6.4 / 3.3.
    constexpr int rows = GATED ? 2 * R : R;
    const int64_t groups = (g.N + R - 1) / R, row_bytes = g.K * (int64_t)sizeof(T);
    const int64_t flight = 512 * depth_of(rows);
    int share = 1;
    while (share < 8 && groups * share * 2 <= kNumSms * 24 && row_bytes > flight * share) share *= 2;
    auto kern = share > 1 ? wide_rows(g) ? few_tokens_kernel<T, GATED, OUT, MT, R, true, true> : few_tokens_kernel<T, GATED, OUT, MT, R, false, true>
                          : wide_rows(g) ? few_tokens_kernel<T, GATED, OUT, MT, R, true, false> : few_tokens_kernel<T, GATED, OUT, MT, R, false, false>;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((groups * share + 7) / 8), 1, 1);
    cfg.blockDim = dim3(256, 1, 1);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;   // the kernel waits (griddepcontrol.wait) first
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (!cuda_ok(cudaLaunchKernelEx(&cfg, kern, g, share), "cudaLaunchKernelEx(few tokens)")) return LRD_ERR_CUDA;
    count_launch();
    return LRD_OK;
}

template <typename T, bool GATED, typename OUT> lrd_status_t by_tokens(const GluArgs& g, cudaStream_t s) {
    if (g.M == 1) return launch<T, GATED, OUT, 1, 1>(g, s);
    if (g.M == 2) return launch<T, GATED, OUT, 2, 1>(g, s);
    return launch<T, GATED, OUT, 4, 2>(g, s);
}

}  // namespace

// Against the tensor-core kernel, us: one token, bf16, 2 x 2816 rows of W of 2 KB 4.0 / 6.4, 2 x 10752 of 8 KB 30.8 / 34.7; two 4.5 / 6.5 and 32.3 /
// 34.9; four 5.8 / 6.4 and 46 / 35 (8-bit, 4096 rows of 4 KB 5.9 / 9.0, 2 x 10752 of 4 KB 31 / 20): from three tokens on it is bound by
// its instructions where W is long.
bool few_tokens_best(const GluArgs& g) {
    if (g.M > kFewTokens) return false;
    const size_t w_bytes = (size_t)(g.gated ? 2 * g.N : g.N) * (size_t)g.K * (g.x_scale ? 1 : elem_size(g.dtype));
    return g.M <= 2 || w_bytes <= ((size_t)32 << 20) || !wide_rows(g);
}

lrd_status_t few_tokens(const GluArgs& g, cudaStream_t s) {
    if (!g.x_scale) return g.dtype == LRD_BF16 ? by_tokens<__nv_bfloat16, true, __nv_bfloat16>(g, s) : by_tokens<float, true, float>(g, s);
    if (g.dtype == LRD_BF16) return g.gated ? by_tokens<int8_t, true, __nv_bfloat16>(g, s) : by_tokens<int8_t, false, __nv_bfloat16>(g, s);
    return g.gated ? by_tokens<int8_t, true, float>(g, s) : by_tokens<int8_t, false, float>(g, s);
}

}  // namespace lrd
