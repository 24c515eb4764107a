// Gated blocks and 8-bit products of a few tokens (decoding): out = act(G) * U or X W^T + bias with at most four rows of X.
//
// Such a call reads W once and computes next to nothing, so the floor is W's bytes over the memory's rate, and what counts is how
// little stands before the first load and how many bytes are on their way.  A warp takes R columns of the output: the R rows of W (2 R
// gated) stream through its registers in 16-byte pieces, 512 consecutive bytes an instruction and several of them in flight; the
// tokens' pieces come from L1, where the block's other warps find them too.  Sums are fp32 (or exact 32-bit integers, four products
// an instruction), added over the lanes at the end; one lane per result applies scales, bias and gate.  No shared memory, tensor
// memory or descriptors to set up.
#include "glu.cuh"
#include "ptx.cuh"
#include "tc.cuh"

namespace lrd {
namespace {

template <typename T> __device__ __forceinline__ float element(T x) { return (float)x; }

// 16 bytes of W: used once, not kept in L1
__device__ __forceinline__ uint4 load_stream(const void* p) {
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
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

template <typename T> struct Sum { using type = float; };
template <> struct Sum<int8_t> { using type = int; };

// MT: tokens, rounded up (those past M repeat the last and are dropped).  WIDE: rows on 16-byte boundaries; else element by element.
template <typename T, bool GATED, typename OUT, int MT, int R, bool WIDE>
__global__ void __launch_bounds__(256) few_tokens_kernel(const GluArgs a) {
    using S = typename Sum<T>::type;
    constexpr bool I8 = sizeof(T) == 1, EXACT = sizeof(OUT) == 4;
    constexpr int ROWS = GATED ? 2 * R : R;                  // rows of W: R of the gate, then R of the other half
    constexpr int E = 16 / sizeof(T);
    constexpr int DEPTH = ROWS >= 4 ? 2 : ROWS == 2 ? 4 : 8; // pieces of a row in flight
    constexpr int LOOSE = WIDE ? 1 : 8;
    static_assert(MT * R <= 32, "a lane per result");
    ptx::griddep_wait();
    ptx::griddep_launch_dependents();
    const int lane = threadIdx.x & 31;
    const int64_t n0 = ((int64_t)blockIdx.x * 8 + threadIdx.x / 32) * R;
    if (n0 >= a.N) return;
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
        for (int64_t p0 = lane; p0 < pieces; p0 += 32 * DEPTH) {
            uint4 wv[DEPTH][ROWS];
#pragma unroll
            for (int d = 0; d < DEPTH; ++d)
#pragma unroll
                for (int r = 0; r < ROWS; ++r)
                    wv[d][r] = p0 + 32 * d < pieces ? load_stream(w[r] + (p0 + 32 * d) * E) : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int d = 0; d < DEPTH; ++d) {
                if (p0 + 32 * d >= pieces) break;
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    const uint4 xv = *reinterpret_cast<const uint4*>(x[m] + (p0 + 32 * d) * E);
#pragma unroll
                    for (int r = 0; r < ROWS; ++r) piece_products(acc[m][r], xv, wv[d][r], (const T*)nullptr);
                }
            }
        }
    }
    for (int64_t k0 = done + lane; k0 < a.K; k0 += 32 * LOOSE) {     // single elements, several of each row in flight
        T wv[LOOSE][ROWS], xv[LOOSE][MT];
#pragma unroll
        for (int d = 0; d < LOOSE; ++d) {
            const int64_t k = k0 + 32 * d;
#pragma unroll
            for (int r = 0; r < ROWS; ++r) wv[d][r] = k < a.K ? w[r][k] : (T)0.0f;
#pragma unroll
            for (int m = 0; m < MT; ++m) xv[d][m] = k < a.K ? x[m][k] : (T)0.0f;
        }
#pragma unroll
        for (int d = 0; d < LOOSE; ++d)
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int r = 0; r < ROWS; ++r) acc[m][r] += (S)xv[d][m] * (S)wv[d][r];
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
    const int64_t m = lane / R, n = n0 + lane % R;
    if (m >= a.M || m >= MT || n >= a.N) return;
    auto projection = [&](S sum, int64_t col) {
        const float bias = a.bias ? element(((const OUT*)a.bias)[col]) : 0.0f;
        return I8 ? fmaf((float)sum * a.x_scale[m], a.w_scale[col], bias) : (float)sum + bias;
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
    auto kern = wide_rows(g) ? few_tokens_kernel<T, GATED, OUT, MT, R, true> : few_tokens_kernel<T, GATED, OUT, MT, R, false>;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((g.N + 8 * R - 1) / (8 * R)), 1, 1);
    cfg.blockDim = dim3(256, 1, 1);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;   // the kernel waits (griddepcontrol.wait) first
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (!cuda_ok(cudaLaunchKernelEx(&cfg, kern, g), "cudaLaunchKernelEx(few tokens)")) return LRD_ERR_CUDA;
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
