// The gate of a feed-forward block on its own (element by element), rows quantized to 8 bits, and the general fp32-FMA form of the
// gated block.
#include <cstdint>

#include "glu.cuh"
#include "ptx.cuh"
#include "tc.cuh"

namespace lrd {
namespace {

template <typename T> __device__ __forceinline__ float to_f32(T x) { return (float)x; }
template <typename T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// VEC consecutive elements: one 16-byte access where VEC fills it, else one element
template <typename T, int VEC> struct Pack { float v[VEC]; };
template <typename T, int VEC> __device__ __forceinline__ void load_pack(Pack<T, VEC>& p, const T* at) {
    if constexpr (VEC == 1) {
        p.v[0] = to_f32(*at);
    } else {
        const uint4 w = *reinterpret_cast<const uint4*>(at);
        const T* e = reinterpret_cast<const T*>(&w);
#pragma unroll
        for (int i = 0; i < VEC; ++i) p.v[i] = to_f32(e[i]);
    }
}
template <typename T, int VEC> __device__ __forceinline__ void store_pack(T* at, const Pack<T, VEC>& p) {
    if constexpr (VEC == 1) {
        *at = from_f32<T>(p.v[0]);
    } else {
        uint4 w;
        T* e = reinterpret_cast<T*>(&w);
#pragma unroll
        for (int i = 0; i < VEC; ++i) e[i] = from_f32<T>(p.v[i]);
        *reinterpret_cast<uint4*>(at) = w;
    }
}

struct GateParams {
    int64_t M, N;
    const void *P, *dH;
    void *H, *dP;
    int64_t ldp, ldh, lddp;
    int act;
};

// BWD = false: H = act(G) * U.  BWD = true: dP = [dH * U * act'(G) | dH * act(G)].  Bound by memory: 3 or 5 elements move for each of
// H, in 16-byte accesses where bases, strides and N allow, else one element at a time.  A thread steps over the (row, piece) pairs
// by a fixed stride, kept as a row and a column so that only its first step divides, and has the loads of DEPTH steps in flight.  P and dP may
// be the same memory: a thread reads both halves' pieces before it writes them, and no other thread touches those.
template <typename T, int VEC, bool BWD, int ACT>
__global__ void __launch_bounds__(256) gate_kernel(const GateParams p) {
    constexpr bool EXACT = sizeof(T) == 4;
    constexpr int DEPTH = VEC == 1 ? 4 : 1;
    ptx::griddep_wait();
    ptx::griddep_launch_dependents();
    const int64_t cols = p.N / VEC, step = (int64_t)gridDim.x * 256;
    const int64_t first = (int64_t)blockIdx.x * 256 + threadIdx.x, drow = step / cols, dcol = step % cols;
    int64_t row = first / cols, col = first % cols;
    while (row < p.M) {
        Pack<T, VEC> g[DEPTH], u[DEPTH], d[DEPTH];
        int64_t rows[DEPTH], at[DEPTH];
#pragma unroll
        for (int i = 0; i < DEPTH; ++i) {
            rows[i] = row;
            at[i] = col * VEC;
            if (row < p.M) {
                const T* P = (const T*)p.P + row * p.ldp + at[i];
                load_pack(g[i], P);
                load_pack(u[i], P + p.N);
                if (BWD) load_pack(d[i], (const T*)p.dH + row * p.ldh + at[i]);
            }
            row += drow;
            col += dcol;
            if (col >= cols) { col -= cols; ++row; }
        }
#pragma unroll
        for (int i = 0; i < DEPTH; ++i) {
            if (rows[i] >= p.M) break;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                if (!BWD) {
                    g[i].v[e] = act_value<ACT, EXACT>(g[i].v[e]) * u[i].v[e];
                } else {
                    float value, slope;
                    act_both<ACT, EXACT>(g[i].v[e], value, slope);
                    g[i].v[e] = d[i].v[e] * u[i].v[e] * slope;
                    u[i].v[e] = d[i].v[e] * value;
                }
            }
            T* to = BWD ? (T*)p.dP + rows[i] * p.lddp + at[i] : (T*)p.H + rows[i] * p.ldh + at[i];
            store_pack(to, g[i]);
            if (BWD) store_pack(to + p.N, u[i]);
        }
    }
}

bool launch_pdl(const void* kern, dim3 grid, unsigned threads, void** args, cudaStream_t s) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads, 1, 1);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;   // every kernel here waits (griddepcontrol.wait) first
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (!cuda_ok(cudaLaunchKernelExC(&cfg, kern, args), "cudaLaunchKernelExC(gate)")) return false;
    count_launch();
    return true;
}

template <typename T, int VEC, bool BWD> lrd_status_t launch_gate(const GateParams& p, cudaStream_t s) {
    auto kern = p.act == LRD_ACT_SILU ? gate_kernel<T, VEC, BWD, LRD_ACT_SILU>
              : p.act == LRD_ACT_GELU ? gate_kernel<T, VEC, BWD, LRD_ACT_GELU> : gate_kernel<T, VEC, BWD, LRD_ACT_GELU_TANH>;
    // (a block of 256 threads per piece of 256 accesses, at most 16 blocks for each SM: the rows that are left follow in the loop)
    const int64_t cols = p.N / VEC, most = (int64_t)kNumSms * 16;
    const int64_t blocks = p.M > most * 256 / cols ? most : (p.M * cols + 255) / 256;
    GateParams q = p;
    void* args[] = {&q};
    return launch_pdl((const void*)kern, dim3((unsigned)blocks), 256, args, s) ? LRD_OK : LRD_ERR_CUDA;
}

bool on16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

template <bool BWD> lrd_status_t run_gate(const GateParams& p, lrd_dtype_t dt, cudaStream_t s) {
    if (p.M <= 0) return LRD_OK;
    const int vec = 16 / (int)elem_size(dt);
    const int64_t out_ld = BWD ? p.lddp : p.ldh;
    const bool wide = p.N % vec == 0 && p.ldp % vec == 0 && p.ldh % vec == 0 && out_ld % vec == 0 && on16(p.P) && (BWD ? on16(p.dH) && on16(p.dP) : on16(p.H));
    if (dt == LRD_BF16) return wide ? launch_gate<__nv_bfloat16, 8, BWD>(p, s) : launch_gate<__nv_bfloat16, 1, BWD>(p, s);
    return wide ? launch_gate<float, 4, BWD>(p, s) : launch_gate<float, 1, BWD>(p, s);
}

// ---- rows to 8 bits -----------------------------------------------------------------------------------------------
// scale = max |x| fl(1 / 127), q = x / scale rounded to the nearest integer, ties to even: of the real quotient, not of a
// rounded one.  fma(x, 1 / scale, 1.5 2^23) holds an integer in its low bits that is off by one step at most; the remainder
// x - q scale, which an fma forms exactly (x and q scale are multiples of the last place of either, and no more than some scale
// apart), then says whether it is the nearest.  No branch: in bf16 quotients within 2^-23 of a border are nothing rare (8192 x 4096: 26 us
// so, 43 to 55 with a branch for them).
// PARITY: quotients that lie on a border exactly need the even one of the two.  With bf16 rows the scale is then a power of two (it is
// the largest value, 8 bits, times fl(1 / 127); of all such products only powers of two are a 2 / (2 n + 1) of an 8-bit number), its
// reciprocal exact, and the fma has rounded to even already.
struct RowScale { float scale, inv, half, past_half; };      // past_half: the next fp32 number after scale / 2
template <bool PARITY> __device__ __forceinline__ uint32_t quantize_one(float x, const RowScale& r) {
    constexpr float kRound = 12582912.0f;                    // 1.5 2^23
    const float t = fmaf(x, r.inv, kRound), rest = fmaf(kRound - t, r.scale, x);
    uint32_t q = __float_as_uint(t);
    if (PARITY ? fabsf(rest) >= (q & 1u ? r.half : r.past_half) : fabsf(rest) > r.half) q += (uint32_t)((__float_as_int(rest) >> 31) | 1);
    return q;                                                // (the low byte)
}
// Scales too small for that (their reciprocal or the remainder may leave fp32's normal range): the quotient in fp64.  A subnormal scale
// is rounded by more than its last bit, so that the largest quotients may pass 127.
__device__ __forceinline__ int quantize_tiny(float x, float scale) {
    if (scale == 0.0f) return 0;
    const double q = rint((double)x / (double)scale);
    return (int)fmin(fmax(q, -127.0), 127.0);
}
// A row with such a scale, or (NaN) without one
template <typename T> __device__ __noinline__ void quantize_odd_row(const T* x, int8_t* q, int64_t K, float scale, int t, int step) {
    for (int64_t k = t; k < K; k += step) q[k] = scale == scale ? (int8_t)quantize_tiny(to_f32(x[k]), scale) : (int8_t)0;
}

// A piece: 16 bytes as they were loaded (or one element, VEC = 1)
template <typename T, int VEC> struct Raw { uint32_t w[VEC == 1 ? 1 : 4]; };
template <typename T, int VEC> __device__ __forceinline__ Raw<T, VEC> load_raw(const T* at) {
    Raw<T, VEC> r;
    if constexpr (VEC == 1) {
        r.w[0] = __float_as_uint(to_f32(*at));
    } else {
        const uint4 v = *reinterpret_cast<const uint4*>(at);
        r.w[0] = v.x; r.w[1] = v.y; r.w[2] = v.z; r.w[3] = v.w;
    }
    return r;
}
template <typename T, int VEC> __device__ __forceinline__ float raw_value(const Raw<T, VEC>& r, int e) {
    if constexpr (VEC == 8) return __uint_as_float(e & 1 ? r.w[e / 2] & 0xFFFF0000u : r.w[e / 2] << 16);
    else return __uint_as_float(r.w[e]);
}
// largest |x| so far, by its bits (infinities and NaN are above every number); of bf16 pairs, both halves side by side
template <typename T, int VEC> __device__ __forceinline__ void raw_top(uint32_t& top, const Raw<T, VEC>& r) {
    if constexpr (VEC == 8) {
#pragma unroll
        for (int i = 0; i < 4; ++i) top = __vmaxu2(top, r.w[i] & 0x7FFF7FFFu);
    } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) top = max(top, r.w[i] & 0x7FFFFFFFu);
    }
}

// A row's elements by `TPR` threads, a piece at a time; the first KEEP pieces of a thread stay in registers between the two passes,
// longer rows are read again (from L2).  Bound by memory.
template <typename T, int VEC, int TPR, int KEEP>
__global__ void __launch_bounds__(256) i8_quantize_kernel(const T* __restrict__ X, int64_t ldx, int64_t M, int64_t K, int8_t* __restrict__ Xq, int64_t ldq,
                                                          float* __restrict__ scale_out) {
    constexpr int ROWS = 256 / TPR;
    __shared__ uint32_t part[8];
    ptx::griddep_wait();
    ptx::griddep_launch_dependents();
    const int t = threadIdx.x % TPR;
    const int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / TPR, pieces = K / VEC;
    const bool live = row < M;
    const T* x = X + (live ? row : 0) * ldx;
    Raw<T, VEC> kept[KEEP];
    uint32_t top = 0;
    if (live) {
#pragma unroll
        for (int i = 0; i < KEEP; ++i)
            if (t + (int64_t)i * TPR < pieces) kept[i] = load_raw<T, VEC>(x + (t + (int64_t)i * TPR) * VEC);
#pragma unroll
        for (int i = 0; i < KEEP; ++i)
            if (t + (int64_t)i * TPR < pieces) raw_top<T, VEC>(top, kept[i]);
        for (int64_t at = t + (int64_t)KEEP * TPR; at < pieces; at += TPR) raw_top<T, VEC>(top, load_raw<T, VEC>(x + at * VEC));
    }
    if (VEC == 8) top = max(top & 0xFFFF0000u, top << 16);
    top = __reduce_max_sync(0xffffffffu, top);
    if (TPR > 32) {
        if (threadIdx.x % 32 == 0) part[threadIdx.x / 32] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < TPR / 32; ++w) top = max(top, part[(threadIdx.x / TPR) * (TPR / 32) + w]);
    }
    if (!live) return;
    const bool finite = top < 0x7F800000u;
    const float scale = finite ? __uint_as_float(top) * (1.0f / 127.0f) : __uint_as_float(0x7FC00000u);
    if (t == 0) scale_out[row] = scale;
    int8_t* q = Xq + row * ldq;
    if (!(scale >= 7.888609e-31f)) {                         // 2^-100; NaN
        quantize_odd_row(x, q, K, scale, t, TPR);
        return;
    }
    const float half = 0.5f * scale;
    const RowScale r{scale, 1.0f / scale, half, __uint_as_float(__float_as_uint(half) + 1u)};
    auto put = [&](const Raw<T, VEC>& v, int64_t at) {
        uint32_t b[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) b[e] = quantize_one<sizeof(T) == 4>(raw_value<T, VEC>(v, e), r);
        if constexpr (VEC == 1) {
            q[at] = (int8_t)b[0];
        } else {
            uint32_t w[VEC / 4];
#pragma unroll
            for (int i = 0; i < VEC / 4; ++i)
                w[i] = __byte_perm(__byte_perm(b[4 * i], b[4 * i + 1], 0x0040), __byte_perm(b[4 * i + 2], b[4 * i + 3], 0x0040), 0x5410);
            if constexpr (VEC == 8) *reinterpret_cast<uint2*>(q + at * 8) = make_uint2(w[0], w[1]);
            else *reinterpret_cast<uint32_t*>(q + at * 4) = w[0];
        }
    };
#pragma unroll
    for (int i = 0; i < KEEP; ++i)
        if (t + (int64_t)i * TPR < pieces) put(kept[i], t + (int64_t)i * TPR);
    for (int64_t at = t + (int64_t)KEEP * TPR; at < pieces; at += TPR) put(load_raw<T, VEC>(x + at * VEC), at);
}

template <typename T, int VEC, int TPR, int KEEP>
lrd_status_t launch_quantize_as(const T* x, int64_t ldx, int64_t M, int64_t K, int8_t* Xq, int64_t ldq, float* scale, cudaStream_t s) {
    void* args[] = {&x, &ldx, &M, &K, &Xq, &ldq, &scale};
    const int64_t rows = 256 / TPR;
    return launch_pdl((const void*)i8_quantize_kernel<T, VEC, TPR, KEEP>, dim3((unsigned)((M + rows - 1) / rows)), 256, args, s) ? LRD_OK : LRD_ERR_CUDA;
}
template <typename T, int VEC> lrd_status_t launch_quantize(const void* X, int64_t ldx, int64_t M, int64_t K, int8_t* Xq, int64_t ldq, float* scale, cudaStream_t s) {
    const T* x = (const T*)X;
    // as few threads a row as hold it in four pieces each (eight past a block of them)
    if (K <= 32 * 4 * VEC) return launch_quantize_as<T, VEC, 32, 4>(x, ldx, M, K, Xq, ldq, scale, s);
    if (K <= 64 * 4 * VEC) return launch_quantize_as<T, VEC, 64, 4>(x, ldx, M, K, Xq, ldq, scale, s);
    if (K <= 128 * 4 * VEC) return launch_quantize_as<T, VEC, 128, 4>(x, ldx, M, K, Xq, ldq, scale, s);
    return K <= 256 * 4 * VEC ? launch_quantize_as<T, VEC, 256, 4>(x, ldx, M, K, Xq, ldq, scale, s) : launch_quantize_as<T, VEC, 256, 8>(x, ldx, M, K, Xq, ldq, scale, s);
}

__global__ void __launch_bounds__(256) copy2d_bytes_kernel(uint8_t* __restrict__ dst, int64_t ldd, const uint8_t* __restrict__ src, int64_t lds, int64_t rows, int64_t cols) {
    ptx::griddep_wait();
    ptx::griddep_launch_dependents();
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x)
        for (int64_t c = threadIdx.x; c < cols; c += 256) dst[row * ldd + c] = src[row * lds + c];
}

// ---- the gated block in fp32 FMA ----------------------------------------------------------------------------------
// A block forms 64 rows x 32 columns of H: 64 rows of X against 32 rows of the gate's and 32 of the other half's weights, 16 deep
// at a time, the next tile on its way in registers.  A thread holds 4 rows x 2 columns of G and of U, so that the gate is applied
// where the sums stand.
constexpr int kTM = 64, kTH = 32, kTK = 16;
template <typename T> __device__ __forceinline__ void load4(float (&v)[4], const T* row, int64_t k, int64_t K, bool live, bool wide) {
    if (live && wide && k + 4 <= K) {
        if constexpr (sizeof(T) == 4) {
            const float4 w = *reinterpret_cast<const float4*>(row + k);
            v[0] = w.x; v[1] = w.y; v[2] = w.z; v[3] = w.w;
        } else {
            const uint2 w = *reinterpret_cast<const uint2*>(row + k);
            v[0] = __uint_as_float(w.x << 16); v[1] = __uint_as_float(w.x & 0xFFFF0000u);
            v[2] = __uint_as_float(w.y << 16); v[3] = __uint_as_float(w.y & 0xFFFF0000u);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = live && k + i < K ? to_f32(row[k + i]) : 0.0f;
    }
}

template <typename T> __global__ void __launch_bounds__(256) simt_glu_kernel(const GluArgs a, int wide_x, int wide_w) {
    constexpr bool EXACT = sizeof(T) == 4;
    __shared__ __align__(16) float xs[2][kTK][kTM + 4], ws[2][kTK][2 * kTH + 4];
    ptx::griddep_wait();
    ptx::griddep_launch_dependents();
    const int t = threadIdx.x, tx = t % 16, ty = t / 16;
    const int64_t n_tiles = (a.N + kTH - 1) / kTH;
    const int64_t m0 = blockIdx.x / n_tiles * kTM, n0 = blockIdx.x % n_tiles * kTH;
    // this thread's four elements of the X tile and of the W tile (rows 0 .. 31: gate, 32 .. 63: the other half)
    const int lr = t / 4, lk = t % 4 * 4;
    const int64_t wn = n0 + lr % kTH;
    const bool x_live = m0 + lr < a.M, w_live = wn < a.N;
    const T* xrow = (const T*)a.X + (x_live ? m0 + lr : 0) * a.ldx;
    const T* wrow = (const T*)a.W + (w_live ? wn + (lr < kTH ? 0 : a.N) : 0) * a.ldw;
    float xv[4], wv[4], g[4][2] = {}, u[4][2] = {};
    auto fetch = [&](int64_t k0) {
        load4(xv, xrow, k0 + lk, a.K, x_live, wide_x);
        load4(wv, wrow, k0 + lk, a.K, w_live, wide_w);
    };
    auto put = [&](int b) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            xs[b][lk + i][lr] = xv[i];
            ws[b][lk + i][lr] = wv[i];
        }
    };
    fetch(0);
    put(0);
    __syncthreads();
    int b = 0;
    for (int64_t k0 = 0; k0 < a.K; k0 += kTK, b ^= 1) {
        const bool more = k0 + kTK < a.K;
        if (more) fetch(k0 + kTK);
#pragma unroll
        for (int k = 0; k < kTK; ++k) {
            const float4 x4 = *reinterpret_cast<const float4*>(&xs[b][k][4 * ty]);
            const float2 g2 = *reinterpret_cast<const float2*>(&ws[b][k][2 * tx]), u2 = *reinterpret_cast<const float2*>(&ws[b][k][kTH + 2 * tx]);
            const float x[4] = {x4.x, x4.y, x4.z, x4.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                g[i][0] = fmaf(x[i], g2.x, g[i][0]);
                g[i][1] = fmaf(x[i], g2.y, g[i][1]);
                u[i][0] = fmaf(x[i], u2.x, u[i][0]);
                u[i][1] = fmaf(x[i], u2.y, u[i][1]);
            }
        }
        if (more) put(b ^ 1);
        __syncthreads();
    }
    with_act(a.act, [&](auto tag) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int64_t n = n0 + 2 * tx + j;
            if (n >= a.N) continue;
            const float bg = a.bias ? to_f32(((const T*)a.bias)[n]) : 0.0f, bu = a.bias ? to_f32(((const T*)a.bias)[a.N + n]) : 0.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int64_t m = m0 + 4 * ty + i;
                if (m >= a.M) continue;
                const float gv = g[i][j] + bg, uv = u[i][j] + bu;
                ((T*)a.out)[m * a.ldo + n] = from_f32<T>(act_value<decltype(tag)::value, EXACT>(gv) * uv);
                if (a.p_save) {
                    T* p = (T*)a.p_save + m * a.ldp + n;
                    p[0] = from_f32<T>(gv);
                    p[a.N] = from_f32<T>(uv);
                }
            }
        }
    });
}

}  // namespace

lrd_status_t gate_fwd(int64_t M, int64_t N, const void* P, int64_t ldp, void* H, int64_t ldh, int act, lrd_dtype_t dt, cudaStream_t s) {
    return run_gate<false>(GateParams{M, N, P, nullptr, H, nullptr, ldp, ldh, 0, act}, dt, s);
}

lrd_status_t gate_bwd(int64_t M, int64_t N, const void* dH, int64_t ldh, const void* P, int64_t ldp, void* dP, int64_t lddp, int act,
                      lrd_dtype_t dt, cudaStream_t s) {
    return run_gate<true>(GateParams{M, N, P, dH, nullptr, dP, ldp, ldh, lddp, act}, dt, s);
}

lrd_status_t i8_quantize(const void* X, int64_t ldx, int64_t M, int64_t K, int8_t* Xq, int64_t ldq, float* scale, lrd_dtype_t dt, cudaStream_t s) {
    if (M <= 0) return LRD_OK;
    const int vec = 16 / (int)elem_size(dt);                 // 8 or 4 elements in, as many bytes out
    const bool wide = K % vec == 0 && ldx % vec == 0 && ldq % vec == 0 && on16(X) && (uintptr_t)Xq % vec == 0;
    if (dt == LRD_BF16)
        return wide ? launch_quantize<__nv_bfloat16, 8>(X, ldx, M, K, Xq, ldq, scale, s) : launch_quantize<__nv_bfloat16, 1>(X, ldx, M, K, Xq, ldq, scale, s);
    return wide ? launch_quantize<float, 4>(X, ldx, M, K, Xq, ldq, scale, s) : launch_quantize<float, 1>(X, ldx, M, K, Xq, ldq, scale, s);
}

lrd_status_t copy2d_bytes(void* dst, int64_t ldd, const void* src, int64_t lds, int64_t rows, int64_t cols, cudaStream_t s) {
    if (rows <= 0 || cols <= 0) return LRD_OK;
    uint8_t* d = (uint8_t*)dst;
    const uint8_t* c = (const uint8_t*)src;
    void* args[] = {&d, &ldd, &c, &lds, &rows, &cols};
    return launch_pdl((const void*)copy2d_bytes_kernel, dim3((unsigned)(rows < kNumSms * 8 ? rows : kNumSms * 8)), 256, args, s) ? LRD_OK : LRD_ERR_CUDA;
}

lrd_status_t simt_glu(const GluArgs& g, cudaStream_t s) {
    if (g.M <= 0) return LRD_OK;
    const int64_t tiles = (g.M + kTM - 1) / kTM * ((g.N + kTH - 1) / kTH);
    if (tiles > 0x7FFFFFFF) return LRD_ERR_TOO_LARGE;
    const size_t four = 4 * elem_size(g.dtype);              // bytes of four elements, one access where rows start on such boundaries
    GluArgs a = g;
    int wide_x = g.ldx % 4 == 0 && (uintptr_t)g.X % four == 0, wide_w = g.ldw % 4 == 0 && (uintptr_t)g.W % four == 0;
    void* args[] = {&a, &wide_x, &wide_w};
    const void* kern = g.dtype == LRD_BF16 ? (const void*)simt_glu_kernel<__nv_bfloat16> : (const void*)simt_glu_kernel<float>;
    return launch_pdl(kern, dim3((unsigned)tiles), 256, args, s) ? LRD_OK : LRD_ERR_CUDA;
}

}  // namespace lrd
