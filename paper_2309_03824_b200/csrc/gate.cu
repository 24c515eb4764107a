// The gate of a feed-forward block on its own (element by element), rows quantized to 8 bits, and the general fp32-FMA form of the
// gated block.
#include <algorithm>
#include <cstdint>

#include "glu.cuh"
#include "ptx.cuh"
#include "tc.cuh"

namespace lrd {
namespace {

// No pointer here is __restrict__: the kernels start before the launch in front of them has ended, and what they read may be written until
// griddep_wait returns, so no load may count as one of memory that never changes.

template <typename T> __device__ __forceinline__ float to_f32(T x) { return (float)x; }
template <typename T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

struct Quad { uint32_t w[4]; };                              // 16 bytes

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
__device__ __forceinline__ Quad to_quad(const Pack<__nv_bfloat16, 8>& p) {
    Quad q;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 pair = __floats2bfloat162_rn(p.v[2 * i], p.v[2 * i + 1]);
        q.w[i] = *reinterpret_cast<const uint32_t*>(&pair);
    }
    return q;
}

// A piece: 16 bytes as they were loaded (or one element, VEC = 1)
template <typename T, int VEC> struct Raw { Quad q; };
template <typename T, int VEC> __device__ __forceinline__ Raw<T, VEC> load_raw(const T* at) {
    Raw<T, VEC> r;
    if constexpr (VEC == 1) {
        r.q.w[0] = __float_as_uint(to_f32(*at));
    } else {
        const uint4 v = *reinterpret_cast<const uint4*>(at);
        r.q = {{v.x, v.y, v.z, v.w}};
    }
    return r;
}
template <typename T, int VEC> __device__ __forceinline__ float raw_value(const Raw<T, VEC>& r, int e) {
    if constexpr (VEC == 8) return __uint_as_float(e & 1 ? r.q.w[e / 2] & 0xFFFF0000u : r.q.w[e / 2] << 16);
    else return __uint_as_float(r.q.w[e]);
}

// ---- rows that start or end off 16-byte boundaries -----------------------------------------------------------------
// A lane of a warp takes a piece of columns [c, c + 8), 16 bytes, where the row written starts such that the piece lies on a
// boundary of it; c may be below 0 or the piece may pass N.  An input's elements come from its two aligned pieces that hold them where both lie
// between the first and the last element of the whole input (`begin`, `end`: what stands outside the row is read then, and not used), else one by
// one.  bf16 only: fp32 is no faster so than element by element (4096 x 2815, us: forward 27.0 / 27.2, backward 45 / 40).
constexpr int kPiece = 8;

// The 16 bytes from byte `shift` (below 16, the same in all lanes) of two neighbouring pieces on
__device__ __forceinline__ Quad window(const Quad& a, const Quad& b, uint32_t shift) {
    uint32_t v[8] = {a.w[0], a.w[1], a.w[2], a.w[3], b.w[0], b.w[1], b.w[2], b.w[3]};
#pragma unroll
    for (int i = 0; i < 6; ++i) v[i] = shift & 8 ? v[i + 2] : v[i];
#pragma unroll
    for (int i = 0; i < 5; ++i) v[i] = shift & 4 ? v[i + 1] : v[i];
    Quad q;
#pragma unroll
    for (int i = 0; i < 4; ++i) q.w[i] = __funnelshift_r(v[i], v[i + 1], 8 * (shift & 3));
    return q;
}
__device__ __forceinline__ Quad load_loose(const __nv_bfloat16* row, int64_t c, int64_t N, const __nv_bfloat16* begin, const __nv_bfloat16* end) {
    constexpr int E = kPiece;
    Quad q = {};
    const uint32_t shift = (uint32_t)(uintptr_t)(row + c) & 15;
    const uintptr_t from = (uintptr_t)(row + c) - shift;
    if (from >= (uintptr_t)begin && from + 32 <= (uintptr_t)end) {
        const uint4* at = reinterpret_cast<const uint4*>(from);
        const uint4 a = at[0];
        q = {{a.x, a.y, a.z, a.w}};
        if (shift) {
            const uint4 b = at[1];
            q = window(q, {{b.x, b.y, b.z, b.w}}, shift);
        }
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (c + e >= 0 && c + e < N)
                q.w[e / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(row)[c + e] << (16 * (e & 1));
    }
    return q;
}
__device__ __forceinline__ void store_element(__nv_bfloat16* row, int64_t c, const Quad& q, int e) {
    reinterpret_cast<uint16_t*>(row)[c + e] = (uint16_t)(q.w[e / 2] >> (16 * (e & 1)));
}
__device__ __forceinline__ void store_quad(__nv_bfloat16* at, const Quad& q) { *reinterpret_cast<uint4*>(at) = make_uint4(q.w[0], q.w[1], q.w[2], q.w[3]); }
// a piece on a boundary
__device__ __forceinline__ void store_whole(__nv_bfloat16* row, int64_t c, int64_t N, const Quad& q) {
    if (c >= 0 && c + kPiece <= N) {
        store_quad(row + c, q);
        return;
    }
#pragma unroll
    for (int e = 0; e < kPiece; ++e)
        if (c + e >= 0 && c + e < N) store_element(row, c, q, e);
}
// Pieces off the boundaries, of a warp whose lanes hold neighbouring ones: 16 bytes from a lane's boundary on, the next lane's first elements
// among them, where both pieces lie inside the row; what no such store takes goes element by element.  All lanes call.
__device__ __forceinline__ void store_across(__nv_bfloat16* row, int64_t c, int64_t N, const Quad& q) {
    constexpr int E = kPiece;
    const uint32_t shift = (uint32_t)(-(uintptr_t)(row + c)) & 15;       // (the same in all lanes)
    if (shift == 0) {
        store_whole(row, c, N, q);
        return;
    }
    const int lane = threadIdx.x & 31, first = (int)(shift / 2);
    Quad next;
#pragma unroll
    for (int i = 0; i < 4; ++i) next.w[i] = __shfl_down_sync(0xffffffffu, q.w[i], 1);
    const bool mine = lane < 31 && c >= 0 && c + 2 * E <= N, before = lane > 0 && c >= E && c + E <= N;
    if (mine) store_quad(row + c + first, window(q, next, shift));
    if (__all_sync(0xffffffffu, c >= 0 && c + E <= N)) {     // left: the first lane's first elements, the last lane's others, one each for E lanes
        const int from = lane < first ? 0 : 31;
        Quad end;
#pragma unroll
        for (int i = 0; i < 4; ++i) end.w[i] = __shfl_sync(0xffffffffu, q.w[i], from);
        uint32_t word = end.w[0];
#pragma unroll
        for (int i = 1; i < 4; ++i) word = lane / 2 == i ? end.w[i] : word;
        if (lane >= E) return;
        __nv_bfloat16* at = row + (c - lane * E) + from * E + lane;
        *reinterpret_cast<uint16_t*>(at) = (uint16_t)(word >> (16 * (lane & 1)));
        return;
    }
    if (mine && before) return;
#pragma unroll
    for (int e = 0; e < E; ++e)
        if (c + e >= 0 && c + e < N && !(e < first ? before : mine)) store_element(row, c, q, e);
}

struct GateParams {
    int64_t M, N;
    const void *P, *dH;
    void *H, *dP;
    int64_t ldp, ldh, lddp;
    int act;
};

// BWD = false: H = act(G) * U.  BWD = true: dP = [dH * U * act'(G) | dH * act(G)].  Bound by memory: 3 or 5 elements move for each of
// H, in 16-byte accesses where bases, strides and N allow, else (short rows, fp32) one element at a time and four in flight.  A block's threads stand as
// 256 / tx rows of tx, so that a thread finds its row once for all its pieces, DEPTH of them tx apart.  P and dP may be the same memory: a
// thread reads both halves' pieces before it writes them, and no other thread touches those.
template <typename T, int VEC, bool BWD, int ACT>
__global__ void __launch_bounds__(256) gate_kernel(const GateParams p, int log_tx, uint32_t spans, uint32_t across) {
    constexpr bool EXACT = sizeof(T) == 4;
    constexpr int DEPTH = VEC == 1 ? 4 : 1;
    ptx::griddep_wait();
    ptx::griddep_launch_dependents();
    const int tx = 1 << log_tx, ty = 256 >> log_tx;
    // a span: ty rows x (tx DEPTH) pieces, `across` of them side by side; blocks walk over them, across the columns first
    for (uint32_t s = blockIdx.x; s < spans; s += gridDim.x) {
        const uint32_t down = s / across;
        const int64_t row = (int64_t)down * ty + (threadIdx.x >> log_tx), piece0 = (int64_t)(s - down * across) * (tx * DEPTH) + (threadIdx.x & (tx - 1));
        if (row >= p.M) continue;
        const T *P = (const T*)p.P + row * p.ldp, *dH = BWD ? (const T*)p.dH + row * p.ldh : nullptr;
        T* to = BWD ? (T*)p.dP + row * p.lddp : (T*)p.H + row * p.ldh;
        Pack<T, VEC> g[DEPTH], u[DEPTH], d[DEPTH];
#pragma unroll
        for (int i = 0; i < DEPTH; ++i) {
            const int64_t c = (piece0 + tx * i) * VEC;
            if (c >= p.N) break;
            load_pack(g[i], P + c);
            load_pack(u[i], P + p.N + c);
            if (BWD) load_pack(d[i], dH + c);
        }
#pragma unroll
        for (int i = 0; i < DEPTH; ++i) {
            const int64_t c = (piece0 + tx * i) * VEC;
            if (c >= p.N) break;
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
            store_pack(to + c, g[i]);
            if (BWD) store_pack(to + p.N + c, u[i]);
        }
    }
}

// The same over rows off 16-byte boundaries: in the pieces of the row of H, or of dP's first half.
template <bool BWD, int ACT> __global__ void __launch_bounds__(256) gate_loose_kernel(const GateParams p, uint32_t spans, uint32_t across) {
    using T = __nv_bfloat16;
    constexpr bool EXACT = false;
    constexpr int E = kPiece;
    ptx::griddep_wait();
    ptx::griddep_launch_dependents();
    // a span: eight rows, one a warp, x 32 pieces
    for (uint32_t s = blockIdx.x; s < spans; s += gridDim.x) {
        const uint32_t down = s / across;
        const int64_t row = (int64_t)down * 8 + threadIdx.x / 32;
        if (row >= p.M) continue;
        const T *P = (const T*)p.P + row * p.ldp, *dH = BWD ? (const T*)p.dH + row * p.ldh : nullptr;
        T* to = BWD ? (T*)p.dP + row * p.lddp : (T*)p.H + row * p.ldh;
        const int head = (int)((-(uintptr_t)to & 15) / sizeof(T));
        const int64_t c = ((int64_t)(s - down * across) * 32 + (threadIdx.x & 31)) * E + (head ? head - E : 0);
        const T *endP = (const T*)p.P + (p.M - 1) * p.ldp + 2 * p.N, *enddH = (const T*)p.dH + (p.M - 1) * p.ldh + p.N;
        const Raw<T, E> g{load_loose(P, c, p.N, (const T*)p.P, endP)}, u{load_loose(P + p.N, c, p.N, (const T*)p.P, endP)};
        const Raw<T, E> d{BWD ? load_loose(dH, c, p.N, (const T*)p.dH, enddH) : Quad{}};
        Pack<T, E> a, b;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if (!BWD) {
                a.v[e] = act_value<ACT, EXACT>(raw_value<T, E>(g, e)) * raw_value<T, E>(u, e);
            } else {
                float value, slope;
                act_both<ACT, EXACT>(raw_value<T, E>(g, e), value, slope);
                a.v[e] = raw_value<T, E>(d, e) * raw_value<T, E>(u, e) * slope;
                b.v[e] = raw_value<T, E>(d, e) * value;
            }
        }
        store_whole(to, c, p.N, to_quad(a));
        if (BWD) store_across(to + p.N, c, p.N, to_quad(b));
    }
}

// The same backward pass with the column sums of dP (before its rounding) on the way: a block takes 32 pieces of columns and a chunk of
// rows, eight rows at a time, so that a thread's columns stay its own; the eight threads of a column are added in shared memory
// and each chunk leaves one partial sum per column, added in order by column_sums_kernel: the same bits every time.  (As a
// by-product of dW they cost an MMA against ones for every k-block of every tile of a column: 200 of 1350 us at 8192 x 4096 -> 2 x 10752.)
constexpr int kSumCols = 32, kSumRows = 8;
// LOOSE: dP's rows are on 16-byte boundaries, other rows or dP's second half are not.
template <int VEC, bool LOOSE, int ACT>
__global__ void __launch_bounds__(256, 3) gate_bwd_sums_kernel(const GateParams p, float* partial, int64_t rows_per_chunk) {
    using T = __nv_bfloat16;
    constexpr bool EXACT = false;
    constexpr int DEPTH = VEC == 1 ? 4 : LOOSE ? 1 : 2;      // rows of a thread in flight
    __shared__ float sums[kSumRows][kSumCols * VEC + 1];
    ptx::griddep_wait();
    ptx::griddep_launch_dependents();
    const int tx = threadIdx.x % kSumCols, ty = threadIdx.x / kSumCols;
    const int64_t col = ((int64_t)blockIdx.x * kSumCols + tx) * VEC, first = (int64_t)blockIdx.y * rows_per_chunk;
    const int64_t last = first + rows_per_chunk < p.M ? first + rows_per_chunk : p.M;
    const bool live = LOOSE || col < p.N;                    // (LOOSE: a warp's lanes pass elements on)
    float sum_g[VEC] = {}, sum_u[VEC] = {};
    for (int64_t r0 = first + ty; r0 < last && live; r0 += kSumRows * DEPTH) {
        Raw<T, VEC> g[DEPTH], u[DEPTH], d[DEPTH];
#pragma unroll
        for (int i = 0; i < DEPTH; ++i) {
            const int64_t row = r0 + kSumRows * i;
            if (row >= last) break;
            const T *at = (const T*)p.P + row * p.ldp, *dh = (const T*)p.dH + row * p.ldh;
            if constexpr (LOOSE) {
                const T *endP = (const T*)p.P + (p.M - 1) * p.ldp + 2 * p.N, *enddH = (const T*)p.dH + (p.M - 1) * p.ldh + p.N;
                g[i].q = load_loose(at, col, p.N, (const T*)p.P, endP);
                u[i].q = load_loose(at + p.N, col, p.N, (const T*)p.P, endP);
                d[i].q = load_loose(dh, col, p.N, (const T*)p.dH, enddH);
            } else {
                g[i] = load_raw<T, VEC>(at + col);
                u[i] = load_raw<T, VEC>(at + p.N + col);
                d[i] = load_raw<T, VEC>(dh + col);
            }
        }
#pragma unroll
        for (int i = 0; i < DEPTH; ++i) {
            const int64_t row = r0 + kSumRows * i;
            if (row >= last) break;
            Pack<T, VEC> dg, du;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                float value, slope;
                act_both<ACT, EXACT>(raw_value<T, VEC>(g[i], e), value, slope);
                dg.v[e] = raw_value<T, VEC>(d[i], e) * raw_value<T, VEC>(u[i], e) * slope;
                du.v[e] = raw_value<T, VEC>(d[i], e) * value;
                sum_g[e] += dg.v[e];
                sum_u[e] += du.v[e];
            }
            T* to = (T*)p.dP + row * p.lddp;
            if constexpr (LOOSE) {
                store_whole(to, col, p.N, to_quad(dg));
                store_across(to + p.N, col, p.N, to_quad(du));
            } else {
                store_pack(to + col, dg);
                store_pack(to + p.N + col, du);
            }
        }
    }
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < VEC; ++e) sums[ty][tx * VEC + e] = half ? sum_u[e] : sum_g[e];
        __syncthreads();
        for (int c = threadIdx.x; c < kSumCols * VEC; c += 256) {
            const int64_t n = (int64_t)blockIdx.x * kSumCols * VEC + c;
            if (n >= p.N) continue;
            float s = 0.0f;
#pragma unroll
            for (int r = 0; r < kSumRows; ++r) s += sums[r][c];
            partial[(int64_t)blockIdx.y * 2 * p.N + half * p.N + n] = s;
        }
    }
}
// 32 columns a block, the chunks dealt out to its eight rows of threads: few loads stand one behind another
template <typename T> __global__ void __launch_bounds__(256) column_sums_kernel(const float* partial, int64_t chunks, int64_t n, T* out) {
    __shared__ float sums[kSumRows][kSumCols];
    ptx::griddep_wait();
    ptx::griddep_launch_dependents();
    const int tx = threadIdx.x % kSumCols, ty = threadIdx.x / kSumCols;
    const int64_t c = (int64_t)blockIdx.x * kSumCols + tx;
    float s = 0.0f;
    if (c < n)
#pragma unroll 8
        for (int64_t i = ty; i < chunks; i += kSumRows) s += partial[i * n + c];
    sums[ty][tx] = s;
    __syncthreads();
    if (ty || c >= n) return;
#pragma unroll
    for (int r = 1; r < kSumRows; ++r) s += sums[r][tx];
    out[c] = from_f32<T>(s);
}

bool launch_pdl(const void* kern, dim3 grid, unsigned threads, void** args, cudaStream_t s, size_t smem = 0) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads, 1, 1);
    cfg.dynamicSmemBytes = smem;
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
    // as many threads side by side as a row has use for, 8 to 256; at most 16 blocks for each SM, which walk over what is left
    const int64_t pieces = p.N / VEC, depth = VEC == 1 ? 4 : 1;
    int log_tx = 3;
    while (log_tx < 8 && ((int64_t)1 << log_tx) * depth < pieces) ++log_tx;
    const int64_t rows = 256 >> log_tx, wide = (pieces + (depth << log_tx) - 1) / (depth << log_tx), all = (p.M + rows - 1) / rows * wide;
    if (all > 0x7FFFFFFF) return LRD_ERR_TOO_LARGE;          // (over 10^12 elements)
    GateParams q = p;
    uint32_t spans = (uint32_t)all, across = (uint32_t)wide;
    void* args[] = {&q, &log_tx, &spans, &across};
    return launch_pdl((const void*)kern, dim3((unsigned)(spans < kNumSms * 16 ? spans : kNumSms * 16)), 256, args, s) ? LRD_OK : LRD_ERR_CUDA;
}

bool on16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

template <int VEC, bool LOOSE> lrd_status_t launch_gate_sums(const GateParams& p, float* partial, __nv_bfloat16* sums, cudaStream_t s) {
    auto kern = p.act == LRD_ACT_SILU ? gate_bwd_sums_kernel<VEC, LOOSE, LRD_ACT_SILU>
              : p.act == LRD_ACT_GELU ? gate_bwd_sums_kernel<VEC, LOOSE, LRD_ACT_GELU> : gate_bwd_sums_kernel<VEC, LOOSE, LRD_ACT_GELU_TANH>;
    GateParams q = p;
    int64_t chunks = gate_sum_chunks(p.M, p.N), n = 2 * p.N;
    if (VEC == 1) chunks = std::min(chunks, (p.M + 63) / 64);     // (a thread then takes 32 rows at once, and the columns make more blocks)
    int64_t rows = (p.M + chunks - 1) / chunks;
    chunks = (p.M + rows - 1) / rows;
    void* args[] = {&q, &partial, &rows};
    const int64_t blocks = (p.N + kSumCols * VEC - 1) / (kSumCols * VEC);
    if (!launch_pdl((const void*)kern, dim3((unsigned)blocks, (unsigned)chunks), 256, args, s)) return LRD_ERR_CUDA;
    const float* from = partial;
    void* more[] = {&from, &chunks, &n, &sums};
    return launch_pdl((const void*)column_sums_kernel<__nv_bfloat16>, dim3((unsigned)((n + kSumCols - 1) / kSumCols)), 256, more, s) ? LRD_OK : LRD_ERR_CUDA;
}

template <bool BWD> lrd_status_t launch_gate_loose(const GateParams& p, cudaStream_t s) {
    auto kern = p.act == LRD_ACT_SILU ? gate_loose_kernel<BWD, LRD_ACT_SILU>
              : p.act == LRD_ACT_GELU ? gate_loose_kernel<BWD, LRD_ACT_GELU> : gate_loose_kernel<BWD, LRD_ACT_GELU_TANH>;
    // a row's pieces may start one below its first element and end one past its last
    const int64_t pieces = (p.N + 2 * kPiece - 2) / kPiece, wide = (pieces + 31) / 32, all = (p.M + 7) / 8 * wide;
    if (all > 0x7FFFFFFF) return LRD_ERR_TOO_LARGE;          // (over 10^12 elements)
    GateParams q = p;
    uint32_t spans = (uint32_t)all, across = (uint32_t)wide;
    void* args[] = {&q, &spans, &across};
    return launch_pdl((const void*)kern, dim3((unsigned)(spans < kNumSms * 16 ? spans : kNumSms * 16)), 256, args, s) ? LRD_OK : LRD_ERR_CUDA;
}

bool bwd_wide(const GateParams& p, int vec) {
    return p.N % vec == 0 && p.ldp % vec == 0 && p.ldh % vec == 0 && p.lddp % vec == 0 && on16(p.P) && on16(p.dH) && on16(p.dP);
}

// Rows of bf16 off the boundaries, element by element / in pieces, us: forward 8192 x 4095 97 / 41, 2748 x 2681 25.7 / 11.4, 8192 x 511 15.0 / 9.6,
// 8192 x 255 6.4 / 7.0; backward 8192 x 4095 107 / 78, 1021 x 2731 12.8 / 9.9, 8192 x 1023 29.5 / 25.9, 8192 x 511 15.5 / 17.0,
// 512 x 1535 4.1 / 4.8.  With the sums, backward passes of whole blocks: 4096 x 1024 -> 2 x 2815 138 / 110, 2413 x 592 -> 2 x 515 22.5 / 26.5.
bool loose_best(int64_t M, int64_t N, bool bwd) { return bwd ? N >= 768 && M * N >= (1 << 21) : N >= 384; }

template <bool BWD> lrd_status_t run_gate(const GateParams& p, lrd_dtype_t dt, cudaStream_t s) {
    if (p.M <= 0) return LRD_OK;
    const int vec = 16 / (int)elem_size(dt);
    const bool wide = BWD ? bwd_wide(p, vec) : p.N % vec == 0 && p.ldp % vec == 0 && p.ldh % vec == 0 && on16(p.P) && on16(p.H);
    if (!wide && dt == LRD_BF16 && loose_best(p.M, p.N, BWD)) return launch_gate_loose<BWD>(p, s);
    if (dt == LRD_BF16) return wide ? launch_gate<__nv_bfloat16, 8, BWD>(p, s) : launch_gate<__nv_bfloat16, 1, BWD>(p, s);
    return wide ? launch_gate<float, 4, BWD>(p, s) : launch_gate<float, 1, BWD>(p, s);
}

// ---- rows to 8 bits -----------------------------------------------------------------------------------------------
// scale = max |x| fl(1 / 127), q = x / scale rounded to the nearest integer, ties to even: of the real quotient, not of a
// rounded one.  fma(x, 1 / scale, 1.5 2^23) holds an integer in its low bits that is off by one step at most; the remainder
// x - q scale, which an fma forms exactly (x and q scale are multiples of the last place of either, and no more than some scale
// apart), then says whether it is the nearest.  (In bf16 quotients within 2^-23 of a border are nothing rare: 8192 x 4096 took 43 to 55 us
// with a branch that did those over.)
// PARITY: quotients that lie on a border exactly need the even one of the two.  With bf16 rows the scale is then a power of two (it is
// the largest value, 8 bits, times fl(1 / 127); of all such products only powers of two are a 2 / (2 n + 1) of an 8-bit number), its
// reciprocal exact, and the fma has rounded to even already.
struct RowScale { float scale, inv, half, past_half; };      // past_half: the next fp32 number after scale / 2
constexpr float kRound = 12582912.0f;                        // 1.5 2^23
template <bool PARITY> __device__ __forceinline__ uint32_t to_nearest(uint32_t q, float rest, const RowScale& r) {
    if (PARITY ? fabsf(rest) >= (q & 1u ? r.half : r.past_half) : fabsf(rest) > r.half) q += (uint32_t)((__float_as_int(rest) >> 31) | 1);
    return q;                                                // (the low byte)
}
template <bool PARITY> __device__ __forceinline__ uint32_t quantize_one(float x, const RowScale& r) {
    const float t = fmaf(x, r.inv, kRound);
    return to_nearest<PARITY>(__float_as_uint(t), fmaf(kRound - t, r.scale, x), r);
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

// largest |x| so far, by its bits (infinities and NaN are above every number); of bf16 pairs, both halves side by side
template <typename T, int VEC> __device__ __forceinline__ void raw_top(uint32_t& top, const Raw<T, VEC>& r) {
    if constexpr (VEC == 8) {
#pragma unroll
        for (int i = 0; i < 4; ++i) top = __vmaxu2(top, r.q.w[i] & 0x7FFF7FFFu);
    } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) top = max(top, r.q.w[i] & 0x7FFFFFFFu);
    }
}

// A row's elements by `TPR` threads, a piece at a time; the first KEEP pieces of a thread stay in registers between the two passes,
// longer rows are read again (from L2).  Bound by memory.
template <typename T, int VEC, int TPR, int KEEP>
__global__ void __launch_bounds__(256) i8_quantize_kernel(const T* X, int64_t ldx, int64_t M, int64_t K, int8_t* Xq, int64_t ldq, float* scale_out) {
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
#pragma unroll 4
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
        if constexpr (VEC == 1) {
            b[0] = quantize_one<sizeof(T) == 4>(raw_value<T, VEC>(v, 0), r);
        } else {
            // quantize_one's first half two at a time; its second only where one of the remainders asks for it
            const uint64_t inv2 = pair_both(r.inv), scale2 = pair_both(r.scale), round2 = pair_both(kRound);
            float rest[VEC], far = 0.0f;
#pragma unroll
            for (int e = 0; e < VEC; e += 2) {
                const uint64_t x = pair_of(raw_value<T, VEC>(v, e), raw_value<T, VEC>(v, e + 1)), q2 = pair_fma(x, inv2, round2);
                pair_split(pair_fma(pair_fma(q2, pair_both(-1.0f), round2), scale2, x), rest[e], rest[e + 1]);
                b[e] = (uint32_t)q2;
                b[e + 1] = (uint32_t)(q2 >> 32);
                far = fmaxf(far, fmaxf(fabsf(rest[e]), fabsf(rest[e + 1])));
            }
            if (sizeof(T) == 4 ? far >= r.half : far > r.half) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) b[e] = to_nearest<sizeof(T) == 4>(b[e], rest[e], r);
            }
        }
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
    // (loads ahead of stores, which X and Xq being any memory keeps the compiler from: 512 x 65536 in fp32 61 us without)
    constexpr int AHEAD = VEC == 1 ? 8 : 4;
    for (int64_t at = t + (int64_t)KEEP * TPR; at < pieces; at += AHEAD * TPR) {
        Raw<T, VEC> r[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
            if (at + i * TPR < pieces) r[i] = load_raw<T, VEC>(x + (at + i * TPR) * VEC);
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
            if (at + i * TPR < pieces) put(r[i], at + i * TPR);
    }
}

template <typename T, int VEC, int TPR, int KEEP>
lrd_status_t launch_quantize_as(const T* x, int64_t ldx, int64_t M, int64_t K, int8_t* Xq, int64_t ldq, float* scale, cudaStream_t s) {
    void* args[] = {&x, &ldx, &M, &K, &Xq, &ldq, &scale};
    const int64_t rows = 256 / TPR;
    return launch_pdl((const void*)i8_quantize_kernel<T, VEC, TPR, KEEP>, dim3((unsigned)((M + rows - 1) / rows)), 256, args, s) ? LRD_OK : LRD_ERR_CUDA;
}
// Rows of any alignment and length, up to kLooseBytes of them, through shared memory: 16 bytes at a time from the first boundary in the row
// to the last, what stands before and behind element by element, and eight results at a time out of shared memory, whose elements then need
// no boundary (8192 x 4095 in bf16, every access of one element: 67 us).
constexpr size_t kLooseBytes = 40 << 10;
template <typename T>
__global__ void __launch_bounds__(256) i8_quantize_loose_kernel(const T* X, int64_t ldx, int64_t M, int K, int8_t* Xq, int64_t ldq, float* scale_out) {
    constexpr int TPR = 256, VEC = 16 / (int)sizeof(T);
    extern __shared__ __align__(16) uint8_t loose_smem[];
    __shared__ uint32_t part[8];
    ptx::griddep_wait();
    ptx::griddep_launch_dependents();
    const int t = threadIdx.x;
    const int64_t row = blockIdx.x;
    const T* x = X + row * ldx;
    const int head = min(K, (int)((16u - (uint32_t)((uintptr_t)x & 15u)) & 15u) / (int)sizeof(T)), body = (K - head) / VEC;
    T* const at = reinterpret_cast<T*>(loose_smem) + (VEC - head) % VEC;     // element 0; the body then starts on 16 bytes
    uint32_t top = 0;
    auto see = [&](float v) { top = max(top, __float_as_uint(v) & 0x7FFFFFFFu); };
#pragma unroll 4
    for (int i = t; i < body; i += TPR) {
        const Raw<T, VEC> r = load_raw<T, VEC>(x + head + i * VEC);
#pragma unroll
        for (int e = 0; e < VEC; ++e) see(raw_value<T, VEC>(r, e));
        *reinterpret_cast<uint4*>(at + head + i * VEC) = make_uint4(r.q.w[0], r.q.w[1], r.q.w[2], r.q.w[3]);
    }
    const int loose = K - body * VEC;                        // before the body, then behind it
    for (int i = t; i < loose; i += TPR) {
        const int k = i < head ? i : body * VEC + i;
        const T v = x[k];
        at[k] = v;
        see(to_f32(v));
    }
    top = __reduce_max_sync(0xffffffffu, top);
    if (t % 32 == 0) part[t / 32] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 8; ++w) top = max(top, part[w]);
    const float scale = top < 0x7F800000u ? __uint_as_float(top) * (1.0f / 127.0f) : __uint_as_float(0x7FC00000u);
    if (t == 0) scale_out[row] = scale;
    int8_t* q = Xq + row * ldq;
    if (!(scale >= 7.888609e-31f)) {                         // 2^-100; NaN
        quantize_odd_row(x, q, (int64_t)K, scale, t, TPR);
        return;
    }
    const float half = 0.5f * scale;
    const RowScale r{scale, 1.0f / scale, half, __uint_as_float(__float_as_uint(half) + 1u)};
    // eight results a thread and step, from a boundary of the row of results on; those before the first and behind the last one by one
    const int q_head = (int)(-(uintptr_t)q & 7);
    for (int first = (q_head ? q_head - 8 : 0) + t * 8; first < K; first += TPR * 8) {
        uint32_t b[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) b[e] = first + e >= 0 && first + e < K ? quantize_one<sizeof(T) == 4>(to_f32(at[first + e]), r) : 0u;
        if (first >= 0 && first + 8 <= K) {
            uint32_t w[2];
#pragma unroll
            for (int i = 0; i < 2; ++i)
                w[i] = __byte_perm(__byte_perm(b[4 * i], b[4 * i + 1], 0x0040), __byte_perm(b[4 * i + 2], b[4 * i + 3], 0x0040), 0x5410);
            *reinterpret_cast<uint2*>(q + first) = make_uint2(w[0], w[1]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (first + e >= 0 && first + e < K) q[first + e] = (int8_t)b[e];
        }
    }
}
template <typename T> lrd_status_t launch_quantize_loose(const T* x, int64_t ldx, int64_t M, int64_t K, int8_t* Xq, int64_t ldq, float* scale, cudaStream_t s) {
    int k = (int)K;
    void* args[] = {&x, &ldx, &M, &k, &Xq, &ldq, &scale};
    const size_t smem = (size_t)(K * sizeof(T) + 31) / 16 * 16;        // (the row, up to 15 bytes on)
    return launch_pdl((const void*)i8_quantize_loose_kernel<T>, dim3((unsigned)M), 256, args, s, smem) ? LRD_OK : LRD_ERR_CUDA;
}

template <typename T, int VEC> lrd_status_t launch_quantize(const void* X, int64_t ldx, int64_t M, int64_t K, int8_t* Xq, int64_t ldq, float* scale, cudaStream_t s) {
    const T* x = (const T*)X;
    if constexpr (VEC == 1) {
        // (4093 x 1023 in fp32: 9.0 us in registers, 14.6 through shared memory; 8192 x 4095 in bf16 67 and 40)
        if (K > 1024 && K * sizeof(T) <= kLooseBytes) return launch_quantize_loose(x, ldx, M, K, Xq, ldq, scale, s);
    }
    // as few threads a row as hold it in four pieces each (eight past a block of them)
    if (K <= 32 * 4 * VEC) return launch_quantize_as<T, VEC, 32, 4>(x, ldx, M, K, Xq, ldq, scale, s);
    if (K <= 64 * 4 * VEC) return launch_quantize_as<T, VEC, 64, 4>(x, ldx, M, K, Xq, ldq, scale, s);
    if (K <= 128 * 4 * VEC) return launch_quantize_as<T, VEC, 128, 4>(x, ldx, M, K, Xq, ldq, scale, s);
    return K <= 256 * 4 * VEC ? launch_quantize_as<T, VEC, 256, 4>(x, ldx, M, K, Xq, ldq, scale, s) : launch_quantize_as<T, VEC, 256, 8>(x, ldx, M, K, Xq, ldq, scale, s);
}

// ---- rows copied to 16-byte boundaries -----------------------------------------------------------------------------
// A warp takes up to 128 pieces of a row where it is written: each from its two aligned pieces of the source where both lie between the
// source's first and last byte, else byte by byte.  Byte by byte throughout, whole 8-bit products, us: 7525 x 5847 -> 512 59.4 / 41.3 so,
// 3688 x 767 -> 2688 23.2 / 18.0, 4103 x 1224 -> 1280 26.9 / 22.0.
struct RowCopies { RowCopy job[2]; int64_t first[3]; int n; };
__global__ void __launch_bounds__(256) rows_to_boundaries_kernel(const __grid_constant__ RowCopies b) {
    constexpr int DEPTH = 4;
    ptx::griddep_wait();
    ptx::griddep_launch_dependents();
    const int lane = threadIdx.x & 31;
    for (int64_t unit = (int64_t)blockIdx.x * 8 + threadIdx.x / 32; unit < b.first[b.n]; unit += (int64_t)gridDim.x * 8) {
        const int j = b.n > 1 && unit >= b.first[1];
        const RowCopy& job = b.job[j];
        const int64_t row = (unit - b.first[j]) / job.units, c0 = ((unit - b.first[j] - row * job.units) * 32 * DEPTH + lane) * 16;
        const uint8_t *src = (const uint8_t*)job.src + row * job.lds, *begin = (const uint8_t*)job.src, *end = begin + (job.rows - 1) * job.lds + job.bytes;
        uint8_t* dst = (uint8_t*)job.dst + row * job.ldd;
        Quad v[DEPTH];
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            const int64_t c = c0 + d * 512;
            v[d] = Quad{};
            if (c >= job.bytes) continue;
            const uint32_t shift = (uint32_t)(uintptr_t)(src + c) & 15;
            const uintptr_t from = (uintptr_t)(src + c) - shift;
            if (from >= (uintptr_t)begin && from + 32 <= (uintptr_t)end) {
                const uint4 lo = reinterpret_cast<const uint4*>(from)[0];
                v[d] = {{lo.x, lo.y, lo.z, lo.w}};
                if (shift) {
                    const uint4 hi = reinterpret_cast<const uint4*>(from)[1];
                    v[d] = window(v[d], {{hi.x, hi.y, hi.z, hi.w}}, shift);
                }
            } else {
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (c + e < job.bytes) v[d].w[e / 4] |= (uint32_t)src[c + e] << (8 * (e & 3));
            }
        }
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            const int64_t c = c0 + d * 512;
            if (c >= job.bytes) break;
            if (c + 16 > job.bytes)                          // zeros behind the row
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int64_t left = job.bytes - c - 4 * i;
                    v[d].w[i] = left >= 4 ? v[d].w[i] : left <= 0 ? 0u : v[d].w[i] & ((1u << (8 * (int)left)) - 1);
                }
            *reinterpret_cast<uint4*>(dst + c) = make_uint4(v[d].w[0], v[d].w[1], v[d].w[2], v[d].w[3]);
        }
    }
}

// ---- the gated block in fp32 FMA ----------------------------------------------------------------------------------
// A block forms TM rows x 32 columns of H: TM rows of X against 32 rows of the gate's and 32 of the other half's weights, 32 deep
// at a time, the next tile on its way in registers.  A lane gets four bytes of shared memory a clock, the SM 128 products: a thread
// holds 8 rows x 4 columns of G and of U, 64 products for 16 values read (4 rows: 12 for 32, bound by shared memory).  A tile then
// takes TM threads only; the block's 256 / TM such groups take a share of each tile's depth each and leave their sums in
// shared memory, where all threads add them up and apply the gate.  Tiles stand as they come, a row's 32 elements side by side and 4
// more between rows; a thread's rows and columns lie TM / 8 and 8 apart, so that a warp's reads never meet in a bank.
// fp32 rows on 16-byte boundaries are copied into shared memory directly, two tiles of 64 deep ahead of the one at work; others pass through registers,
// one tile ahead (1024 x 1024 -> 2048 in fp32: 250 us that way).
constexpr int kTH = 32, kSumStride = 2 * kTH + 8;
template <int TM, bool ASYNC> constexpr size_t simt_glu_smem() {
    const size_t tiles = (ASYNC ? 3 : 2) * (TM + 2 * kTH) * (ASYNC ? 68 : 36) * sizeof(float), sums = (size_t)256 * kSumStride * sizeof(float);
    return tiles > sums ? tiles : sums;
}
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

__device__ __forceinline__ void copy16_async(float* to, const float* from, int64_t left) {     // `left`: elements that exist from there on
    const int bytes = left >= 4 ? 16 : left > 0 ? (int)left * 4 : 0;                          // (the rest reads as zero)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(ptx::smem_u32(to)), "l"(from), "r"(bytes) : "memory");
}
template <typename T, int TM, bool ASYNC> __global__ void __launch_bounds__(256, 2) simt_glu_kernel(const GluArgs a, int wide_x, int wide_w) {
    constexpr bool EXACT = sizeof(T) == 4;
    constexpr int kTK = ASYNC ? 64 : 32, kRowStride = kTK + 4;       // depth of a tile, elements from row to row of it
    constexpr int GROUPS = 256 / TM, DEPTH = kTK / GROUPS, TY = TM / 8;
    constexpr int XPARTS = (TM + 31) / 32, XROWS = TM < 32 ? TM : 32;      // passes of all threads over X's rows, rows of a pass
    constexpr int TILE = (TM + 2 * kTH) * kRowStride;
    extern __shared__ __align__(16) float simt_smem[];
    ptx::griddep_wait();
    ptx::griddep_launch_dependents();
    const int t = threadIdx.x, group = t / TM, tx = t % 8, ty = t % TM / 8;
    const int64_t n_tiles = (a.N + kTH - 1) / kTH;
    const int64_t m0 = blockIdx.x / n_tiles * TM, n0 = blockIdx.x % n_tiles * kTH;
    // this thread's four elements of each of 32 rows of the X tile, of the gate's and of the other half's rows
    const int lr = t / 8, lk = t % 8 * 4;
    const bool w_live = n0 + lr < a.N;
    const T* grow = (const T*)a.W + (w_live ? n0 + lr : 0) * a.ldw;
    const T* urow = grow + a.N * a.ldw;
    float xv[XPARTS][4], gv4[4], uv4[4], g[8][4] = {}, u[8][4] = {};
    auto fetch = [&](int64_t k0) {
#pragma unroll
        for (int i = 0; i < XPARTS; ++i) {
            const int64_t m = m0 + lr + 32 * i;
            const bool live = lr < XROWS && m < a.M;
            load4(xv[i], (const T*)a.X + (live ? m : 0) * a.ldx, k0 + lk, a.K, live, wide_x);
        }
        load4(gv4, grow, k0 + lk, a.K, w_live, wide_w);
        load4(uv4, urow, k0 + lk, a.K, w_live, wide_w);
    };
    auto put = [&](float* tile) {
        auto row = [&](int r, const float (&v)[4]) { *reinterpret_cast<float4*>(tile + r * kRowStride + lk) = make_float4(v[0], v[1], v[2], v[3]); };
#pragma unroll
        for (int i = 0; i < XPARTS; ++i)
            if (lr < XROWS) row(lr + 32 * i, xv[i]);
        row(TM + lr, gv4);
        row(TM + kTH + lr, uv4);
    };
    constexpr int STAGES = ASYNC ? 3 : 2;
    auto copy = [&](int64_t k0, float* tile) {               // (ASYNC) one group each time, an empty one past the end
        if constexpr (ASYNC) {
#pragma unroll
            for (int at = lk; at < kTK && k0 < a.K; at += 32) {
                const int64_t k = k0 + at < a.K ? k0 + at : 0, left = a.K - (k0 + at);
#pragma unroll
                for (int i = 0; i < XPARTS; ++i) {
                    const int64_t m = m0 + lr + 32 * i;
                    const bool live = m < a.M;
                    if (lr < XROWS) copy16_async(tile + (lr + 32 * i) * kRowStride + at, (const float*)a.X + (live ? m : 0) * a.ldx + k, live ? left : 0);
                }
                copy16_async(tile + (TM + lr) * kRowStride + at, (const float*)grow + k, w_live ? left : 0);
                copy16_async(tile + (TM + kTH + lr) * kRowStride + at, (const float*)urow + k, w_live ? left : 0);
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        }
    };
    if (ASYNC) {
#pragma unroll
        for (int i = 0; i < STAGES - 1; ++i) copy((int64_t)i * kTK, simt_smem + i * TILE);
    } else {
        fetch(0);
        put(simt_smem);
        __syncthreads();
    }
    int b = 0;
    for (int64_t k0 = 0; k0 < a.K; k0 += kTK, b = b + 1 == STAGES ? 0 : b + 1) {
        const bool more = k0 + kTK < a.K;
        if (ASYNC) {
            asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 2) : "memory");
            __syncthreads();                                 // this tile is there, and the one before has been read by all
            copy(k0 + (STAGES - 1) * kTK, simt_smem + (b == 0 ? STAGES - 1 : b - 1) * TILE);
        } else if (more) {
            fetch(k0 + kTK);
        }
        const float* tile = simt_smem + b * TILE;
#pragma unroll
        for (int i = 0; i < DEPTH; i += 2) {
            const float* at = tile + group * DEPTH + i;
            float2 x[8], gw[4], uw[4];
#pragma unroll
            for (int r = 0; r < 8; ++r) x[r] = *reinterpret_cast<const float2*>(at + (ty + TY * r) * kRowStride);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                gw[c] = *reinterpret_cast<const float2*>(at + (TM + tx + 8 * c) * kRowStride);
                uw[c] = *reinterpret_cast<const float2*>(at + (TM + kTH + tx + 8 * c) * kRowStride);
            }
#pragma unroll
            for (int r = 0; r < 8; ++r)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    g[r][c] = fmaf(x[r].y, gw[c].y, fmaf(x[r].x, gw[c].x, g[r][c]));
                    u[r][c] = fmaf(x[r].y, uw[c].y, fmaf(x[r].x, uw[c].x, u[r][c]));
                }
        }
        if (!ASYNC) {
            if (more) put(simt_smem + (b ^ 1) * TILE);
            __syncthreads();
        }
    }
    __syncthreads();                 // (ASYNC: no copy is under way any more, those past the end were empty)
    // sums of group `group`, row `r`, accumulator column `c` (0 .. 31: G, 32 .. 63: U): [group][r][c]
#pragma unroll
    for (int r = 0; r < 8; ++r)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            float* at = simt_smem + (group * TM + ty + TY * r) * kSumStride + tx + 8 * c;
            at[0] = g[r][c];
            at[kTH] = u[r][c];
        }
    __syncthreads();
    const int64_t n = n0 + t % kTH;
    if (n >= a.N) return;
    const float bg = a.bias ? to_f32(((const T*)a.bias)[n]) : 0.0f, bu = a.bias ? to_f32(((const T*)a.bias)[a.N + n]) : 0.0f;
    with_act(a.act, [&](auto tag) {
#pragma unroll 1
        for (int r = t / kTH; r < TM && m0 + r < a.M; r += 256 / kTH) {
            float gv = bg, uv = bu;
#pragma unroll
            for (int p = 0; p < GROUPS; ++p) {
                gv += simt_smem[(p * TM + r) * kSumStride + t % kTH];
                uv += simt_smem[(p * TM + r) * kSumStride + kTH + t % kTH];
            }
            const int64_t m = m0 + r;
            ((T*)a.out)[m * a.ldo + n] = from_f32<T>(act_value<decltype(tag)::value, EXACT>(gv) * uv);
            if (a.p_save) {
                T* p = (T*)a.p_save + m * a.ldp + n;
                p[0] = from_f32<T>(gv);
                p[a.N] = from_f32<T>(uv);
            }
        }
    });
}

}  // namespace

lrd_status_t gate_fwd(int64_t M, int64_t N, const void* P, int64_t ldp, void* H, int64_t ldh, int act, lrd_dtype_t dt, cudaStream_t s) {
    return run_gate<false>(GateParams{M, N, P, nullptr, H, nullptr, ldp, ldh, 0, act}, dt, s);
}

// enough chunks of rows for some six blocks an SM, of 16 rows or more
int64_t gate_sum_chunks(int64_t M, int64_t N) {
    const int64_t across = (N + kSumCols * 8 - 1) / (kSumCols * 8), most = (M + 15) / 16;
    const int64_t chunks = kNumSms * 6 / across;
    return chunks < 1 ? 1 : chunks > most ? (most < 1 ? 1 : most) : chunks;
}
lrd_status_t gate_bwd_sums(int64_t M, int64_t N, const void* dH, int64_t ldh, const void* P, int64_t ldp, void* dP, int64_t lddp, void* sums, float* partial,
                           int act, lrd_dtype_t dt, cudaStream_t s) {
    const GateParams p{M, N, P, dH, nullptr, dP, ldp, ldh, lddp, act};
    if (dt != LRD_BF16 || p.lddp % 8 || !on16(dP)) return LRD_ERR_UNSUPPORTED;       // (the backward pass asks for no others)
    __nv_bfloat16* to = (__nv_bfloat16*)sums;
    if (bwd_wide(p, 8)) return launch_gate_sums<8, false>(p, partial, to, s);
    return loose_best(M, N, true) ? launch_gate_sums<8, true>(p, partial, to, s) : launch_gate_sums<1, false>(p, partial, to, s);
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

lrd_status_t rows_to_boundaries(const RowCopy* jobs, int n, cudaStream_t s) {
    RowCopies b = {};
    for (int i = 0; i < n; ++i) {
        if (jobs[i].rows <= 0) continue;
        if (b.n == 2 || jobs[i].ldd % 16 || ((uintptr_t)jobs[i].dst & 15u)) return LRD_ERR_UNSUPPORTED;
        RowCopy& c = b.job[b.n] = jobs[i];
        c.units = (c.bytes + 2047) / 2048;
        b.first[b.n + 1] = b.first[b.n] + c.rows * c.units;
        ++b.n;
    }
    if (b.n == 0) return LRD_OK;
    void* args[] = {&b};
    const int64_t blocks = std::min<int64_t>((b.first[b.n] + 7) / 8, kNumSms * 16);
    return launch_pdl((const void*)rows_to_boundaries_kernel, dim3((unsigned)blocks), 256, args, s) ? LRD_OK : LRD_ERR_CUDA;
}

lrd_status_t simt_glu(const GluArgs& g, cudaStream_t s) {
    if (g.M <= 0) return LRD_OK;
    // rows of a tile: 16 where all such tiles find a place at once (two an SM) or there are no more, else 64 where such tiles are two for each SM
    // and would not be half empty, else 32
    // (16 / 32 / 64, us: 111 x 640 -> 1280 16.6 / 25.6 / 27.0, 503 x 768 -> 128 11.4 / 17.4 / 31.9, 400 x 512 -> 700, 550 tiles of 16 rows, 25.9 / 21.1 /
    // 37.8, 256 x 512 -> 1376 32.1 / 30.7 / 38.0)
    const int64_t across = (g.N + kTH - 1) / kTH;
    const int tm = g.M <= 16 || (g.M + 15) / 16 * across <= 2 * kNumSms ? 16 : g.M > 32 && (g.M + 63) / 64 * across >= 2 * kNumSms ? 64 : 32;
    const int64_t tiles = (g.M + tm - 1) / tm * across;
    if (tiles > 0x7FFFFFFF) return LRD_ERR_TOO_LARGE;
    const size_t four = 4 * elem_size(g.dtype);              // bytes of four elements, one access where rows start on such boundaries
    GluArgs a = g;
    int wide_x = g.ldx % 4 == 0 && (uintptr_t)g.X % four == 0, wide_w = g.ldw % 4 == 0 && (uintptr_t)g.W % four == 0;
    void* args[] = {&a, &wide_x, &wide_w};
    auto run = [&](const void* kern, size_t smem, bool (&configured_on)[kMaxDevices]) -> lrd_status_t {
        bool& configured = configured_on[device_slot()];     // per instantiation; the attribute is sticky per function
        if (!configured) {
            if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) return LRD_ERR_CUDA;
            configured = true;
        }
        return launch_pdl(kern, dim3((unsigned)tiles), 256, args, s, smem) ? LRD_OK : LRD_ERR_CUDA;
    };
    static bool configured[9][kMaxDevices] = {};
    auto by_rows = [&](auto type, auto async, int first) -> lrd_status_t {
        using T = decltype(type);
        constexpr bool A = decltype(async)::value != 0;
        if (tm == 64) return run((const void*)simt_glu_kernel<T, 64, A>, simt_glu_smem<64, A>(), configured[first]);
        if (tm == 32) return run((const void*)simt_glu_kernel<T, 32, A>, simt_glu_smem<32, A>(), configured[first + 1]);
        return run((const void*)simt_glu_kernel<T, 16, A>, simt_glu_smem<16, A>(), configured[first + 2]);
    };
    if (g.dtype == LRD_BF16) return by_rows(__nv_bfloat16(), ActTag<0>(), 0);
    return wide_x && wide_w ? by_rows(float(), ActTag<1>(), 3) : by_rows(float(), ActTag<0>(), 6);
}

}  // namespace lrd
