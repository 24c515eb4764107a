// Gated feed-forward blocks and products in 8-bit integers: internal interface and the activations.
//   P = X W^T + bias = [G | U]  (W[2N x K]: rows 0 .. N-1 give G, the others U),   H = act(G) * U
#pragma once
#include "common.cuh"

namespace lrd {

// One product on the tensor cores with its epilogue.  gated: out[M x N] = act(G) * U, p_save (nullable) = P; else
// out[M x N] = X W^T + bias with W[N x K].
struct GluArgs {
    int64_t M, N, K;
    const void* X; int64_t ldx;
    const void* W; int64_t ldw;
    const void* bias;                                        // [2N] or [N], in `dtype`; nullable
    void* out; int64_t ldo;
    void* p_save = nullptr; int64_t ldp = 0;
    const float *x_scale = nullptr, *w_scale = nullptr;      // 8-bit operands: of each row of X and of W
    lrd_dtype_t dtype;                                       // of out, bias and p_save (and of X and W where they are not 8-bit)
    int act;
    bool gated;
};
// bf16 operands, gated; 8-bit operands, gated or not.  X and W on 16-byte boundaries with rows of whole 16-byte groups; the
// others as they come.
lrd_status_t tc_glu_bf16(const GluArgs& g, cudaStream_t s);
lrd_status_t tc_glu_i8(const GluArgs& g, cudaStream_t s);
// Test hook of the calling host thread: tiles of `columns` accumulator columns on `blocks` blocks per MMA, the reduction over `split` blocks (0: automatic).
struct GluForm { int columns, blocks, split; };
GluForm& glu_form();
// At most kFewTokens rows of X, any alignment; few_tokens_best: where the other kernels would take it too, whether this one is the faster.
constexpr int kFewTokens = 4;
bool few_tokens_best(const GluArgs& g);
lrd_status_t few_tokens(const GluArgs& g, cudaStream_t s);
// Gated, fp32 or bf16, any alignment: fp32 FMA.
lrd_status_t simt_glu(const GluArgs& g, cudaStream_t s);

lrd_status_t gate_fwd(int64_t M, int64_t N, const void* P, int64_t ldp, void* H, int64_t ldh, int act, lrd_dtype_t dt, cudaStream_t s);
// dP may be P itself.
lrd_status_t gate_bwd(int64_t M, int64_t N, const void* dH, int64_t ldh, const void* P, int64_t ldp, void* dP, int64_t lddp, int act,
                      lrd_dtype_t dt, cudaStream_t s);
// With the column sums of dP (2N of them); partial: scratch of gate_sum_chunks(M, N) x 2N floats.  M > 0.
int64_t gate_sum_chunks(int64_t M, int64_t N);
lrd_status_t gate_bwd_sums(int64_t M, int64_t N, const void* dH, int64_t ldh, const void* P, int64_t ldp, void* dP, int64_t lddp, void* sums, float* partial,
                           int act, lrd_dtype_t dt, cudaStream_t s);
lrd_status_t i8_quantize(const void* X, int64_t ldx, int64_t M, int64_t K, int8_t* Xq, int64_t ldq, float* scale, lrd_dtype_t dt, cudaStream_t s);
// `bytes` of each row, which may start anywhere, to rows on 16-byte boundaries (ldd, a multiple of 16; zeros behind the bytes up to the next
// one); up to two such copies in one launch.  Sources must not overlap destinations.
struct RowCopy {
    void* dst; int64_t ldd;
    const void* src; int64_t lds;
    int64_t rows, bytes, units;                              // units: the copy's own
};
lrd_status_t rows_to_boundaries(const RowCopy* jobs, int n, cudaStream_t s);

#ifdef __CUDACC__
// EXACT: CUDA's accurate exp, for fp32 results.  Otherwise 2^(x log2 e) by the hardware's approximation: some 2^-21 of the value for
// arguments of ordinary size, far below the rounding to bf16 (2^-8) that follows.  The reciprocal's approximation is off by one unit in
// the last place either way.  Both without the steps that would keep subnormals: x < -87 gives a sigmoid of 0.
__device__ __forceinline__ float reciprocal(float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
template <bool EXACT> __device__ __forceinline__ float exponential(float x) {
    if (EXACT) return expf(x);
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x * 1.4426950408889634f));
    return r;
}
template <bool EXACT> __device__ __forceinline__ float sigmoid(float x) { return reciprocal(1.0f + exponential<EXACT>(-x)); }
// s = sigmoid(x) and t = 1 - s.  EXACT: t from the exponential, not as a difference, of which next to s = 1 only 2^-24 of 1 is left: times x
// that was 8 last places of SiLU's slope, times x^3 16 of the tanh form's (x = 5 to 10).
template <bool EXACT> __device__ __forceinline__ void sigmoid_both(float x, float& s, float& t) {
    if (EXACT) {
        const float e = expf(-fabsf(x)), r = reciprocal(1.0f + e), er = e * r;
        s = x < 0.0f ? er : r;
        t = x < 0.0f ? r : er;
    } else {
        s = sigmoid<false>(x);
        t = 1.0f - s;
    }
}
constexpr float kGeluTanhScale = 1.5957691216057308f;        // 2 sqrt(2 / pi)
constexpr float kGeluTanhCubic = 0.044715f;

// The normal distribution's cdf, and e = exp(-x^2 / 2).  For fp32 results by erfc, so that the lower tail keeps its digits.  For bf16 ones
// (erfc took the gate on 8192 x 4096 from 34 to 70 us) by exp(-z^2) t q(t), t = 1 / (1 + p z), z = |x| / sqrt 2, q of degree four: t q(t) is
// fitted to exp(z^2) erfc(z) over z <= 9.4 for the smallest weighted error (least squares, weighted anew by the errors until the largest are
// equal: Lawson's algorithm).  The weights ask for 2.4e-4 of the value in the lower tail, an eighth of half a step of bf16, and for an
// absolute 8e-7 where the cdf is large: evaluated in fp32, 2.5e-4 of the value for -13 <= x <= -4, 7e-5 above, 9.2e-7 everywhere.
// Below -13.2 exp(-x^2 / 2) leaves the normal range and the cdf is 0.
constexpr float kTailP = 0.50081127f, kTail0 = 0.27922285f, kTail1 = 0.32230422f, kTail2 = 0.075421915f, kTail3 = 0.51245784f, kTail4 = -0.18940841f;
template <bool EXACT> __device__ __forceinline__ float normal_cdf(float x, float& e) {
    if (EXACT) {
        e = expf(-0.5f * x * x);
        return 0.5f * erfcf(x * -0.70710678118654752f);
    }
    const float z = fabsf(x) * 0.70710678118654752f, t = reciprocal(fmaf(kTailP, z, 1.0f));
    e = exponential<false>(-z * z);
    const float poly = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, kTail4, kTail3), kTail2), kTail1), kTail0);
    const float tail = 0.5f * poly * e;
    return x < 0.0f ? tail : 1.0f - tail;
}

template <int ACT, bool EXACT> __device__ __forceinline__ float act_value(float x) {
    if (ACT == LRD_ACT_SILU) return x * sigmoid<EXACT>(x);
    if (ACT == LRD_ACT_GELU) {
        float e;
        return x * normal_cdf<EXACT>(x, e);
    }
    // 0.5 (1 + tanh z) = sigmoid(2 z)
    return x * sigmoid<EXACT>(kGeluTanhScale * (x + kGeluTanhCubic * x * x * x));
}
// value and derivative
template <int ACT, bool EXACT> __device__ __forceinline__ void act_both(float x, float& value, float& slope) {
    if (ACT == LRD_ACT_GELU) {
        float e;
        const float cdf = normal_cdf<EXACT>(x, e);
        value = x * cdf;
        slope = cdf + x * e * 0.3989422804014327f;
    } else if (ACT == LRD_ACT_SILU) {
        float s, t;
        sigmoid_both<EXACT>(x, s, t);
        value = x * s;
        slope = s * (1.0f + x * t);
    } else {
        // beyond +-30 the sigmoid is 0 or 1 to the last bit and the second term nothing; clamped, no power of x overflows
        const float c = fminf(fmaxf(x, -30.0f), 30.0f);
        float s, t;
        sigmoid_both<EXACT>(kGeluTanhScale * (c + kGeluTanhCubic * c * c * c), s, t);
        value = x * s;
        slope = s + c * s * t * kGeluTanhScale * (1.0f + 3.0f * kGeluTanhCubic * c * c);
        if (x != x) slope = x;
    }
}
// ---- pairs: two fp32 numbers in 64 bits, one instruction for both (the epilogue of a tensor-core tile is bound by its instructions)
__device__ __forceinline__ uint64_t pair_of(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void pair_split(uint64_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t pair_fma(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t pair_mul(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t pair_add(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t pair_both(float a) { return pair_of(a, a); }
__device__ __forceinline__ uint64_t pair_exp2(uint64_t v) {              // 2^x
    float a, b;
    pair_split(v, a, b);
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(a));
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(b));
    return pair_of(a, b);
}
__device__ __forceinline__ uint64_t pair_reciprocal(uint64_t v) {
    float a, b;
    pair_split(v, a, b);
    return pair_of(reciprocal(a), reciprocal(b));
}
// act(x) * u, as act_value does it
template <int ACT, bool EXACT> __device__ __forceinline__ uint64_t pair_gate(uint64_t x, uint64_t u) {
    constexpr float kLog2E = 1.4426950408889634f;
    if (EXACT) {
        float a, b, p, q;
        pair_split(x, a, b);
        pair_split(u, p, q);
        return pair_of(act_value<ACT, true>(a) * p, act_value<ACT, true>(b) * q);
    }
    if (ACT == LRD_ACT_GELU) {
        const uint64_t z = pair_mul(x & 0x7FFFFFFF7FFFFFFFull, pair_both(0.70710678118654752f));
        const uint64_t t = pair_reciprocal(pair_fma(z, pair_both(kTailP), pair_both(1.0f)));
        const uint64_t e = pair_exp2(pair_mul(pair_mul(z, z), pair_both(-kLog2E)));
        uint64_t poly = pair_fma(t, pair_both(kTail4), pair_both(kTail3));
        poly = pair_fma(t, poly, pair_both(kTail2));
        poly = pair_fma(t, poly, pair_both(kTail1));
        poly = pair_fma(t, poly, pair_both(kTail0));
        const uint64_t tail = pair_mul(pair_mul(t, poly), pair_mul(e, pair_both(0.5f)));
        const uint64_t rest = pair_fma(tail, pair_both(-1.0f), pair_both(1.0f));
        float a, b, p, q, c, d;
        pair_split(x, a, b);
        pair_split(tail, p, q);
        pair_split(rest, c, d);
        return pair_mul(pair_mul(x, pair_of(a < 0.0f ? p : c, b < 0.0f ? q : d)), u);
    }
    uint64_t n;                                              // -z log2 e, the sigmoid of z being wanted
    if (ACT == LRD_ACT_SILU) n = pair_mul(x, pair_both(-kLog2E));
    else n = pair_mul(x, pair_fma(pair_mul(x, x), pair_both(-kLog2E * kGeluTanhScale * kGeluTanhCubic), pair_both(-kLog2E * kGeluTanhScale)));
    const uint64_t s = pair_reciprocal(pair_add(pair_exp2(n), pair_both(1.0f)));
    return pair_mul(pair_mul(x, s), u);
}

template <int A> struct ActTag { static constexpr int value = A; };
// f(ActTag<act>): one branch a call, the activation a constant inside
template <typename F> __device__ __forceinline__ void with_act(int act, const F& f) {
    if (act == LRD_ACT_SILU) f(ActTag<LRD_ACT_SILU>());
    else if (act == LRD_ACT_GELU) f(ActTag<LRD_ACT_GELU>());
    else f(ActTag<LRD_ACT_GELU_TANH>());
}
#endif

}  // namespace lrd
