// Entry points of gated feed-forward blocks and of products in 8-bit integers: argument checks and the launches of a call.
#include <cstdint>

#include "api.cuh"
#include "glu.cuh"
#include "tc.cuh"

using namespace lrd;

namespace {

// tile and tensor-map coordinates are 32-bit
constexpr int64_t kMaxSize = 0x7FFFFFFF - 1024;
// largest reduction whose sum of products of 8-bit integers (-128 among them) always fits 32 bits
constexpr int64_t kMaxI8K = 131071;

struct Glu {
    int64_t M, K, N, ldx, ldw, ldh, ldp;
    lrd_dtype_t dt;
    int act;
};

bool bad_act(int act) { return act != LRD_ACT_SILU && act != LRD_ACT_GELU && act != LRD_ACT_GELU_TANH; }

// products: the call reads X and W (else the gate alone: K, ldx and ldw are not looked at)
lrd_status_t parse_glu(const lrd_glu_desc_t* d, Glu* G, bool products) {
    if (!d || d->M < 0 || d->N < 1 || bad_act(d->act)) return LRD_ERR_INVALID_ARG;
    if (d->dtype != LRD_F32 && d->dtype != LRD_BF16) return LRD_ERR_INVALID_ARG;
    if (d->M > kMaxSize || d->N > kMaxSize / 2) return LRD_ERR_TOO_LARGE;
    *G = Glu{d->M, d->K, d->N, d->ldx ? d->ldx : d->K, d->ldw ? d->ldw : d->K, d->ldh ? d->ldh : d->N, d->ldp ? d->ldp : 2 * d->N, (lrd_dtype_t)d->dtype, d->act};
    if (G->ldh < G->N || G->ldp < 2 * G->N) return LRD_ERR_INVALID_ARG;
    if (!products) return LRD_OK;
    if (d->K < 1 || G->ldx < G->K || G->ldw < G->K) return LRD_ERR_INVALID_ARG;
    return d->K > kMaxSize ? LRD_ERR_TOO_LARGE : LRD_OK;
}

// bf16 rows that TMA cannot address are copied into the workspace with padded rows, as the factors of decomposed layers are.  A forward
// pass of few tokens reads its operands as they lie: copying W would cost more than the product.
// A backward pass does it for every K that is no multiple of 8, so that its results are copied out and end with their last column.
bool repacked(const Glu& G, bool bwd) { return G.dt == LRD_BF16 && (bwd ? G.ldx % 8 || G.ldw % 8 || G.K % 8 : (G.ldx % 8 || G.ldw % 8) && G.M > kFewTokens); }

struct GluLayout {              // offsets into the workspace
    int64_t ldk, ldd;           // leading dimensions of the copies of X, W, dX, dW and of dP
    size_t Xp, Wp, dP, dXp, dWp, sums, split, split_bytes, total;
};
GluLayout glu_layout(const Glu& G, bool bwd) {
    GluLayout o = {};
    const size_t e = elem_size(G.dt), M = (size_t)(G.M > 0 ? G.M : 1), rows_w = 2 * (size_t)G.N;
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t here = at; at += align_up(bytes, 256); return here; };
    o.ldk = (G.K + 7) / 8 * 8;
    o.ldd = G.dt == LRD_BF16 ? (2 * G.N + 7) / 8 * 8 : 2 * G.N;
    if (repacked(G, bwd)) {
        o.Xp = take(M * (size_t)o.ldk * e);
        o.Wp = take(rows_w * (size_t)o.ldk * e);
    }
    if (bwd) {
        o.dP = take(M * (size_t)o.ldd * e);
        if (repacked(G, true)) {
            o.dXp = take(M * (size_t)o.ldk * e);
            o.dWp = take(rows_w * (size_t)o.ldk * e);
        }
        o.sums = take((size_t)gate_sum_chunks(G.M, G.N) * rows_w * sizeof(float));
        o.split_bytes = G.dt == LRD_BF16 && G.M > 0 ? tc_split_workspace_bytes(2 * G.N, G.K, G.M) : 0;
        o.split = take(o.split_bytes);
    }
    o.total = at > 256 ? at : 256;
    return o;
}

bool on16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

// X and W as the tensor-core kernels take them: copies where their rows are repacked.  (A base off a 16-byte boundary is copied too
// where the rows are; elsewhere the general kernels take it.)
lrd_status_t repack_inputs(const Glu& G, const GluLayout& o, uint8_t* w, const void** X, int64_t* ldx, const void** W, int64_t* ldw, cudaStream_t s) {
    const int K = (int)G.K, ldk = (int)o.ldk;
    const Copy2d in[2] = {{w + o.Xp, o.ldk, *X, G.ldx, G.M, G.M, K, ldk}, {w + o.Wp, o.ldk, *W, G.ldw, 2 * G.N, 2 * G.N, K, ldk}};
    LRD_TRY(copy2d_bf16(in, 2, s));
    *X = w + o.Xp; *W = w + o.Wp;
    *ldx = *ldw = o.ldk;
    return LRD_OK;
}

lrd_status_t dense_glu_fwd(const lrd_glu_desc_t* desc, const void* X, const void* W, const void* bias, void* H, void* P_save, void* workspace,
                           size_t workspace_bytes, void* cuda_stream) {
    Glu G;
    LRD_TRY(parse_glu(desc, &G, true));
    if (!X || !W || !H) return LRD_ERR_INVALID_ARG;
    for (const void* p : {X, W, bias, (const void*)H, (const void*)P_save})
        if (p && !elem_aligned(p, G.dt)) return LRD_ERR_ALIGNMENT;
    const GluLayout o = glu_layout(G, false);
    if (repacked(G, false)) LRD_TRY(check_ws(workspace, workspace_bytes, o.total));
    LRD_TRY(check_arch());
    if (G.M == 0) return LRD_OK;
    cudaStream_t s = (cudaStream_t)cuda_stream;
    GluArgs a;
    a.M = G.M; a.N = G.N; a.K = G.K; a.X = X; a.ldx = G.ldx; a.W = W; a.ldw = G.ldw; a.bias = bias;
    a.out = H; a.ldo = G.ldh; a.p_save = P_save; a.ldp = G.ldp; a.dtype = G.dt; a.act = G.act; a.gated = true;
    const bool forced = glu_form().columns != 0;             // (the test hook asks for a tensor-core form)
    if (G.M <= kFewTokens && current_path() != LRD_PATH_GENERAL && !forced && (G.dt != LRD_BF16 || few_tokens_best(a))) return few_tokens(a, s);
    if (G.dt != LRD_BF16 || current_path() == LRD_PATH_GENERAL) return simt_glu(a, s);
    if (repacked(G, false)) LRD_TRY(repack_inputs(G, o, (uint8_t*)workspace, &a.X, &a.ldx, &a.W, &a.ldw, s));
    return a.ldx % 8 == 0 && a.ldw % 8 == 0 && on16(a.X) && on16(a.W) ? tc_glu_bf16(a, s) : simt_glu(a, s);
}

lrd_status_t dense_glu_bwd(const lrd_glu_desc_t* desc, const void* dH, const void* X, const void* W, const void* P, void* dX, void* dW, void* dbias,
                           void* workspace, size_t workspace_bytes, void* cuda_stream) {
    Glu G;
    LRD_TRY(parse_glu(desc, &G, true));
    if (!dH || !X || !W || !P || !dW) return LRD_ERR_INVALID_ARG;
    for (const void* p : {dH, X, W, P, (const void*)dX, (const void*)dW, (const void*)dbias})
        if (p && !elem_aligned(p, G.dt)) return LRD_ERR_ALIGNMENT;
    const GluLayout o = glu_layout(G, true);
    LRD_TRY(check_ws(workspace, workspace_bytes, o.total));
    LRD_TRY(check_arch());
    cudaStream_t s = (cudaStream_t)cuda_stream;
    const int64_t rows_w = 2 * G.N;
    if (G.M == 0) {                      // no tokens: the gradients are sums over nothing
        LRD_TRY(zero_fill(dW, rows_w, G.K, G.ldw, G.dt, s));
        return zero_fill(dbias, 1, rows_w, rows_w, G.dt, s);
    }
    const int path = current_path();
    uint8_t* w = (uint8_t*)workspace;
    int64_t ldx = G.ldx, ldw = G.ldw;
    void *to_dX = dX, *to_dW = dW;
    const bool repack = repacked(G, true) && path != LRD_PATH_GENERAL;
    if (repack) {
        LRD_TRY(repack_inputs(G, o, w, &X, &ldx, &W, &ldw, s));
        if (dX) to_dX = w + o.dXp;
        to_dW = w + o.dWp;
    }
    // dP is rounded to the storage type: both products read it, and in bf16 the tensor cores take nothing wider beside bf16 X and W (one more
    // rounding of 2^-8 in the sums: off by 0.0023 of their norm instead of 0.0017)
    void* dP = w + o.dP;
    GemmArgs gw = make_gemm(rows_w, G.K, G.M, dP, o.ldd, true, X, ldx, true, to_dW, ldw, nullptr, G.dt);
    const GemmArgs gx = make_gemm(G.M, G.K, rows_w, dP, o.ldd, false, W, ldw, true, to_dX, ldx, nullptr, G.dt);
    const bool walk = path != LRD_PATH_GENERAL && tc_wgrad_walks(gw), both = path != LRD_PATH_GENERAL && dX && tc_two_products_best(gx, gw, walk, dbias && !walk ? 4.0 : 0.0);
    // The bias gradient beside the gate where dW takes an unsplit walk, which has no place for it; a by-product of dW elsewhere, where it
    // costs less than a launch (1336 x 256 -> 2 x 768: 21.3 us with it beside the gate, 16.9 so, 16.5 without a bias).  Beside the gate dP is summed
    // before its rounding, as a by-product after it: either is within the bound that the roundings of dP give.
    if (dbias && (walk || both)) LRD_TRY(gate_bwd_sums(G.M, G.N, dH, G.ldh, P, G.ldp, dP, o.ldd, dbias, (float*)(w + o.sums), G.act, G.dt, s));
    else LRD_TRY(gate_bwd(G.M, G.N, dH, G.ldh, P, G.ldp, dP, o.ldd, G.act, G.dt, s));
    if (both) {
        LRD_TRY(tc_two_products(gx, gw, s));
    } else {
        if (dX) LRD_TRY(run_gemm(gx, path, false, nullptr, 0, s));
        if (walk) {
            LRD_TRY(tc_wgrad_persistent(gw, s));
        } else {
            gw.a_colsum = dbias;
            LRD_TRY(run_gemm(gw, path, true, (float*)(w + o.split), o.split_bytes, s));
        }
    }
    if (!repack) return LRD_OK;
    const int K = (int)G.K;
    const Copy2d out[2] = {{dX, G.ldx, to_dX, o.ldk, G.M, dX ? G.M : 0, K, K}, {dW, G.ldw, to_dW, o.ldk, rows_w, rows_w, K, K}};
    return copy2d_bf16(out, 2, s);
}

lrd_status_t gate_fwd_call(const lrd_glu_desc_t* desc, const void* P, void* H, void* cuda_stream) {
    Glu G;
    LRD_TRY(parse_glu(desc, &G, false));
    if (!P || !H) return LRD_ERR_INVALID_ARG;
    if (!elem_aligned(P, G.dt) || !elem_aligned(H, G.dt)) return LRD_ERR_ALIGNMENT;
    LRD_TRY(check_arch());
    return gate_fwd(G.M, G.N, P, G.ldp, H, G.ldh, G.act, G.dt, (cudaStream_t)cuda_stream);
}

lrd_status_t gate_bwd_call(const lrd_glu_desc_t* desc, const void* dH, const void* P, void* dP, void* cuda_stream) {
    Glu G;
    LRD_TRY(parse_glu(desc, &G, false));
    if (!dH || !P || !dP) return LRD_ERR_INVALID_ARG;
    for (const void* p : {dH, P, (const void*)dP})
        if (!elem_aligned(p, G.dt)) return LRD_ERR_ALIGNMENT;
    LRD_TRY(check_arch());
    return gate_bwd(G.M, G.N, dH, G.ldh, P, G.ldp, dP, G.ldp, G.act, G.dt, (cudaStream_t)cuda_stream);
}

struct I8 {
    int64_t M, K, N, ldx, ldw, ldy;
    lrd_dtype_t dt;
};
lrd_status_t parse_i8(const lrd_i8_desc_t* d, I8* L, bool gated) {
    if (!d || d->M < 0 || d->K < 1 || d->N < 1 || (gated && bad_act(d->act))) return LRD_ERR_INVALID_ARG;
    if (d->dtype != LRD_F32 && d->dtype != LRD_BF16) return LRD_ERR_INVALID_ARG;
    *L = I8{d->M, d->K, d->N, d->ldx ? d->ldx : d->K, d->ldw ? d->ldw : d->K, d->ldy ? d->ldy : d->N, (lrd_dtype_t)d->dtype};
    if (L->ldx < L->K || L->ldw < L->K || L->ldy < L->N) return LRD_ERR_INVALID_ARG;
    return d->K > kMaxI8K || d->M > kMaxSize || d->N > kMaxSize / 2 ? LRD_ERR_TOO_LARGE : LRD_OK;
}
// 8-bit rows that do not start at multiples of 16 bytes are copied into the workspace
struct I8Layout { int64_t ld; size_t Xp, Wp, total; };
I8Layout i8_layout(const I8& L, bool gated) {
    I8Layout o = {(L.K + 15) / 16 * 16, 0, 0, 0};
    if (L.M <= kFewTokens) return o;                       // read as they lie
    if (L.ldx % 16) o.total += align_up((size_t)(L.M > 0 ? L.M : 1) * (size_t)o.ld, 256);
    o.Wp = o.total;
    if (L.ldw % 16) o.total += align_up((size_t)(gated ? 2 * L.N : L.N) * (size_t)o.ld, 256);
    return o;
}

lrd_status_t i8_product(const lrd_i8_desc_t* desc, const void* Xq, const float* x_scale, const void* Wq, const float* w_scale, const void* bias, void* Y,
                        void* workspace, size_t workspace_bytes, bool gated, void* cuda_stream) {
    I8 L;
    LRD_TRY(parse_i8(desc, &L, gated));
    if (!Xq || !x_scale || !Wq || !w_scale || !Y) return LRD_ERR_INVALID_ARG;
    if (!on16(Xq) || !on16(Wq) || (uintptr_t)x_scale % 4 || (uintptr_t)w_scale % 4 || !elem_aligned(Y, L.dt) || (bias && !elem_aligned(bias, L.dt)))
        return LRD_ERR_ALIGNMENT;
    const I8Layout o = i8_layout(L, gated);
    LRD_TRY(check_ws(workspace, workspace_bytes, o.total));
    LRD_TRY(check_arch());
    if (L.M == 0) return LRD_OK;
    cudaStream_t s = (cudaStream_t)cuda_stream;
    GluArgs a;
    a.M = L.M; a.N = L.N; a.K = L.K; a.X = Xq; a.ldx = L.ldx; a.W = Wq; a.ldw = L.ldw; a.bias = bias; a.out = Y; a.ldo = L.ldy;
    a.x_scale = x_scale; a.w_scale = w_scale; a.dtype = L.dt; a.act = desc->act; a.gated = gated;
    if (L.M <= kFewTokens) {
        const bool rows16 = L.ldx % 16 == 0 && L.ldw % 16 == 0;
        if (glu_form().columns == 0 && (!rows16 || few_tokens_best(a))) return few_tokens(a, s);
        return rows16 ? tc_glu_i8(a, s) : LRD_ERR_UNSUPPORTED;       // (the test hook asks for a tensor-core form)
    }
    uint8_t* w = (uint8_t*)workspace;
    const RowCopy in[2] = {{w + o.Xp, o.ld, Xq, L.ldx, L.ldx % 16 ? L.M : 0, L.K, 0},
                           {w + o.Wp, o.ld, Wq, L.ldw, L.ldw % 16 ? gated ? 2 * L.N : L.N : 0, L.K, 0}};
    LRD_TRY(rows_to_boundaries(in, 2, s));
    if (in[0].rows) { a.X = w + o.Xp; a.ldx = o.ld; }
    if (in[1].rows) { a.W = w + o.Wp; a.ldw = o.ld; }
    return tc_glu_i8(a, s);
}

lrd_status_t i8_quantize_call(const void* X, int64_t ldx, int64_t M, int64_t K, void* Xq, int64_t ldq, float* scale, lrd_dtype_t dtype, void* cuda_stream) {
    if (M < 0 || K < 1 || (dtype != LRD_F32 && dtype != LRD_BF16)) return LRD_ERR_INVALID_ARG;
    if (ldx == 0) ldx = K;
    if (ldq == 0) ldq = K;
    if (ldx < K || ldq < K || !X || !Xq || !scale) return LRD_ERR_INVALID_ARG;
    if (M > kMaxSize) return LRD_ERR_TOO_LARGE;
    if (!elem_aligned(X, dtype) || (uintptr_t)scale % 4) return LRD_ERR_ALIGNMENT;
    LRD_TRY(check_arch());
    return i8_quantize(X, ldx, M, K, (int8_t*)Xq, ldq, scale, dtype, (cudaStream_t)cuda_stream);
}

}  // namespace

GluForm& lrd::glu_form() {
    static thread_local GluForm form = {0, 0, 0};
    return form;
}

extern "C" {

lrd_status_t lrd_glu_tuning(int columns, int blocks_per_mma, int split) {
    if (columns != 0 && columns != 32 && columns != 64 && columns != 128 && columns != 256) return LRD_ERR_INVALID_ARG;
    if (blocks_per_mma < 0 || blocks_per_mma > 2) return LRD_ERR_INVALID_ARG;
    if (split < 0 || split > 8 || (split & (split - 1)) || (split > 1 && (!columns || blocks_per_mma == 2))) return LRD_ERR_INVALID_ARG;
    glu_form() = GluForm{columns, blocks_per_mma, split};
    return LRD_OK;
}

size_t lrd_glu_workspace_bytes(const lrd_glu_desc_t* desc, int is_bwd) {
    Glu G;
    return parse_glu(desc, &G, true) == LRD_OK ? glu_layout(G, is_bwd != 0).total : 0;
}

size_t lrd_i8_workspace_bytes(const lrd_i8_desc_t* desc, int gated) {
    I8 L;
    if (parse_i8(desc, &L, gated != 0) != LRD_OK) return 0;
    const size_t need = i8_layout(L, gated != 0).total;
    return need > 256 ? need : 256;
}

lrd_status_t lrd_dense_glu_fwd(const lrd_glu_desc_t* desc, const void* X, const void* W, const void* bias, void* H, void* P_save, void* workspace,
                               size_t workspace_bytes, void* cuda_stream) {
    return debug_checked(dense_glu_fwd(desc, X, W, bias, H, P_save, workspace, workspace_bytes, cuda_stream), cuda_stream);
}

lrd_status_t lrd_dense_glu_bwd(const lrd_glu_desc_t* desc, const void* dH, const void* X, const void* W, const void* P, void* dX, void* dW, void* dbias,
                               void* workspace, size_t workspace_bytes, void* cuda_stream) {
    return debug_checked(dense_glu_bwd(desc, dH, X, W, P, dX, dW, dbias, workspace, workspace_bytes, cuda_stream), cuda_stream);
}

lrd_status_t lrd_gate_fwd(const lrd_glu_desc_t* desc, const void* P, void* H, void* cuda_stream) {
    return debug_checked(gate_fwd_call(desc, P, H, cuda_stream), cuda_stream);
}

lrd_status_t lrd_gate_bwd(const lrd_glu_desc_t* desc, const void* dH, const void* P, void* dP, void* cuda_stream) {
    return debug_checked(gate_bwd_call(desc, dH, P, dP, cuda_stream), cuda_stream);
}

lrd_status_t lrd_i8_quantize(const void* X, int64_t ldx, int64_t M, int64_t K, void* Xq, int64_t ldq, float* scale, lrd_dtype_t dtype, void* cuda_stream) {
    return debug_checked(i8_quantize_call(X, ldx, M, K, Xq, ldq, scale, dtype, cuda_stream), cuda_stream);
}

lrd_status_t lrd_i8_dense_fwd(const lrd_i8_desc_t* desc, const void* Xq, const float* x_scale, const void* Wq, const float* w_scale, const void* bias,
                              void* Y, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    return debug_checked(i8_product(desc, Xq, x_scale, Wq, w_scale, bias, Y, workspace, workspace_bytes, false, cuda_stream), cuda_stream);
}

lrd_status_t lrd_i8_glu_fwd(const lrd_i8_desc_t* desc, const void* Xq, const float* x_scale, const void* Wq, const float* w_scale, const void* bias,
                            void* H, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    return debug_checked(i8_product(desc, Xq, x_scale, Wq, w_scale, bias, H, workspace, workspace_bytes, true, cuda_stream), cuda_stream);
}

}  // extern "C"
