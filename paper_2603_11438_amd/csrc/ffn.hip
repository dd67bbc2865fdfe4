// Gated feed-forward block (gfx950): h = act(x Wg^T) * (x Wu^T) in one kernel,
// and its backward pass (formulas in ar_ops.h).
//
// Compute-bound with many tokens: one product kernel (gemm_nt.h) whose waves
// hold both projections of the same columns, so that the activation and the
// product happen in registers and only h is written.  8192 x 4096 x 11264, silu:
// 1200 us, 1260 TFLOP/s.  Bound by the weights' bytes with few: up to 64 tokens
// share a tile of 64 columns of both, 1 x 4096 x 11264: 41 us, 4.5 TB/s.  Bound by the
// length of k where there are few tiles, as in a rank's share of the columns: there
// k is split, and a second kernel joins the runs and applies the activation (1 x
// 4096 x 1408: 13 us, in one piece 32; 256 x 4096 x 1408: 19 us, in one piece 63).
//
// Backward: dG and dU by one pass over the saved projections (4096 x 11264: 128
// us, 5.0 TB/s), dx as one product over both pairs of operands, both weights'
// gradients as another, operands read by rows or by k where they lie.  Forward
// with saved projections and backward, 4096 x 4096 x 11264: 2060 us, 1100
// TFLOP/s; a third of that the forward, a third the weights' gradients, 28 % dx.
#include <type_traits>

#include "products.h"

#pragma clang fp contract(fast)

namespace ar {
namespace dev {

// act(g), and with `slope` its derivative.
template <int ACT> __device__ __forceinline__ float activation(float g, float *slope = nullptr)
{
    if constexpr (ACT == AR_ACT_RELU) {
        if (slope) *slope = g > 0.0f ? 1.0f : 0.0f;
        return g <= 0.0f ? 0.0f : g;  // NaN stays NaN
    } else if constexpr (ACT == AR_ACT_SILU) {
        const float p = 1.0f / (1.0f + __expf(-g));
        if (slope) *slope = p * (1.0f + g * (1.0f - p));
        return g * p;
    } else {
        // 1 + tanh(z) = 2 / (1 + e^-2z)
        const float c = 0.7978845608028654f, z = c * (g + 0.044715f * g * g * g);
        const float p = 1.0f / (1.0f + __expf(-2.0f * z));
        if (slope) *slope = p + g * 2.0f * p * (1.0f - p) * c * (1.0f + 0.134145f * g * g);
        return g * p;
    }
}

struct FfnOut {
    bf16 *h;
    float *saved;  // G, then U; null: not kept
    float *part;   // with k split: the runs' sums, [run][G, U][m][n]
    uint64_t ld_h;
};

template <typename S, int ACT> __global__ __launch_bounds__(S::THREADS) void ffn_kernel(const GemmArgs g, const FfnOut o)
{
    constexpr int NT = S::NT, HALF = NT * 16;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const TileAt at = tile_at(g.tiles_m, g.tiles_n, 1);
    f32x16 acc[S::MT][NT];
    gemm_tile<bf16, S, true>(g, at, lds, acc);
    const uint32_t wave = threadIdx.x >> 6;
    const uint32_t row0 = at.m * S::BM + (wave >> 1) * S::MT * 32, col0 = at.n * (S::BN / 2) + (wave & 1u) * HALF;
    if (col0 >= g.n) return;
    const uint32_t cols = g.n - col0;
    char *stage = lds + wave * kStageBytes<float, HALF>;
    static_for<S::MT>([&](auto block) {
        constexpr int i = block.value;
        float v[NT][16];
        take(acc[i], v);
        const uint32_t first = row0 + i * 32;
        if (first >= g.m) return;
        const uint32_t rows = g.m - first;
        float *keep = g.splits > 1 ? o.part + (uint64_t)blockIdx.y * 2 * g.m * g.n : o.saved;
        if (keep) {
            float *to = keep + (uint64_t)first * g.n + col0;
            stage_rows<float, HALF>(stage, [&](int j, int r) { return v[j][r]; });
            write_rows<float, HALF>(stage, to, g.n, 0, rows, cols);
            stage_rows<float, HALF>(stage, [&](int j, int r) { return v[j + NT / 2][r]; });
            write_rows<float, HALF>(stage, to + (uint64_t)g.m * g.n, g.n, 0, rows, cols);
        }
        if (g.splits > 1) return;
        stage_rows<bf16, HALF>(stage, [&](int j, int r) { return activation<ACT>(v[j][r]) * v[j + NT / 2][r]; });
        write_rows<bf16, HALF>(stage, o.h + (uint64_t)first * o.ld_h + col0, o.ld_h, 0, rows, cols);
    });
}

// The projections from the runs' sums, added in their order, and h; four columns
// a thread.
template <int ACT> __global__ __launch_bounds__(256) void ffn_join_kernel(const FfnOut o, uint32_t m, uint32_t n, uint32_t splits)
{
    const uint64_t half = (uint64_t)m * n, per = (n + 3) / 4, all = m * per;
    for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (uint64_t)gridDim.x * 256) {
        const uint32_t row = (uint32_t)(i / per), c = (uint32_t)(i % per) * 4;
        const int have = n - c < 4 ? (int)(n - c) : 4;
        const uint64_t at = (uint64_t)row * n + c;
        float g[4] = {0.0f, 0.0f, 0.0f, 0.0f}, u[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        auto add = [&](auto load) {
#pragma unroll 8
            for (uint32_t s = 0; s < splits; ++s) {
                float a[4], b[4];
                load(o.part + s * 2 * half + at, a), load(o.part + (s * 2 + 1) * half + at, b);
#pragma unroll
                for (int k = 0; k < 4; ++k) g[k] += a[k], u[k] += b[k];
            }
        };
        if (have == 4) add([](const float *p, float *v) { load_vec<float, 4>(p, v); });
        else add([&](const float *p, float *v) { load_part<float, 4>(p, have, v); });
        if (o.saved) {
            store_part<float, 4>(o.saved + at, have, g);
            store_part<float, 4>(o.saved + half + at, have, u);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) u[k] *= activation<ACT>(g[k]);
        store_part<bf16, 4>(o.h + row * o.ld_h + c, have, u);
    }
}

// dG = dh * U * act'(G) and dU = dh * act(G) from the saved projections, rounded
// to bf16 as operands of the backward products: rows of dG, then dU, with zeros
// behind the columns of each.
struct GradArgs {
    const float *saved;
    const bf16 *dh;
    bf16 *to;
    uint64_t ld_dh, tokens;
    uint32_t hidden, to_hidden;
};
template <int ACT> __global__ __launch_bounds__(256) void ffn_grad_kernel(const GradArgs a)
{
    const uint64_t per = a.to_hidden / 8, n = a.tokens * per, half = a.tokens * a.hidden;
    for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (uint64_t)gridDim.x * 256) {
        const uint64_t t = i / per;
        const uint32_t f = (uint32_t)(i % per) * 8;
        float g[8], u[8], d[8];
        const int have = f < a.hidden ? (int)(a.hidden - f) : 0;
        const float *from = a.saved + t * a.hidden + f;
        const bf16 *dh = a.dh + t * a.ld_dh + f;
        if (have >= 8) {
            load_vec<float, 8>(from, g);
            load_vec<float, 8>(from + half, u);
            load_vec<bf16, 8>(dh, d);
        } else {
            load_part<float, 8>(from, have, g);
            load_part<float, 8>(from + half, have, u);
            load_part<bf16, 8>(dh, have, d);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            float slope;
            const float act = activation<ACT>(g[k], &slope);
            g[k] = d[k] * u[k] * slope;
            u[k] = d[k] * act;
        }
        bf16 *to = a.to + t * 2 * a.to_hidden + f;
        store_vec<bf16, 8>(to, g);
        store_vec<bf16, 8>(to + a.to_hidden, u);
    }
}

}  // namespace dev

namespace {

using namespace dev;

int check_ffn(const ar_ffn_desc *d)
{
    if (!d) return AR_ERR_ARG;
    if (d->dtype != AR_BFLOAT16) return AR_ERR_UNSUPPORTED;
    if (d->act < AR_ACT_SILU || d->act > AR_ACT_RELU) return AR_ERR_ARG;
    // rows and columns are counted in 32 bits on the device, and a tile's rows reached by 31
    if (d->dim < 1 || d->hidden < 1 || d->tokens > (1u << 30) || d->dim > (1u << 20) || d->hidden > (1u << 20)) return AR_ERR_ARG;
    if (d->tokens * d->hidden > kOpsMaxSize || d->tokens * d->dim > kOpsMaxSize || d->hidden * d->dim > kOpsMaxSize) return AR_ERR_ARG;
    const struct {
        size_t ld, cols, rows;
    } lds[] = {{d->ld_x, d->dim, d->tokens},       {d->ld_w_gate, d->dim, d->hidden}, {d->ld_w_up, d->dim, d->hidden},
               {d->ld_h, d->hidden, d->tokens},    {d->ld_dx, d->dim, d->tokens},     {d->ld_dw_gate, d->dim, d->hidden},
               {d->ld_dw_up, d->dim, d->hidden}};
    for (const auto &l : lds)
        if (l.ld && (l.ld < l.cols || l.ld > kOpsMaxSize / (l.rows ? l.rows : 1))) return AR_ERR_ARG;
    return AR_OK;
}

template <typename S, int ACT> int launch_ffn(GemmArgs &g, const FfnOut &o, hipStream_t st)
{
    g.tiles_m = (g.m + S::BM - 1) / S::BM;
    g.tiles_n = (g.n + S::BN / 2 - 1) / (S::BN / 2);
    static_assert(4 * kStageBytes<float, S::NT * 16> <= S::LDS, "the epilogue's staging fits");
    static OncePerDevice once;
    int rc = allow_lds(once, (const void *)ffn_kernel<S, ACT>, S::LDS);
    if (rc != AR_OK) return rc;
    hipLaunchKernelGGL((ffn_kernel<S, ACT>), dim3(g.tiles_m * g.tiles_n, g.splits), dim3(S::THREADS), S::LDS, st, g, o);
    rc = launch_status();
    if (rc != AR_OK || g.splits == 1) return rc;
    const uint64_t groups = ((uint64_t)g.m * ((g.n + 3) / 4) + 255) / 256;
    hipLaunchKernelGGL((ffn_join_kernel<ACT>), dim3((uint32_t)(groups < 8192 ? groups : 8192)), dim3(256), 0, st, o, g.m, g.n, g.splits);
    return launch_status();
}

size_t ffn_part_bytes(const ar_ffn_desc &d, const Cut &c) { return c.splits > 1 ? c.splits * 2 * d.tokens * d.hidden * sizeof(float) : 0; }

template <int ACT> int launch_ffn_tiles(const Cut &c, bool ahead, GemmArgs &g, const FfnOut &o, hipStream_t st)
{
    if (c.tile == kFlat) return launch_ffn<Flat, ACT>(g, o, st);
    if (c.tile == kPairDeep) return launch_ffn<Deep, ACT>(g, o, st);
    if (c.tile == kPairSmall) return launch_ffn<Small, ACT>(g, o, st);
    return ahead ? launch_ffn<Large, ACT>(g, o, st) : launch_ffn<LargeEven, ACT>(g, o, st);
}

struct FfnMats {
    Mat x, wg, wu, h;
};
FfnMats ffn_mats(const ar_ffn_desc &d, const void *x, const void *wg, const void *wu, const void *h)
{
    return {mat(x, d.tokens, d.dim, d.ld_x, d.dtype), mat(wg, d.hidden, d.dim, d.ld_w_gate, d.dtype),
            mat(wu, d.hidden, d.dim, d.ld_w_up, d.dtype), mat(h, d.tokens, d.hidden, d.ld_h, d.dtype)};
}

// The most the workspace can be asked for: pointers' alignment is not known
// before the call, so every operand counts.
size_t ffn_workspace(const ar_ffn_desc &d)
{
    return packed_bytes(d.tokens, d.dim) + 2 * packed_bytes(d.hidden, d.dim) + ffn_part_bytes(d, ffn_cut(d.tokens, d.dim, d.hidden));
}

// What a call with these operands uses: copies of those that cannot be read where
// they lie, and the runs' sums.
size_t ffn_need(const ar_ffn_desc &d, const FfnMats &m, const Cut &cut)
{
    size_t need = ffn_part_bytes(d, cut);
    for (const Mat &in : {m.x, m.wg, m.wu})
        if (!direct(in)) need += packed_bytes(in.rows, in.cols);
    return need;
}
size_t ffn_workspace_for(const ar_ffn_desc *desc, const void *x, const void *wg, const void *wu)
{
    if (check_ffn(desc) != AR_OK || desc->tokens == 0) return 0;
    return ffn_need(*desc, ffn_mats(*desc, x, wg, wu, nullptr), ffn_cut(desc->tokens, desc->dim, desc->hidden));
}

int ffn(const ar_ffn_desc *desc, const void *x, const void *wg, const void *wu, void *h, float *saved, void *ws,
        size_t ws_bytes, void *stream)
{
    int rc = check_ffn(desc);
    if (rc != AR_OK) return rc;
    const ar_ffn_desc &d = *desc;
    if (d.tokens == 0) return AR_OK;
    const FfnMats m = ffn_mats(d, x, wg, wu, h);
    if (!m.x.ok() || !m.wg.ok() || !m.wu.ok() || !m.h.ok() || (uintptr_t)saved % 16 != 0) return AR_ERR_ARG;
    const Mat sv = mat(saved, 2 * d.tokens, d.hidden, 0, AR_FLOAT32);
    for (const Mat &in : {m.x, m.wg, m.wu})
        if (meet(m.h, in) || meet(sv, in)) return AR_ERR_ARG;
    if (meet(m.h, sv)) return AR_ERR_ARG;
    const Cut cut = ffn_cut(d.tokens, d.dim, d.hidden);
    const size_t need = ffn_need(d, m, cut);
    if (need) {
        if (!ws || ws_bytes < need) return AR_ERR_SCRATCH;
        if ((uintptr_t)ws % 256 != 0) return AR_ERR_ARG;
        const Mat wsm{ws, 1, need, need, 1};
        for (const Mat &o : {m.x, m.wg, m.wu, m.h, sv})
            if (meet(wsm, o)) return AR_ERR_ARG;
    }
    hipStream_t st = (hipStream_t)stream;
    char *at = (char *)ws;
    Operand px, pg, pu;
    PackList packs{};
    pack(m.x, direct(m.x), at, &packs, &px);
    pack(m.wg, direct(m.wg), at, &packs, &pg);
    pack(m.wu, direct(m.wu), at, &packs, &pu);
    if ((rc = run_packs(packs, st)) != AR_OK) return rc;
    GemmArgs g{};
    g.a[0] = px.p, g.b[0] = pg.p, g.b2 = pu.p;
    g.lda = px.ld, g.ldb = pg.ld, g.ldb2 = pu.ld;
    g.segments = 1, g.steps = (uint32_t)(round_up(d.dim, kStepK) / kStepK);
    g.ka = g.kb = (uint32_t)round_up(d.dim, 8);
    g.m = (uint32_t)d.tokens, g.n = (uint32_t)d.hidden, g.batch = 1, g.splits = cut.splits;
    const FfnOut o{(bf16 *)h, saved, (float *)at, m.h.ld};  // the runs' sums behind the copies
    const bool ahead = pair_ahead(d.tokens, d.dim, d.hidden, saved != nullptr);
    switch (d.act) {
    case AR_ACT_SILU: return launch_ffn_tiles<AR_ACT_SILU>(cut, ahead, g, o, st);
    case AR_ACT_GELU: return launch_ffn_tiles<AR_ACT_GELU>(cut, ahead, g, o, st);
    default: return launch_ffn_tiles<AR_ACT_RELU>(cut, ahead, g, o, st);
    }
}

// ---- backward ---------------------------------------------------------------

// Where the backward pass keeps what, in bytes from the workspace's start.
// Copies of operands lie behind the rest, as many as there are.
struct FfnBackwardSpace {
    size_t hidden;  // padded: a tile's block of rows belongs to one of dG and dU
    size_t steps;   // of tokens
    size_t part, copies;  // dG and dU lie at the start
};
FfnBackwardSpace ffn_backward_space(const ar_ffn_desc &d, bool dx, bool dw)
{
    FfnBackwardSpace s{};
    s.hidden = round_up(d.hidden, kStepK), s.steps = (d.tokens + kStepK - 1) / kStepK;
    size_t parts = 0;
    if (dx) parts = part_bytes(dx_cut(d.tokens, d.dim, s.hidden), d.tokens, d.dim);
    if (dw) {
        const size_t p = part_bytes(dw_cut(d.tokens, d.dim, s.hidden), 2 * s.hidden, d.dim);
        parts = p > parts ? p : parts;
    }
    s.part = round_up(d.tokens * 2 * s.hidden * 2, 256);
    s.copies = s.part + parts;
    return s;
}

// What a caller is asked for.  Pointers' alignment is not known before the call,
// and what is wanted neither, so everything counts.
size_t ffn_backward_bytes(const ar_ffn_desc &d)
{
    return ffn_backward_space(d, true, true).copies + 2 * packed_bytes(d.hidden, d.dim) + packed_bytes(d.tokens, d.dim);
}

int ffn_backward(const ar_ffn_desc *desc, const void *dh, const void *x, const void *wg, const void *wu, const float *saved,
                 void *dx, void *dwg, void *dwu, void *ws, size_t ws_bytes, void *stream)
{
    int rc = check_ffn(desc);
    if (rc != AR_OK) return rc;
    const ar_ffn_desc &d = *desc;
    hipStream_t st = (hipStream_t)stream;
    if ((dwg != nullptr) != (dwu != nullptr)) return AR_ERR_ARG;
    const FfnMats m = ffn_mats(d, x, wg, wu, dh);
    const Mat odx = mat(dx, d.tokens, d.dim, d.ld_dx, d.dtype), og = mat(dwg, d.hidden, d.dim, d.ld_dw_gate, d.dtype),
              ou = mat(dwu, d.hidden, d.dim, d.ld_dw_up, d.dtype), sv = mat(saved, 2 * d.tokens, d.hidden, 0, AR_FLOAT32);
    if (!odx.aligned() || !og.aligned() || !ou.aligned()) return AR_ERR_ARG;
    if (meet(og, ou) || meet(odx, og) || meet(odx, ou)) return AR_ERR_ARG;
    if (d.tokens == 0) {
        if (!dwg) return AR_OK;
        rc = zero_rows(og, st);  // sums over no tokens
        return rc != AR_OK ? rc : zero_rows(ou, st);
    }
    if (!m.x.ok() || !m.wg.ok() || !m.wu.ok() || !m.h.ok() || !saved || (uintptr_t)saved % 16 != 0) return AR_ERR_ARG;
    if (!dx && !dwg) return AR_OK;  // nothing wanted
    const FfnBackwardSpace s = ffn_backward_space(d, dx != nullptr, dwg != nullptr);
    // both weights are read with one row stride
    const bool w_direct = direct(m.wg) && direct(m.wu) && m.wg.ld == m.wu.ld, x_direct = direct(m.x);
    size_t need = s.copies;  // of this call
    if (dx && !w_direct) need += 2 * packed_bytes(d.hidden, d.dim);
    if (dwg && !x_direct) need += packed_bytes(d.tokens, d.dim);
    if (!ws || ws_bytes < ffn_backward_bytes(d)) return AR_ERR_SCRATCH;
    if ((uintptr_t)ws % 256 != 0) return AR_ERR_ARG;
    const Mat wsm{ws, 1, need, need, 1};
    for (const Mat &in : {m.x, m.wg, m.wu, m.h, sv, wsm})
        if (meet(odx, in) || meet(og, in) || meet(ou, in)) return AR_ERR_ARG;
    for (const Mat &in : {m.x, m.wg, m.wu, m.h, sv})
        if (meet(wsm, in)) return AR_ERR_ARG;

    char *w = (char *)ws, *copies = w + s.copies;
    const GradArgs ga{saved, (const bf16 *)dh, (bf16 *)w, m.h.ld, d.tokens, (uint32_t)d.hidden, (uint32_t)s.hidden};
    const uint64_t groups = (d.tokens * (s.hidden / 8) + 255) / 256;
    const dim3 grid((uint32_t)(groups < 16384 ? groups : 16384));
    switch (d.act) {
    case AR_ACT_SILU: hipLaunchKernelGGL((ffn_grad_kernel<AR_ACT_SILU>), grid, dim3(256), 0, st, ga); break;
    case AR_ACT_GELU: hipLaunchKernelGGL((ffn_grad_kernel<AR_ACT_GELU>), grid, dim3(256), 0, st, ga); break;
    default: hipLaunchKernelGGL((ffn_grad_kernel<AR_ACT_RELU>), grid, dim3(256), 0, st, ga);
    }
    if ((rc = launch_status()) != AR_OK) return rc;
    Operand px, pg, pu;
    PackList packs{};
    if (dx) pack(m.wg, w_direct, copies, &packs, &pg), pack(m.wu, w_direct, copies, &packs, &pu);
    if (dwg) pack(m.x, x_direct, copies, &packs, &px);
    if ((rc = run_packs(packs, st)) != AR_OK) return rc;
    if (dx) {
        GemmArgs g{};
        g.segments = 2, g.steps = (uint32_t)(s.hidden / kStepK);
        g.ka = (uint32_t)s.hidden, g.kb = (uint32_t)d.hidden;
        g.a[0] = w, g.a[1] = w + s.hidden * 2;
        g.b[0] = pg.p, g.b[1] = pu.p;
        g.lda = (uint32_t)(s.hidden * 4), g.ldb = pg.ld;
        g.m = (uint32_t)d.tokens, g.n = pg.cols;
        const ProductOut o{{(bf16 *)dx, nullptr}, (float *)(w + s.part), {odx.ld, 0}, 0x80000000u, (uint32_t)d.tokens, (uint32_t)d.dim};
        if ((rc = product<false>(dx_cut(d.tokens, d.dim, s.hidden), g, o, st)) != AR_OK) return rc;
    }
    if (dwg) {
        GemmArgs g{};
        g.segments = 1, g.steps = (uint32_t)s.steps;
        g.ka = g.kb = (uint32_t)d.tokens;
        g.a[0] = w, g.b[0] = px.p;
        g.lda = (uint32_t)(s.hidden * 4), g.ldb = px.ld;
        g.m = (uint32_t)(2 * s.hidden), g.n = px.cols;
        const ProductOut o{{(bf16 *)dwg, (bf16 *)dwu}, (float *)(w + s.part), {og.ld, ou.ld}, (uint32_t)s.hidden, (uint32_t)d.hidden, (uint32_t)d.dim};
        if ((rc = product<true>(dw_cut(d.tokens, d.dim, s.hidden), g, o, st)) != AR_OK) return rc;
    }
    return AR_OK;
}

}  // namespace
}  // namespace ar

extern "C" int ar_gated_ffn_backward(const ar_ffn_desc *desc, const void *dh, const void *x, const void *w_gate,
                                     const void *w_up, const float *saved, void *dx, void *dw_gate, void *dw_up,
                                     void *workspace, size_t workspace_bytes, void *stream)
{
    return ar::ops_ret(ar::ffn_backward(desc, dh, x, w_gate, w_up, saved, dx, dw_gate, dw_up, workspace, workspace_bytes, stream));
}

extern "C" size_t ar_gated_ffn_backward_workspace(const ar_ffn_desc *desc)
{
    return ar::check_ffn(desc) == AR_OK && desc->tokens ? ar::ffn_backward_bytes(*desc) : 0;
}

extern "C" int ar_gated_ffn(const ar_ffn_desc *desc, const void *x, const void *w_gate, const void *w_up, void *h,
                            float *saved, void *workspace, size_t workspace_bytes, void *stream)
{
    return ar::ops_ret(ar::ffn(desc, x, w_gate, w_up, h, saved, workspace, workspace_bytes, stream));
}

extern "C" size_t ar_gated_ffn_workspace(const ar_ffn_desc *desc)
{
    return ar::check_ffn(desc) == AR_OK ? ar::ffn_workspace(*desc) : 0;
}

extern "C" size_t ar_gated_ffn_workspace_for(const ar_ffn_desc *desc, const void *x, const void *w_gate, const void *w_up)
{
    return ar::ffn_workspace_for(desc, x, w_gate, w_up);
}
