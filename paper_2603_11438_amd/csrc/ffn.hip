// Gated feed-forward block (gfx950): h = act(x Wg^T) * (x Wu^T) in one kernel,
// and its backward pass (formulas in ar_ops.h).
//
// Compute-bound with many tokens: one product kernel (gemm_nt.h) whose waves
// hold both projections of the same columns, so that the activation and the
// product happen in registers and only h is written.
#include <type_traits>

#include "gemm_nt.h"

#pragma clang fp contract(fast)

namespace ar {
namespace dev {

// act(g), and with `slope` its derivative.
template <int ACT> __device__ __forceinline__ float activation(float g, float *slope = nullptr)
{
    if constexpr (ACT == AR_ACT_RELU) {
        if (slope) *slope = g > 0.0f ? 1.0f : 0.0f;
        return g > 0.0f ? g : g * 0.0f;  // NaN stays NaN
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
        auto row_of = [&](auto *base, uint64_t ld) {
            return [=](uint32_t r) { return row0 + i * 32 + r < g.m ? base + (uint64_t)(row0 + i * 32 + r) * ld + col0 : nullptr; };
        };
        if (o.saved) {
            store_32_rows<float, HALF>(stage, cols, [&](int j, int r) { return v[j][r]; }, row_of(o.saved, g.n));
            store_32_rows<float, HALF>(stage, cols, [&](int j, int r) { return v[j + NT / 2][r]; },
                                       row_of(o.saved + (uint64_t)g.m * g.n, g.n));
        }
        store_32_rows<bf16, HALF>(stage, cols, [&](int j, int r) { return activation<ACT>(v[j][r]) * v[j + NT / 2][r]; },
                                  row_of(o.h, o.ld_h));
    });
}

// Copies a matrix into rows of `to_ld` elements, zeros behind its columns.
struct PackArgs {
    const bf16 *from;
    bf16 *to;
    uint64_t rows, ld, to_ld;
    uint32_t cols;
};
__global__ void pack_kernel(const PackArgs p)
{
    const uint64_t n = p.rows * (p.to_ld / 8);
    for (uint64_t i = (uint64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (uint64_t)gridDim.x * blockDim.x) {
        const uint64_t row = i / (p.to_ld / 8);
        const uint32_t c = (uint32_t)(i % (p.to_ld / 8)) * 8;
        const bf16 *from = p.from + row * p.ld + c;
        bf16x8 v;
        if (c + 8 <= p.cols) {
            v = (bf16x8)*(const VecOf<bf16, 8>::type *)from;
        } else {
#pragma unroll
            for (uint32_t k = 0; k < 8; ++k) v[k] = c + k < p.cols ? from[k] : (bf16)0.0f;
        }
        *(bf16x8 *)(p.to + row * p.to_ld + c) = v;
    }
}

// The transpose of a matrix, with zeros behind the rows' end up to to_ld
// columns: tiles of 64 x 64 through LDS.  The tile's rows are 66 elements apart
// there, so that the columns read back lie in different banks.
struct TransposeArgs {
    const bf16 *from;
    bf16 *to;
    uint64_t ld, to_ld;
    uint32_t rows, cols;
};
constexpr int kTile = 64, kTilePitch = 66;

// Writes the transpose of a staged tile: to[c][r] for the tile's columns c
// below `cols`, every r of the tile.
__device__ __forceinline__ void store_transposed(const bf16 (*tile)[kTilePitch], bf16 *to, uint64_t to_ld, uint32_t cols)
{
    for (uint32_t i = threadIdx.x; i < kTile * kTile / 8; i += 256) {
        const uint32_t c = i / 8, r = i % 8 * 8;
        bf16x8 v;
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = tile[r + k][c];
        if (c < cols) *(bf16x8 *)(to + (uint64_t)c * to_ld + r) = v;
    }
}

__global__ __launch_bounds__(256) void transpose_kernel(const TransposeArgs t)
{
    __shared__ bf16 tile[kTile][kTilePitch];
    const uint32_t r0 = blockIdx.y * kTile, c0 = blockIdx.x * kTile;
    for (uint32_t i = threadIdx.x; i < kTile * kTile / 8; i += 256) {
        const uint32_t r = i / 8, c = i % 8 * 8;
        const bf16 *from = t.from + (uint64_t)(r0 + r) * t.ld + c0 + c;
        float v[8];
        if (r0 + r < t.rows && c0 + c + 8 <= t.cols) load_vec<bf16, 8>(from, v);
        else load_part<bf16, 8>(from, r0 + r < t.rows && c0 + c < t.cols ? (int)(t.cols - c0 - c) : 0, v);
#pragma unroll
        for (int k = 0; k < 8; ++k) tile[r][c + k] = (bf16)v[k];
    }
    __syncthreads();
    store_transposed(tile, t.to + (uint64_t)c0 * t.to_ld + r0, t.to_ld, t.cols - c0 < kTile ? t.cols - c0 : kTile);
}

// dG = dh * U * act'(G) and dU = dh * act(G) from the saved projections, rounded
// to bf16 as operands of the backward products: by rows for dx, transposed for
// the weights' gradients, zeros in the padding of both.
struct GradArgs {
    const float *saved;
    const bf16 *dh;
    bf16 *by_rows;      // tokens x 2 hidden_ld: dG, then dU in each row; null: not wanted
    bf16 *transposed;   // 2 hidden x tokens_ld: dG^T, then dU^T; null: not wanted
    uint64_t ld_dh, hidden_ld, tokens_ld;
    uint32_t tokens, hidden;
};
template <int ACT> __global__ __launch_bounds__(256) void ffn_grad_kernel(const GradArgs a)
{
    __shared__ bf16 tg[kTile][kTilePitch], tu[kTile][kTilePitch];
    const uint32_t t0 = blockIdx.y * kTile, f0 = blockIdx.x * kTile;
    const uint64_t half = (uint64_t)a.tokens * a.hidden;
    for (uint32_t i = threadIdx.x; i < kTile * kTile / 8; i += 256) {
        const uint32_t r = i / 8, c = i % 8 * 8, t = t0 + r, f = f0 + c;
        float g[8], u[8], d[8];
        const int have = t < a.tokens && f < a.hidden ? (int)(a.hidden - f) : 0;
        const float *from = a.saved + (uint64_t)t * a.hidden + f;
        const bf16 *dh = a.dh + (uint64_t)t * a.ld_dh + f;
        if (have >= 8) {
            load_vec<float, 8>(from, g);
            load_vec<float, 8>(from + half, u);
            load_vec<bf16, 8>(dh, d);
        } else {
            load_part<float, 8>(from, have, g);
            load_part<float, 8>(from + half, have, u);
            load_part<bf16, 8>(dh, have, d);
        }
        bf16x8 vg, vu;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            float slope;
            const float act = activation<ACT>(g[k], &slope);
            vg[k] = (bf16)(d[k] * u[k] * slope);
            vu[k] = (bf16)(d[k] * act);
            tg[r][c + k] = vg[k];
            tu[r][c + k] = vu[k];
        }
        if (a.by_rows && t < a.tokens) {
            bf16 *to = a.by_rows + (uint64_t)t * 2 * a.hidden_ld + f;
            *(bf16x8 *)to = vg;
            *(bf16x8 *)(to + a.hidden_ld) = vu;
        }
    }
    if (!a.transposed) return;
    __syncthreads();
    const uint32_t cols = f0 >= a.hidden ? 0 : a.hidden - f0 < kTile ? a.hidden - f0 : kTile;
    store_transposed(tg, a.transposed + (uint64_t)f0 * a.tokens_ld + t0, a.tokens_ld, cols);
    store_transposed(tu, a.transposed + (uint64_t)(a.hidden + f0) * a.tokens_ld + t0, a.tokens_ld, cols);
}

// A plain product: rows below `split` of the result go to out, the others to
// out2.  With k split, each run's sums go to `part` instead, [run][m][n].
struct ProductOut {
    bf16 *out, *out2;
    float *part;
    uint64_t ld, ld2;
    uint32_t split;
};
template <typename S> __global__ __launch_bounds__(S::THREADS) void product_kernel(const GemmArgs g, const ProductOut o)
{
    constexpr int NT = S::NT, COLS = NT * 32;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const TileAt at = tile_at(g.tiles_m, g.tiles_n, 1);
    f32x16 acc[S::MT][NT];
    gemm_tile<bf16, S, false>(g, at, lds, acc);
    const uint32_t wave = threadIdx.x >> 6;
    const uint32_t row0 = at.m * S::BM + (wave >> 1) * S::MT * 32, col0 = at.n * S::BN + (wave & 1u) * COLS;
    if (col0 >= g.n) return;
    char *stage = lds + wave * kStageBytes<float, COLS>;
    static_for<S::MT>([&](auto block) {
        constexpr int i = block.value;
        float v[NT][16];
        take(acc[i], v);
        auto value = [&](int j, int r) { return v[j][r]; };
        if (g.splits > 1) {
            store_32_rows<float, COLS>(stage, g.n - col0, value, [&](uint32_t r) {
                const uint32_t m = row0 + i * 32 + r;
                return m < g.m ? o.part + ((uint64_t)blockIdx.y * g.m + m) * g.n + col0 : nullptr;
            });
        } else {
            store_32_rows<bf16, COLS>(stage, g.n - col0, value, [&](uint32_t r) {
                const uint32_t m = row0 + i * 32 + r;
                bf16 *to = m < o.split ? o.out + (uint64_t)m * o.ld : o.out2 + (uint64_t)(m - o.split) * o.ld2;
                return m < g.m ? to + col0 : nullptr;
            });
        }
    });
}

// Adds the runs of a split product in their order.
__global__ void join_kernel(const ProductOut o, uint32_t m, uint32_t n, uint32_t splits)
{
    const uint64_t all = (uint64_t)m * n;
    for (uint64_t i = (uint64_t)blockIdx.x * blockDim.x + threadIdx.x; i < all; i += (uint64_t)gridDim.x * blockDim.x) {
        float v = o.part[i];
        for (uint32_t s = 1; s < splits; ++s) v += o.part[s * all + i];
        const uint32_t row = (uint32_t)(i / n), col = (uint32_t)(i % n);
        bf16 *to = row < o.split ? o.out + (uint64_t)row * o.ld : o.out2 + (uint64_t)(row - o.split) * o.ld2;
        to[col] = (bf16)v;
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
    // rows and columns are counted in 32 bits on the device
    if (d->dim < 1 || d->hidden < 1 || d->tokens > (1u << 30) || d->dim > (1u << 20) || d->hidden > (1u << 28)) return AR_ERR_ARG;
    const struct {
        size_t ld, cols, rows;
    } lds[] = {{d->ld_x, d->dim, d->tokens},       {d->ld_w_gate, d->dim, d->hidden}, {d->ld_w_up, d->dim, d->hidden},
               {d->ld_h, d->hidden, d->tokens},    {d->ld_dx, d->dim, d->tokens},     {d->ld_dw_gate, d->dim, d->hidden},
               {d->ld_dw_up, d->dim, d->hidden}};
    for (const auto &l : lds)
        if (l.ld && (l.ld < l.cols || l.ld > kOpsMaxSize / (l.rows ? l.rows : 1))) return AR_ERR_ARG;
    return AR_OK;
}

// Whether the product kernel can read a matrix where it lies.
bool direct(const Mat &m)
{
    return m.cols % kStepK == 0 && (uintptr_t)m.p % 16 == 0 && m.ld % 8 == 0 && gemm_reaches(m.ld * 2, m.cols * 2);
}
size_t packed_bytes(size_t rows, size_t cols) { return round_up(rows * round_up(cols, kStepK) * 2, 256); }

// A matrix as the product kernel takes it: itself, or a copy in the workspace.
struct Operand {
    const void *p;
    uint32_t ld;  // bytes
};

int pack(const Mat &m, char *&ws, hipStream_t st, Operand *out)
{
    if (direct(m)) {
        *out = {m.p, (uint32_t)(m.ld * 2)};
        return AR_OK;
    }
    const size_t to_ld = round_up(m.cols, kStepK);
    PackArgs p{(const bf16 *)m.p, (bf16 *)ws, m.rows, m.ld, to_ld, (uint32_t)m.cols};
    const uint64_t groups = (m.rows * (to_ld / 8) + 255) / 256;
    hipLaunchKernelGGL(pack_kernel, dim3((uint32_t)(groups < 8192 ? groups : 8192)), dim3(256), 0, st, p);
    *out = {ws, (uint32_t)(to_ld * 2)};
    ws += packed_bytes(m.rows, m.cols);
    return launch_status();
}

typedef Shape<4, 4, 1, 64, 2> Large;
typedef Shape<2, 2, 1, 64, 2> Small;

template <typename S, int ACT> int launch_ffn(GemmArgs &g, const FfnOut &o, hipStream_t st)
{
    g.tiles_m = (g.m + S::BM - 1) / S::BM;
    g.tiles_n = (g.n + S::BN / 2 - 1) / (S::BN / 2);
    static_assert(4 * kStageBytes<float, S::NT * 16> <= S::LDS, "the epilogue's staging fits");
    static const hipError_t set = hipFuncSetAttribute((const void *)ffn_kernel<S, ACT>, hipFuncAttributeMaxDynamicSharedMemorySize, S::LDS);
    if (set != hipSuccess) return AR_ERR_HIP;
    hipLaunchKernelGGL((ffn_kernel<S, ACT>), dim3(g.tiles_m * g.tiles_n), dim3(S::THREADS), S::LDS, st, g, o);
    return launch_status();
}

template <int ACT> int launch_ffn_tiles(GemmArgs &g, const FfnOut &o, hipStream_t st)
{
    const size_t large = (size_t)((g.m + 255) / 256) * ((g.n + 127) / 128);
    return large >= 256 ? launch_ffn<Large, ACT>(g, o, st) : launch_ffn<Small, ACT>(g, o, st);
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
    return packed_bytes(d.tokens, d.dim) + 2 * packed_bytes(d.hidden, d.dim);
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
    size_t need = 0;
    for (const Mat &in : {m.x, m.wg, m.wu})
        if (!direct(in)) need += packed_bytes(in.rows, in.cols);
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
    if ((rc = pack(m.x, at, st, &px)) != AR_OK || (rc = pack(m.wg, at, st, &pg)) != AR_OK || (rc = pack(m.wu, at, st, &pu)) != AR_OK)
        return rc;
    GemmArgs g{};
    g.a[0] = px.p, g.b[0] = pg.p, g.b2 = pu.p;
    g.lda = px.ld, g.ldb = pg.ld, g.ldb2 = pu.ld;
    g.segments = 1, g.steps = (uint32_t)(round_up(d.dim, kStepK) / kStepK);
    g.m = (uint32_t)d.tokens, g.n = (uint32_t)d.hidden, g.batch = 1, g.splits = 1;
    const FfnOut o{(bf16 *)h, saved, m.h.ld};
    switch (d.act) {
    case AR_ACT_SILU: return launch_ffn_tiles<AR_ACT_SILU>(g, o, st);
    case AR_ACT_GELU: return launch_ffn_tiles<AR_ACT_GELU>(g, o, st);
    default: return launch_ffn_tiles<AR_ACT_RELU>(g, o, st);
    }
}

// ---- backward ---------------------------------------------------------------

// A product's tile (64 * tile rows and columns) and the runs its k is split
// into.  Large tiles where they fill the device, else small ones; where even
// those leave most of it idle, k is split until they do not, in runs of at
// least four steps.
struct Cut {
    int tile;
    uint32_t splits;
};
Cut cut_of(size_t m, size_t n, size_t steps)
{
    const size_t large = ((m + 255) / 256) * ((n + 255) / 256), small = ((m + 127) / 128) * ((n + 127) / 128);
    if (large >= 256) return {4, 1};
    if (small >= 192) return {2, 1};
    size_t splits = 512 / small;
    if (splits > steps / 4) splits = steps / 4;
    if (splits > 64) splits = 64;
    return {2, (uint32_t)(splits ? splits : 1)};
}
size_t part_bytes(size_t m, size_t n, size_t steps)
{
    const Cut c = cut_of(m, n, steps);
    return c.splits > 1 ? round_up(c.splits * m * n * sizeof(float), 256) : 0;
}

template <typename S> int launch_product(GemmArgs &g, const ProductOut &o, hipStream_t st)
{
    g.tiles_m = (g.m + S::BM - 1) / S::BM;
    g.tiles_n = (g.n + S::BN - 1) / S::BN;
    constexpr int STAGE = 4 * kStageBytes<float, S::NT * 32>, LDS = S::LDS > STAGE ? S::LDS : STAGE;
    static const hipError_t set = hipFuncSetAttribute((const void *)product_kernel<S>, hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
    if (set != hipSuccess) return AR_ERR_HIP;
    hipLaunchKernelGGL((product_kernel<S>), dim3(g.tiles_m * g.tiles_n, g.splits), dim3(S::THREADS), LDS, st, g, o);
    int rc = launch_status();
    if (rc != AR_OK || g.splits == 1) return rc;
    const uint64_t groups = ((uint64_t)g.m * g.n + 255) / 256;
    hipLaunchKernelGGL(join_kernel, dim3((uint32_t)(groups < 4096 ? groups : 4096)), dim3(256), 0, st, o, g.m, g.n, g.splits);
    return launch_status();
}

int product(GemmArgs &g, const ProductOut &o, hipStream_t st)
{
    const Cut c = cut_of(g.m, g.n, (size_t)g.steps * g.segments);
    g.splits = c.splits, g.batch = 1;
    return c.tile == 4 ? launch_product<Large>(g, o, st) : launch_product<Small>(g, o, st);
}

int transpose(const Mat &m, void *to, size_t to_ld, hipStream_t st)
{
    TransposeArgs t{(const bf16 *)m.p, (bf16 *)to, m.ld, to_ld, (uint32_t)m.rows, (uint32_t)m.cols};
    hipLaunchKernelGGL(transpose_kernel, dim3((uint32_t)((m.cols + kTile - 1) / kTile), (uint32_t)(to_ld / kTile)), dim3(256), 0, st, t);
    return launch_status();
}

// Where the backward pass keeps what, in bytes from the workspace's start.
struct FfnBackwardSpace {
    size_t tokens_ld, hidden_ld;
    size_t by_rows, wg_t, wu_t, transposed, x_t, part, bytes;
};
FfnBackwardSpace ffn_backward_space(const ar_ffn_desc &d, bool dx, bool dw)
{
    FfnBackwardSpace s{};
    s.tokens_ld = round_up(d.tokens, kStepK), s.hidden_ld = round_up(d.hidden, kStepK);
    size_t at = 0, parts = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += round_up(bytes, 256);
        return here;
    };
    if (dx) {
        s.by_rows = take(d.tokens * 2 * s.hidden_ld * 2);
        s.wg_t = take(d.dim * s.hidden_ld * 2);
        s.wu_t = take(d.dim * s.hidden_ld * 2);
        parts = part_bytes(d.tokens, d.dim, 2 * s.hidden_ld / kStepK);
    }
    if (dw) {
        s.transposed = take(2 * d.hidden * s.tokens_ld * 2);
        s.x_t = take(d.dim * s.tokens_ld * 2);
        const size_t p = part_bytes(2 * d.hidden, d.dim, s.tokens_ld / kStepK);
        parts = p > parts ? p : parts;
    }
    s.part = take(parts);
    s.bytes = at;
    return s;
}

__global__ void zero_rows_kernel(bf16 *p, uint64_t rows, uint64_t cols, uint64_t ld)
{
    for (uint64_t i = (uint64_t)blockIdx.x * blockDim.x + threadIdx.x; i < rows * cols; i += (uint64_t)gridDim.x * blockDim.x)
        p[i / cols * ld + i % cols] = (bf16)0.0f;
}
int zero_rows(const Mat &m, hipStream_t st)
{
    const uint64_t groups = ((uint64_t)m.rows * m.cols + 255) / 256;
    hipLaunchKernelGGL(zero_rows_kernel, dim3((uint32_t)(groups < 4096 ? groups : 4096)), dim3(256), 0, st, (bf16 *)m.p, m.rows, m.cols, m.ld);
    return launch_status();
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
    const FfnBackwardSpace s = ffn_backward_space(d, dx != nullptr, dwg != nullptr);
    if (s.bytes == 0) return AR_OK;  // nothing wanted
    if (!ws || ws_bytes < s.bytes) return AR_ERR_SCRATCH;
    if ((uintptr_t)ws % 256 != 0) return AR_ERR_ARG;
    const Mat wsm{ws, 1, s.bytes, s.bytes, 1};
    for (const Mat &in : {m.x, m.wg, m.wu, m.h, sv, wsm})
        if (meet(odx, in) || meet(og, in) || meet(ou, in)) return AR_ERR_ARG;
    for (const Mat &in : {m.x, m.wg, m.wu, m.h, sv})
        if (meet(wsm, in)) return AR_ERR_ARG;

    char *w = (char *)ws;
    GradArgs ga{};
    ga.saved = saved, ga.dh = (const bf16 *)dh, ga.ld_dh = m.h.ld;
    ga.by_rows = dx ? (bf16 *)(w + s.by_rows) : nullptr;
    ga.transposed = dwg ? (bf16 *)(w + s.transposed) : nullptr;
    ga.hidden_ld = s.hidden_ld, ga.tokens_ld = s.tokens_ld, ga.tokens = (uint32_t)d.tokens, ga.hidden = (uint32_t)d.hidden;
    const dim3 grid((uint32_t)(s.hidden_ld / kTile), (uint32_t)(s.tokens_ld / kTile));
    switch (d.act) {
    case AR_ACT_SILU: hipLaunchKernelGGL((ffn_grad_kernel<AR_ACT_SILU>), grid, dim3(256), 0, st, ga); break;
    case AR_ACT_GELU: hipLaunchKernelGGL((ffn_grad_kernel<AR_ACT_GELU>), grid, dim3(256), 0, st, ga); break;
    default: hipLaunchKernelGGL((ffn_grad_kernel<AR_ACT_RELU>), grid, dim3(256), 0, st, ga);
    }
    if ((rc = launch_status()) != AR_OK) return rc;
    if (dx) {
        if ((rc = transpose(m.wg, w + s.wg_t, s.hidden_ld, st)) != AR_OK) return rc;
        if ((rc = transpose(m.wu, w + s.wu_t, s.hidden_ld, st)) != AR_OK) return rc;
        GemmArgs g{};
        g.segments = 2, g.steps = (uint32_t)(s.hidden_ld / kStepK);
        g.a[0] = w + s.by_rows, g.a[1] = w + s.by_rows + s.hidden_ld * 2;
        g.b[0] = w + s.wg_t, g.b[1] = w + s.wu_t;
        g.lda = (uint32_t)(s.hidden_ld * 4), g.ldb = (uint32_t)(s.hidden_ld * 2);
        g.m = (uint32_t)d.tokens, g.n = (uint32_t)d.dim;
        const ProductOut o{(bf16 *)dx, nullptr, (float *)(w + s.part), odx.ld, 0, (uint32_t)d.tokens};
        if ((rc = product(g, o, st)) != AR_OK) return rc;
    }
    if (dwg) {
        if ((rc = transpose(m.x, w + s.x_t, s.tokens_ld, st)) != AR_OK) return rc;
        GemmArgs g{};
        g.segments = 1, g.steps = (uint32_t)(s.tokens_ld / kStepK);
        g.a[0] = w + s.transposed, g.b[0] = w + s.x_t;
        g.lda = g.ldb = (uint32_t)(s.tokens_ld * 2);
        g.m = (uint32_t)(2 * d.hidden), g.n = (uint32_t)d.dim;
        const ProductOut o{(bf16 *)dwg, (bf16 *)dwu, (float *)(w + s.part), og.ld, ou.ld, (uint32_t)d.hidden};
        if ((rc = product(g, o, st)) != AR_OK) return rc;
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
    return ar::check_ffn(desc) == AR_OK && desc->tokens ? ar::ffn_backward_space(*desc, true, true).bytes : 0;
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
