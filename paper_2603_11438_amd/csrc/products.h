// Plain bf16 products on the matrix units, C = A B with B by k, and what stands around
// them: copies of operands that cannot be read where they lie, runs of k and their join.
// Shared by the gated feed-forward block and the loss over a vocabulary.
#pragma once

#include "gemm_nt.h"

namespace ar {
namespace dev {

// Copies matrices into rows of `to_ld` elements, zeros behind their columns; all of
// a call's in one launch (5 x 4357 x 157 forward, three of them: 22 us, in three
// launches 27).
struct PackArgs {
    const bf16 *from;
    bf16 *to;
    uint64_t rows, ld, to_ld;
    uint32_t cols;
};
struct PackList {
    PackArgs p[3];
    uint32_t n;
};
static __global__ __launch_bounds__(256) void pack_kernel(const PackList list)
{
    const PackArgs p = list.p[blockIdx.y];
    const uint64_t per = p.to_ld / 8, n = p.rows * per;
    for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (uint64_t)gridDim.x * 256) {
        const uint64_t row = i / per;
        const uint32_t c = (uint32_t)(i % per) * 8;
        const bf16 *from = p.from + row * p.ld + c;
        float v[8];
        if (c + 8 <= p.cols) load_vec<bf16, 8>(from, v);
        else load_part<bf16, 8>(from, (int)p.cols - (int)c, v);
        store_vec<bf16, 8>(p.to + row * p.to_ld + c, v);
    }
}

// Adds staged rows of sums to `out` and the rows behind it: the first `rows` and `cols`.
template <int COLS> __device__ __forceinline__ void add_rows(const char *lds, float *out, uint64_t ld, uint32_t rows, uint32_t cols)
{
    constexpr int PITCH = kStagePitch<float, COLS>, LANES = COLS / 4;
    const uint32_t lane = threadIdx.x & 63u;
#pragma unroll
    for (int k0 = 0; k0 < 32 * LANES; k0 += 64) {
        const uint32_t r = (k0 + lane) / LANES, c = (k0 + lane) % LANES * 4;
        if (r >= rows || c >= cols) continue;
        float *to = out + r * ld + c, v[4];
        const float *at = (const float *)(lds + r * PITCH + c * 4);
        if (c + 4 <= cols) {
            load_vec<float, 4>(to, v);
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] += at[k];
            store_vec<float, 4>(to, v);
        } else {
            for (uint32_t k = c; k < cols; ++k) to[k - c] += at[k - c];
        }
    }
}

// A plain product.  Its rows belong to results of `half` rows each (a multiple
// of 32), of which the first `rows` exist: one result, or dWg and then dWu.
// With k split, each run's sums go to `part` instead, [run][m][cols].  ADD: one of
// several products that make up a result: its sums go to `part` however many runs there
// are, and with `more` are added to what is there.  BY: results are multiplied by
// factor(by) before they are rounded (not what goes to `part`).
struct ProductOut {
    bf16 *out[2];
    float *part;
    uint64_t ld[2];
    uint32_t half, rows, cols;
    bool more;
    const float *by;
};
// The significand, in [1/2, 1), of a value; 1 for one that has none (0, an infinity, NaN).
__device__ __forceinline__ float significand(float v)
{
    const float m = fabsf(__builtin_amdgcn_frexp_mantf(v));
    return m >= 0.5f && m < 1.0f ? m : 1.0f;
}
__device__ __forceinline__ float factor(const float *p) { return significand(*p); }
template <typename S, bool ABYK, bool ADD = false, bool BY = false> __global__ __launch_bounds__(S::THREADS) void product_kernel(const GemmArgs g, const ProductOut o)
{
    constexpr int NT = S::NT, COLS = NT * 32;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const TileAt at = tile_at(g.tiles_m, g.tiles_n, 1);
    f32x16 acc[S::MT][NT];
    gemm_tile<bf16, S, false, ABYK, true>(g, at, lds, acc);
    const uint32_t wave = threadIdx.x >> 6;
    const uint32_t row0 = at.m * S::BM + (wave >> 1) * S::MT * 32, col0 = at.n * S::BN + (wave & 1u) * COLS;
    if (col0 >= o.cols) return;
    char *stage = lds + wave * kStageBytes<float, COLS>;
    static_for<S::MT>([&](auto block) {
        constexpr int i = block.value;
        float v[NT][16];
        take(acc[i], v);
        const uint32_t first = row0 + i * 32, which = first >= o.half, r = first - which * o.half;
        if (first >= g.m || r >= o.rows) return;
        auto value = [&](int j, int q) { return v[j][q]; };
        const float by = BY ? factor(o.by) : 1.0f;
        if (ADD && o.more) {
            stage_rows<float, COLS>(stage, value);
            add_rows<COLS>(stage, o.part + ((uint64_t)blockIdx.y * g.m + first) * o.cols + col0, o.cols, o.rows - r, o.cols - col0);
        } else if (ADD || g.splits > 1) {
            stage_rows<float, COLS>(stage, value);
            write_rows<float, COLS>(stage, o.part + ((uint64_t)blockIdx.y * g.m + first) * o.cols + col0, o.cols, 0, o.rows - r,
                                    o.cols - col0);
        } else {
            stage_rows<bf16, COLS>(stage, [&](int j, int q) { return BY ? v[j][q] * by : v[j][q]; });
            write_rows<bf16, COLS>(stage, o.out[which] + (uint64_t)r * o.ld[which] + col0, o.ld[which], 0, o.rows - r, o.cols - col0);
        }
    });
}

// Adds the runs of a split product in their order, four columns a thread.
template <bool BY> __global__ __launch_bounds__(256) void join_kernel(const ProductOut o, uint32_t m, uint32_t splits)
{
    const uint64_t all = (uint64_t)m * o.cols, per = (o.cols + 3) / 4, n = m * per;
    const float by = BY ? factor(o.by) : 1.0f;
    for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (uint64_t)gridDim.x * 256) {
        const uint32_t row = (uint32_t)(i / per), c = (uint32_t)(i % per) * 4, which = row >= o.half, r = row - which * o.half;
        if (r >= o.rows) continue;
        const float *from = o.part + (uint64_t)row * o.cols + c;
        bf16 *to = o.out[which] + (uint64_t)r * o.ld[which] + c;
        float v[4], w[4];
        if (c + 4 <= o.cols) {
            load_vec<float, 4>(from, v);
#pragma unroll 4
            for (uint32_t s = 1; s < splits; ++s) {
                load_vec<float, 4>(from + s * all, w);
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] += w[k];
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = BY ? v[k] * by : v[k];
            store_vec<bf16, 4>(to, v);
        } else {
            for (uint32_t k = 0; k < o.cols - c; ++k) {
                float t = from[k];
                for (uint32_t s = 1; s < splits; ++s) t += from[s * all + k];
                to[k] = (bf16)(BY ? t * by : t);
            }
        }
    }
}

static __global__ void zero_rows_kernel(bf16 *p, uint64_t rows, uint64_t cols, uint64_t ld)
{
    for (uint64_t i = (uint64_t)blockIdx.x * blockDim.x + threadIdx.x; i < rows * cols; i += (uint64_t)gridDim.x * blockDim.x)
        p[i / cols * ld + i % cols] = (bf16)0.0f;
}

}  // namespace dev

namespace {

using namespace dev;

// Whether the product kernel can read a matrix where it lies.
inline bool direct(const Mat &m)
{
    return (uintptr_t)m.p % 16 == 0 && m.ld % 8 == 0 && m.cols % 8 == 0 && gemm_reaches(m.ld * 2, m.cols * 2);
}
// A copy's rows begin at 128 bytes: a load of 64 elements is one line of the
// cache then, else two (64 to 66 bytes a ns to a compute unit instead of 125;
// 2000 x 1999 x 5001 forward 112 us, with rows of whole 16 bytes alone 17 more).
constexpr size_t kLine = 64;
inline size_t packed_bytes(size_t rows, size_t cols) { return rows * round_up(cols, kLine) * 2; }

// A matrix as the product kernel takes it: itself, or a copy in the workspace.
struct Operand {
    const void *p;
    uint32_t ld;    // bytes
    uint32_t cols;  // that can be read
};

inline void pack(const Mat &m, bool as_is, char *&ws, PackList *list, Operand *out)
{
    if (as_is) {
        *out = {m.p, (uint32_t)(m.ld * 2), (uint32_t)m.cols};
        return;
    }
    const size_t to_ld = round_up(m.cols, kLine);
    list->p[list->n++] = PackArgs{(const bf16 *)m.p, (bf16 *)ws, m.rows, m.ld, to_ld, (uint32_t)m.cols};
    *out = {ws, (uint32_t)(to_ld * 2), (uint32_t)round_up(m.cols, 8)};
    ws += packed_bytes(m.rows, m.cols);
}
inline int run_packs(const PackList &list, hipStream_t st)
{
    if (!list.n) return AR_OK;
    uint64_t groups = 0;
    for (uint32_t k = 0; k < list.n; ++k) {
        const uint64_t here = (list.p[k].rows * (list.p[k].to_ld / 8) + 255) / 256;
        groups = here > groups ? here : groups;
    }
    hipLaunchKernelGGL(pack_kernel, dim3((uint32_t)(groups < 8192 ? groups : 8192), list.n), dim3(256), 0, st, list);
    return launch_status();
}

typedef Shape<4, 4, 1, 64, 2, 2, true> Large;
typedef Shape<4, 4, 1, 64, 2> LargeEven;  // with two buffers of each operand
typedef Shape<3, 3, 1, 64, 2> Middle;
typedef Shape<2, 2, 1, 64, 2> Small;
typedef Shape<1, 1, 1, 64, 4> Tiny;
typedef Shape<2, 2, 1, 64, 3> Deep;  // 128 x 128 alone on its compute unit
typedef Shape<1, 2, 1, 64, 3> Flat;  // 64 tokens, both projections of 64 columns

inline size_t part_bytes(const Cut &c, size_t m, size_t cols)
{
    return c.splits > 1 ? round_up(c.splits * m * cols * sizeof(float), 256) : 0;
}

template <bool BY> int run_join(const ProductOut &o, uint32_t m, uint32_t splits, hipStream_t st)
{
    const uint64_t groups = ((uint64_t)m * ((o.cols + 3) / 4) + 255) / 256;
    hipLaunchKernelGGL((join_kernel<BY>), dim3((uint32_t)(groups < 8192 ? groups : 8192)), dim3(256), 0, st, o, m, splits);
    return launch_status();
}

// ADD: the caller joins once all products are there.
template <typename S, bool ABYK, bool ADD, bool BY> int launch_product(GemmArgs &g, const ProductOut &o, hipStream_t st)
{
    g.tiles_m = (g.m + S::BM - 1) / S::BM;
    g.tiles_n = (o.cols + S::BN - 1) / S::BN;
    constexpr int STAGE = 4 * kStageBytes<float, S::NT * 32>, LDS = S::LDS > STAGE ? S::LDS : STAGE;
    static OncePerDevice once;
    int rc = allow_lds(once, (const void *)product_kernel<S, ABYK, ADD, BY>, LDS);
    if (rc != AR_OK) return rc;
    hipLaunchKernelGGL((product_kernel<S, ABYK, ADD, BY>), dim3(g.tiles_m * g.tiles_n, g.splits), dim3(S::THREADS), LDS, st, g, o);
    rc = launch_status();
    return rc != AR_OK || g.splits == 1 || ADD ? rc : run_join<BY>(o, g.m, g.splits, st);
}

// B by k; A by rows (dx) or by k (the weights' gradients).
template <bool ABYK, bool ADD = false, bool BY = false> int product(const Cut &c, GemmArgs &g, const ProductOut &o, hipStream_t st)
{
    g.splits = c.splits, g.batch = 1;
    switch (c.tile) {
    case 0: return launch_product<Tiny, ABYK, ADD, BY>(g, o, st);
    case 1: return launch_product<Small, ABYK, ADD, BY>(g, o, st);
    case 2: return launch_product<Middle, ABYK, ADD, BY>(g, o, st);
    case 3: return launch_product<Large, ABYK, ADD, BY>(g, o, st);
    default: return launch_product<Deep, ABYK, ADD, BY>(g, o, st);
    }
}

inline int zero_rows(const Mat &m, hipStream_t st)
{
    const uint64_t groups = ((uint64_t)m.rows * m.cols + 255) / 256;
    hipLaunchKernelGGL(zero_rows_kernel, dim3((uint32_t)(groups < 4096 ? groups : 4096)), dim3(256), 0, st, (bf16 *)m.p, m.rows, m.cols, m.ld);
    return launch_status();
}

}  // namespace
}  // namespace ar
