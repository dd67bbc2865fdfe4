// Softmax cross entropy over a vocabulary, or a rank's rows of it (gfx950), without the
// logits in memory (formulas in ar_ops.h).
//
// Forward: one product kernel (gemm_nt.h) whose epilogue keeps, of a tile's logits, the
// maximum and the sum of e^(z - maximum) of each row's columns of a wave; a second
// kernel joins these.  Backward: the logits again, a piece of the vocabulary at a time,
// made into dz in registers and kept as bf16; then dx += dz W and dW = dz^T x of the
// piece as products of operands that are read where they lie.
//
// Bound by the products, and those by the board's power: 4096 tokens of 4096, 131072
// classes, forward 3540 us (1240 TFLOP/s), with gradients 14.5 ms (1210 TFLOP/s of what is
// done, the logits twice).  A few tokens by the weights' bytes: one of 4096, 131072
// classes, 200 us, 5.3 TB/s; 32768 classes 64 us, 4.2 TB/s.
#include "products.h"

#pragma clang fp contract(fast)

namespace ar {
namespace dev {

constexpr float kLog2e = 1.4426950408889634f;

struct Targets {
    const void *p;
    uint64_t first, classes;  // of the rows of the weight at hand; all there are
    bool wide;                // 64 bits
    // the class of a token; false: none, the token has no loss
    __device__ __forceinline__ bool get(uint64_t token, uint64_t *t) const
    {
        const int64_t v = wide ? ((const int64_t *)p)[token] : ((const int32_t *)p)[token];
        *t = (uint64_t)v;
        return *t < classes;  // negative ones are large
    }
};

// Statistics of a run of columns of one row: the sum is of e^(z - top).
struct Stat {
    float top, sum;
};
__device__ __forceinline__ Stat join(Stat a, Stat b)
{
    const float top = fmaxf(a.top, b.top), base = top == -INFINITY ? 0.0f : top;
    return {top, a.sum * __expf(a.top - base) + b.sum * __expf(b.top - base)};
}

struct StatsOut {
    Stat *stats;    // [run of columns][token]
    float *picked;  // [token]: the target's logit, where it is one of these columns
    Targets target;
};

template <typename S> __global__ __launch_bounds__(S::THREADS) void vocab_stats_kernel(const GemmArgs g, const StatsOut o)
{
    constexpr int NT = S::NT, COLS = NT * 32;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const TileAt at = tile_at(g.tiles_m, g.tiles_n, 1);
    f32x16 acc[S::MT][NT];
    gemm_tile<bf16, S, false>(g, at, lds, acc);
    const uint32_t wave = threadIdx.x >> 6, lane = threadIdx.x & 63u, h = lane >> 5;
    const uint32_t row0 = at.m * S::BM + (wave >> 1) * S::MT * 32, run = at.n * 2 + (wave & 1u), col0 = run * COLS;
    if (col0 >= g.n) return;
    const uint32_t cols = g.n - col0;
    static_for<S::MT>([&](auto block) {
        constexpr int i = block.value;
        float v[NT][16];
        take(acc[i], v);
        const uint32_t row = row0 + i * 32 + (lane & 31u);
        auto column = [&](int j, int r) { return (uint32_t)(j * 32 + 8 * (r / 4) + r % 4) + 4 * h; };
        if (cols < COLS) {
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (column(j, r) >= cols) v[j][r] = -INFINITY;
        }
        uint64_t t = 0;
        const bool counts = row < g.m && o.target.get(row, &t);
        const uint64_t place = t - o.target.first - col0;
        const bool here = counts && t >= o.target.first && place < (cols < COLS ? cols : COLS) && (place >> 2 & 1u) == h;
        if (__any(here)) {
            float z = 0.0f;
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (column(j, r) == (uint32_t)place) z = v[j][r];
            if (here) o.picked[row] = z;
        }
        float m[4] = {v[0][0], v[0][1], v[0][2], v[0][3]}, s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) m[r & 3] = fmaxf(m[r & 3], v[j][r]);
        float top = fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float base = top == -INFINITY ? 0.0f : top * kLog2e;
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r & 3] += __builtin_amdgcn_exp2f(v[j][r] * kLog2e - base);
        float sum = (s[0] + s[1]) + (s[2] + s[3]);
        sum += __shfl_xor(sum, 32);
        if (row < g.m && h == 0) o.stats[(uint64_t)run * g.m + row] = Stat{top, sum};
    });
}

// Joins the runs of columns of each token, TOKENS tokens to a workgroup, whose other
// threads have runs of their own, in one order whatever the timing.  One token of 32768
// classes: 512 runs, a token to a workgroup 4 us, sixteen 8.
struct JoinOut {
    const Stat *stats;
    const float *picked;
    Targets target;
    uint64_t rows;      // of the weight at hand
    uint32_t tokens, runs;
    float *loss, *lse, *logit;  // loss null: lse, and the target's logit, 0 where it is none of these rows
};
template <uint32_t TOKENS> __global__ __launch_bounds__(256) void vocab_join_kernel(const JoinOut o)
{
    constexpr uint32_t EACH = 256 / TOKENS;  // threads of a token
    __shared__ Stat part[TOKENS][EACH + 1];
    const uint32_t in = threadIdx.x % TOKENS, k0 = threadIdx.x / TOKENS, t = blockIdx.x * TOKENS + in;
    Stat s{-INFINITY, 0.0f};
    if (t < o.tokens)
        for (uint32_t k = k0; k < o.runs; k += 4 * EACH) {
            Stat a[4];
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) a[j] = k + EACH * j < o.runs ? o.stats[(uint64_t)(k + EACH * j) * o.tokens + t] : Stat{-INFINITY, 0.0f};
            s = join(s, join(join(a[0], a[1]), join(a[2], a[3])));
        }
    part[in][k0] = s;
#pragma unroll
    for (uint32_t half = EACH / 2; half; half /= 2) {
        __syncthreads();
        if (k0 < half) part[in][k0] = s = join(s, part[in][k0 + half]);
    }
    if (k0 || t >= o.tokens) return;
    uint64_t target = 0;
    const bool counts = o.target.get(t, &target);
    const bool here = counts && target >= o.target.first && target - o.target.first < o.rows;
    const float base = s.top == -INFINITY ? 0.0f : s.top, z = here ? o.picked[t] : 0.0f, log = __logf(s.sum);
    o.lse[t] = base + log;
    if (o.loss) o.loss[t] = counts ? log + (base - z) : 0.0f;
    else o.logit[t] = z;
}

// Joins the ranks' (lse, target's logit).
__global__ __launch_bounds__(256) void vocab_ranks_kernel(const float *parts, uint32_t ranks, uint32_t tokens, const Targets target, float *loss,
                                                          float *lse)
{
    const uint32_t t = blockIdx.x * 256 + threadIdx.x;
    if (t >= tokens) return;
    Stat s{-INFINITY, 0.0f};
    float z = 0.0f;
    for (uint32_t r = 0; r < ranks; ++r) {
        s = join(s, Stat{parts[(uint64_t)r * 2 * tokens + t], 1.0f});
        z += parts[((uint64_t)r * 2 + 1) * tokens + t];
    }
    uint64_t unused;
    const float base = s.top == -INFINITY ? 0.0f : s.top, log = __logf(s.sum);
    lse[t] = base + log;
    loss[t] = target.get(t, &unused) ? log + (base - z) : 0.0f;
}

// Which dloss gives dz its factor (below): that of the first token with a class whose
// dloss is a number and not 0.
struct LeadOf {
    const float *dloss;
    uint64_t stride;
    Targets target;
    uint32_t tokens;
    // a token's dloss, 0 if it cannot lead; both loads are on their way at once
    __device__ __forceinline__ float get(uint32_t t) const
    {
        const uint32_t at = t < tokens ? t : tokens - 1;
        uint64_t unused;
        const float v = dloss[at * stride];
        return target.get(at, &unused) && t < tokens && significand(v) < 1.0f ? v : 0.0f;
    }
};
// By a wave, 512 tokens at a time; 0 if there is none.
__device__ __forceinline__ float find_lead(const LeadOf &o)
{
    const uint32_t lane = threadIdx.x & 63u;
    for (uint32_t t0 = 0; t0 < o.tokens; t0 += 512) {
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = o.get(t0 + k * 64 + lane);
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (const uint64_t found = __ballot(v[k] != 0.0f)) return __shfl(v[k], __ffsll((unsigned long long)found) - 1);
    }
    return 0.0f;
}
// By a workgroup, 4096 at a time, where there are more tokens, or more waves, than each
// wave of the next kernel should look through.  3 to 4 us with the launch.
__global__ __launch_bounds__(1024) void vocab_lead_kernel(const LeadOf o, float *lead)
{
    __shared__ uint32_t first;
    if (threadIdx.x == 0) first = o.tokens;
    __syncthreads();
    for (uint32_t t0 = 0; t0 < o.tokens; t0 += 4096) {
        float v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = o.get(t0 + k * 1024 + threadIdx.x);
        uint32_t mine = o.tokens;  // the wave's first
#pragma unroll
        for (int k = 3; k >= 0; --k)
            if (const uint64_t found = __ballot(v[k] != 0.0f)) mine = t0 + k * 1024 + (threadIdx.x & ~63u) + __ffsll((unsigned long long)found) - 1;
        if (mine < o.tokens && (threadIdx.x & 63u) == 0) atomicMin(&first, mine);
        __syncthreads();
        const uint32_t found = first;
        __syncthreads();  // all have read it before any goes on
        if (found < o.tokens) break;
    }
    if (threadIdx.x == 0) *lead = first < o.tokens ? o.dloss[first * o.stride] : 0.0f;
}

// dz of a piece of the vocabulary: (e^(z - lse) - [target]) dloss / f, 0 for a token
// without a loss and up to the next multiple of eight columns.  f is the significand of
// one token's dloss, and the products with dz are multiplied by it in fp32.  With one
// dloss for all tokens, the mean's, most of dz's weight lies in targets' elements, all of
// them near -dloss: rounded to bf16, all would be off in one direction, and the gradients
// by as much (777 tokens of 5001 classes: by 2.6e-3 of their norm, so by 1.7e-3).  So the
// token has to be one that counts: tokens without a loss, a prompt's at the beginning
// say, may hold 0 or anything.
struct DzOut {
    bf16 *dz;
    uint64_t ld;
    const float *lse, *dloss;
    uint64_t dloss_stride;
    Targets target;  // first: of the piece
    uint32_t search; // tokens that the lead is looked for in, and left at `lead`; 0: it is there
    float *lead;
};
template <typename S> __global__ __launch_bounds__(S::THREADS) void vocab_dz_kernel(const GemmArgs g, const DzOut o)
{
    constexpr int NT = S::NT, COLS = NT * 32;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const TileAt at = tile_at(g.tiles_m, g.tiles_n, 1);
    f32x16 acc[S::MT][NT];
    gemm_tile<bf16, S, false>(g, at, lds, acc);
    const uint32_t wave = threadIdx.x >> 6, lane = threadIdx.x & 63u, h = lane >> 5;
    const uint32_t row0 = at.m * S::BM + (wave >> 1) * S::MT * 32, col0 = at.n * S::BN + (wave & 1u) * COLS;
    if (col0 >= g.n) return;
    const uint32_t cols = g.n - col0;
    char *stage = lds + wave * kStageBytes<bf16, COLS>;
    const float lead = o.search ? find_lead({o.dloss, o.dloss_stride, o.target, o.search}) : *o.lead, f = significand(lead);
    if (o.search && at.m == 0 && at.n == 0 && threadIdx.x == 0) *o.lead = lead;
    static_for<S::MT>([&](auto block) {
        constexpr int i = block.value;
        float v[NT][16];
        take(acc[i], v);
        const uint32_t first = row0 + i * 32;
        if (first >= g.m) return;
        const uint32_t row = first + (lane & 31u) < g.m ? first + (lane & 31u) : g.m - 1;
        uint64_t t;
        const bool counts = o.target.get(row, &t);
        const uint64_t place = t - o.target.first - col0;
        const uint32_t hit = counts && t >= o.target.first && place < COLS ? (uint32_t)place : 0xffffffffu;
        const float lse = o.lse[row] * kLog2e, by = o.dloss[row * o.dloss_stride] / f;
        stage_rows<bf16, COLS>(stage, [&](int j, int r) {
            const uint32_t c = (uint32_t)(j * 32 + 8 * (r / 4) + r % 4) + 4 * h;
            const float p = __builtin_amdgcn_exp2f(v[j][r] * kLog2e - lse);
            return counts && c < cols ? (p - (c == hit ? 1.0f : 0.0f)) * by : 0.0f;
        });
        write_rows<bf16, COLS>(stage, o.dz + (uint64_t)first * o.ld + col0, o.ld, 0, g.m - first, (cols + 7) / 8 * 8);
    });
}

}  // namespace dev

namespace {

using namespace dev;

int check_vocab(const ar_vocab_desc *d)
{
    if (!d) return AR_ERR_ARG;
    if (d->dtype != AR_BFLOAT16) return AR_ERR_UNSUPPORTED;
    if (d->target_bytes != 4 && d->target_bytes != 8) return AR_ERR_UNSUPPORTED;
    if (d->dim < 1 || d->rows < 1 || d->tokens > (1u << 24) || d->dim > (1u << 20) || d->rows > (1u << 26)) return AR_ERR_ARG;
    if (d->classes > (1ull << 40) || d->first > d->classes || d->rows > d->classes - d->first) return AR_ERR_ARG;
    // a launch's threads are counted in 32 bits
    if (d->tokens * d->rows > kOpsMaxSize / 4 || d->tokens * d->dim > kOpsMaxSize || d->rows * d->dim > kOpsMaxSize) return AR_ERR_ARG;
    const struct {
        size_t ld, rows;
    } lds[] = {{d->ld_x, d->tokens}, {d->ld_w, d->rows}, {d->ld_dx, d->tokens}, {d->ld_dw, d->rows}};
    for (const auto &l : lds)
        if (l.ld && (l.ld < d->dim || l.ld > kOpsMaxSize / (l.rows ? l.rows : 1))) return AR_ERR_ARG;
    return AR_OK;
}

struct VocabMats {
    Mat x, w, target;
};
VocabMats vocab_mats(const ar_vocab_desc &d, const void *x, const void *w, const void *target)
{
    return {mat(x, d.tokens, d.dim, d.ld_x, d.dtype), mat(w, d.rows, d.dim, d.ld_w, d.dtype), Mat{target, 1, d.tokens, d.tokens, (size_t)d.target_bytes}};
}
Targets targets(const ar_vocab_desc &d, const void *p) { return {p, d.first, d.classes, d.target_bytes == 8}; }

// Columns of a wave of the tile.
size_t wave_columns(int tile) { return tile == 0 ? 32 : tile == 2 ? 96 : tile == 3 ? 128 : 64; }
size_t runs_of(const ar_vocab_desc &d) { return (d.rows + wave_columns(logits_tile(d.tokens, d.dim, d.rows)) - 1) / wave_columns(logits_tile(d.tokens, d.dim, d.rows)); }

// Where the forward pass keeps what: the statistics, the targets' logits, copies.  The
// statistics, a 64th of the logits' bytes in fp32, are kept for so many tokens at a time
// that they stay within this, many rounds of tiles.
constexpr size_t kStatsBytes = (size_t)1 << 28;
struct VocabSpace {
    size_t tokens;  // at a time
    size_t picked, copies;
};
VocabSpace vocab_space(const ar_vocab_desc &d)
{
    VocabSpace s;
    const size_t runs = runs_of(d), most = kStatsBytes / (runs * sizeof(Stat)) / 256 * 256;
    s.tokens = d.tokens <= most ? d.tokens : most < 1024 ? 1024 : most;
    s.tokens = s.tokens < d.tokens ? s.tokens : d.tokens;
    s.picked = round_up(runs * s.tokens * sizeof(Stat), 256);
    s.copies = s.picked + round_up(s.tokens * sizeof(float), 256);
    return s;
}
size_t copy_bytes(const Mat &m) { return round_up(packed_bytes(m.rows, m.cols), 256); }
size_t vocab_need(const ar_vocab_desc &d, const VocabMats &m)
{
    return vocab_space(d).copies + (direct(m.x) ? 0 : copy_bytes(m.x)) + (direct(m.w) ? 0 : copy_bytes(m.w));
}

// x and w as the product kernels take them, and the product's sizes.
int logits_args(const ar_vocab_desc &d, const VocabMats &m, char *copies, GemmArgs *g, Operand *px, Operand *pw, hipStream_t st)
{
    PackList packs{};
    pack(m.x, direct(m.x), copies, &packs, px);
    copies = (char *)round_up((size_t)copies, 256);
    pack(m.w, direct(m.w), copies, &packs, pw);
    g->a[0] = px->p, g->b[0] = pw->p, g->lda = px->ld, g->ldb = pw->ld;
    g->segments = 1, g->steps = (uint32_t)(round_up(d.dim, kStepK) / kStepK);
    g->ka = g->kb = (uint32_t)round_up(d.dim, 8);
    g->m = (uint32_t)d.tokens, g->n = (uint32_t)d.rows, g->batch = 1, g->splits = 1;
    return run_packs(packs, st);
}

template <typename S, typename K, typename O> int launch_logits(OncePerDevice &once, K kernel, GemmArgs &g, const O &o, hipStream_t st)
{
    g.tiles_m = (g.m + S::BM - 1) / S::BM, g.tiles_n = (g.n + S::BN - 1) / S::BN;
    static_assert(4 * kStageBytes<bf16, S::NT * 32> <= S::LDS, "the epilogue's staging fits");
    const int rc = allow_lds(once, (const void *)kernel, S::LDS);
    if (rc != AR_OK) return rc;
    hipLaunchKernelGGL(kernel, dim3(g.tiles_m * g.tiles_n), dim3(S::THREADS), S::LDS, st, g, o);
    return launch_status();
}
template <typename S> int launch_stats(GemmArgs &g, const StatsOut &o, hipStream_t st)
{
    static OncePerDevice once;
    return launch_logits<S>(once, vocab_stats_kernel<S>, g, o, st);
}
template <typename S> int launch_dz(GemmArgs &g, const DzOut &o, hipStream_t st)
{
    static OncePerDevice once;
    return launch_logits<S>(once, vocab_dz_kernel<S>, g, o, st);
}

int vocab_loss(const ar_vocab_desc *desc, const void *x, const void *w, const void *target, float *loss, float *lse, void *ws, size_t ws_bytes,
               void *stream)
{
    int rc = check_vocab(desc);
    if (rc != AR_OK) return rc;
    const ar_vocab_desc &d = *desc;
    if (loss && (d.first != 0 || d.rows != d.classes)) return AR_ERR_ARG;
    if (d.tokens == 0) return AR_OK;
    const VocabMats m = vocab_mats(d, x, w, target);
    if (!m.x.ok() || !m.w.ok() || !m.target.ok() || !lse || (uintptr_t)lse % 4 != 0 || (uintptr_t)loss % 4 != 0) return AR_ERR_ARG;
    const Mat lm = mat(lse, loss ? 1 : 2, d.tokens, 0, AR_FLOAT32), om = mat(loss, 1, d.tokens, 0, AR_FLOAT32);
    const size_t need = vocab_need(d, m);
    if (!ws || ws_bytes < need) return AR_ERR_SCRATCH;
    if ((uintptr_t)ws % 256 != 0) return AR_ERR_ARG;
    const Mat wm{ws, 1, need, need, 1};
    for (const Mat &in : {m.x, m.w, m.target, wm})
        if (meet(lm, in) || meet(om, in)) return AR_ERR_ARG;
    for (const Mat &in : {m.x, m.w, m.target})
        if (meet(wm, in)) return AR_ERR_ARG;
    if (meet(lm, om)) return AR_ERR_ARG;

    hipStream_t st = (hipStream_t)stream;
    const VocabSpace s = vocab_space(d);
    GemmArgs g{};
    Operand px, pw;
    if ((rc = logits_args(d, m, (char *)ws + s.copies, &g, &px, &pw, st)) != AR_OK) return rc;
    const int tile = logits_tile(d.tokens, d.dim, d.rows);
    for (size_t first = 0; first < d.tokens; first += s.tokens) {
        const size_t tokens = d.tokens - first < s.tokens ? d.tokens - first : s.tokens;
        GemmArgs gb = g;
        gb.a[0] = (const char *)px.p + first * px.ld, gb.m = (uint32_t)tokens;
        StatsOut o{(Stat *)ws, (float *)((char *)ws + s.picked), targets(d, target)};
        o.target.p = (const char *)target + first * d.target_bytes;
        switch (tile) {
        case kFewTokens: rc = launch_stats<Flat>(gb, o, st); break;
        case 0: rc = launch_stats<Tiny>(gb, o, st); break;
        case 1: rc = launch_stats<Small>(gb, o, st); break;
        case 2: rc = launch_stats<Middle>(gb, o, st); break;
        case 3: rc = launch_stats<Large>(gb, o, st); break;
        default: rc = launch_stats<Deep>(gb, o, st);
        }
        if (rc != AR_OK) return rc;
        const JoinOut j{o.stats, o.picked, o.target, d.rows, (uint32_t)tokens, (uint32_t)runs_of(d), loss ? loss + first : nullptr, lse + first,
                        loss ? nullptr : lse + d.tokens + first};
        if (tokens <= 64) hipLaunchKernelGGL((vocab_join_kernel<1>), dim3((uint32_t)tokens), dim3(256), 0, st, j);
        else hipLaunchKernelGGL((vocab_join_kernel<16>), dim3((uint32_t)((tokens + 15) / 16)), dim3(256), 0, st, j);
        if ((rc = launch_status()) != AR_OK) return rc;
    }
    return AR_OK;
}

int vocab_join(const ar_vocab_desc *desc, size_t ranks, const float *parts, const void *target, float *loss, float *lse, void *stream)
{
    const int rc = check_vocab(desc);
    if (rc != AR_OK) return rc;
    const ar_vocab_desc &d = *desc;
    if (ranks < 1 || ranks > (1u << 16)) return AR_ERR_ARG;
    if (d.tokens == 0) return AR_OK;
    const Mat pm = mat(parts, 2 * ranks, d.tokens, 0, AR_FLOAT32), om = mat(loss, 1, d.tokens, 0, AR_FLOAT32), lm = mat(lse, 1, d.tokens, 0, AR_FLOAT32),
              tm{target, 1, d.tokens, d.tokens, (size_t)d.target_bytes};
    if (!pm.ok() || !om.ok() || !lm.ok() || !tm.ok()) return AR_ERR_ARG;
    if (meet(om, pm) || meet(om, tm) || meet(lm, pm) || meet(lm, tm) || meet(om, lm)) return AR_ERR_ARG;
    hipLaunchKernelGGL(vocab_ranks_kernel, dim3((uint32_t)((d.tokens + 255) / 256)), dim3(256), 0, (hipStream_t)stream, parts, (uint32_t)ranks,
                       (uint32_t)d.tokens, targets(d, target), loss, lse);
    return launch_status();
}

// ---- backward -------------------------------------------------------------------

// Whether each wave that makes dz looks for the lead by itself: where there are few tokens
// to look through, eight looks at most, and few rounds of tiles that all do so, which is
// less than a launch.  Gradients of 1025 x 1024 x 8192, 98.4 us with the first dloss taken as
// it is: by waves 99, where only the last quarter of the tokens counts 96 (from 93.4); 4097 x
// 512 x 4096, 114.5: by a launch 118.
bool lead_by_waves(const ar_vocab_desc &d) { return d.tokens <= 4096 && d.tokens * d.rows <= (size_t)1 << 24; }

// Where the backward pass keeps what; dz lies at the start, copies behind the rest.
struct VocabBackwardSpace : VocabCut {
    size_t lead;                      // the dloss that gives dz its factor
    size_t part_dx, part_dw, copies;  // with one piece one place after the other
};
VocabBackwardSpace vocab_backward_space(const ar_vocab_desc &d, bool dx, bool dw)
{
    VocabBackwardSpace s{};
    (VocabCut &)s = vocab_cut(d.tokens, d.dim, d.rows);
    s.lead = round_up(d.tokens * s.ld * 2, 256);
    s.part_dx = s.part_dw = s.copies = s.lead + 256;
    const bool several = s.pieces > 1;  // dx's sums stay from piece to piece
    if (dx) {
        s.copies += several ? round_up(s.dx.splits * d.tokens * d.dim * sizeof(float), 256) : part_bytes(s.dx, d.tokens, d.dim);
        if (several) s.part_dw = s.copies;
    }
    if (dw) {
        const size_t end = s.part_dw + part_bytes(s.dw, round_up(s.piece, 8), d.dim);
        s.copies = end > s.copies ? end : s.copies;
    }
    return s;
}
size_t vocab_backward_need(const ar_vocab_desc &d, const VocabMats &m, bool dx, bool dw)
{
    return vocab_backward_space(d, dx, dw).copies + (direct(m.x) ? 0 : copy_bytes(m.x)) + (direct(m.w) ? 0 : copy_bytes(m.w));
}

int vocab_backward(const ar_vocab_desc *desc, const float *dloss, size_t dloss_stride, const void *x, const void *w, const void *target,
                   const float *lse, void *dx, void *dw, void *ws, size_t ws_bytes, void *stream)
{
    int rc = check_vocab(desc);
    if (rc != AR_OK) return rc;
    const ar_vocab_desc &d = *desc;
    hipStream_t st = (hipStream_t)stream;
    if (!dx && !dw) return AR_OK;
    const Mat odx = mat(dx, d.tokens, d.dim, d.ld_dx, d.dtype), odw = mat(dw, d.rows, d.dim, d.ld_dw, d.dtype);
    if (!odx.aligned() || !odw.aligned() || meet(odx, odw)) return AR_ERR_ARG;
    if (d.tokens == 0) return dw ? zero_rows(odw, st) : AR_OK;  // sums over no tokens
    const VocabMats m = vocab_mats(d, x, w, target);
    const Mat gm{dloss, d.tokens, 1, dloss_stride, 4}, lm = mat(lse, 1, d.tokens, 0, AR_FLOAT32);
    if (dloss_stride > kOpsMaxSize / d.tokens) return AR_ERR_ARG;
    if (!m.x.ok() || !m.w.ok() || !m.target.ok() || !gm.ok() || !lm.ok()) return AR_ERR_ARG;
    const size_t need = vocab_backward_need(d, m, dx != nullptr, dw != nullptr);
    if (!ws || ws_bytes < need) return AR_ERR_SCRATCH;
    if ((uintptr_t)ws % 256 != 0) return AR_ERR_ARG;
    const Mat wm{ws, 1, need, need, 1};
    for (const Mat &in : {m.x, m.w, m.target, gm, lm, wm})
        if (meet(odx, in) || meet(odw, in)) return AR_ERR_ARG;
    for (const Mat &in : {m.x, m.w, m.target, gm, lm})
        if (meet(wm, in)) return AR_ERR_ARG;

    const VocabBackwardSpace s = vocab_backward_space(d, dx != nullptr, dw != nullptr);
    bf16 *dz = (bf16 *)ws;
    float *part_dx = (float *)((char *)ws + s.part_dx), *part_dw = (float *)((char *)ws + s.part_dw);
    GemmArgs logits{};
    Operand px, pw;
    if ((rc = logits_args(d, m, (char *)ws + s.copies, &logits, &px, &pw, st)) != AR_OK) return rc;
    float *lead = dloss_stride ? (float *)((char *)ws + s.lead) : (float *)dloss;  // one dloss for all leads itself
    const bool by_waves = lead_by_waves(d);
    if (dloss_stride && !by_waves) {
        hipLaunchKernelGGL(vocab_lead_kernel, dim3(1), dim3(1024), 0, st, LeadOf{dloss, dloss_stride, targets(d, target), (uint32_t)d.tokens}, lead);
        if ((rc = launch_status()) != AR_OK) return rc;
    }
    const ProductOut to_dx{{(bf16 *)dx, nullptr}, part_dx, {odx.ld, 0}, 0x80000000u, (uint32_t)d.tokens, (uint32_t)d.dim, false, lead};
    for (size_t k = 0; k < s.pieces; ++k) {
        const size_t first = k * s.piece, rows = d.rows - first < s.piece ? d.rows - first : s.piece;
        const char *wk = (const char *)pw.p + first * pw.ld;
        GemmArgs g = logits;
        g.b[0] = wk, g.n = (uint32_t)rows;
        DzOut o{dz, s.ld, lse, dloss, dloss_stride, targets(d, target), dloss_stride && by_waves ? (uint32_t)d.tokens : 0, lead};
        o.target.first += first;
        switch (logits_tile(d.tokens, d.dim, rows)) {
        case kFewTokens: rc = launch_dz<Flat>(g, o, st); break;
        case 0: rc = launch_dz<Tiny>(g, o, st); break;
        case 1: rc = launch_dz<Small>(g, o, st); break;
        case 2: rc = launch_dz<Middle>(g, o, st); break;
        case 3: rc = launch_dz<Large>(g, o, st); break;
        default: rc = launch_dz<Deep>(g, o, st);
        }
        if (rc != AR_OK) return rc;
        if (dx) {
            GemmArgs p{};
            p.segments = 1, p.steps = (uint32_t)(round_up(rows, kStepK) / kStepK);
            p.ka = (uint32_t)round_up(rows, 8), p.kb = (uint32_t)rows;
            p.a[0] = dz, p.b[0] = wk, p.lda = (uint32_t)(s.ld * 2), p.ldb = pw.ld;
            p.m = (uint32_t)d.tokens, p.n = pw.cols;
            ProductOut out = to_dx;
            out.more = k > 0;
            Cut cut = s.dx;
            if (cut.splits > p.steps) cut.splits = p.steps;  // a short last piece: the other runs' sums stay
            rc = s.pieces > 1 ? product<false, true, true>(cut, p, out, st) : product<false, false, true>(cut, p, out, st);
            if (rc != AR_OK) return rc;
        }
        if (dw) {
            GemmArgs p{};
            p.segments = 1, p.steps = (uint32_t)((d.tokens + kStepK - 1) / kStepK);
            p.ka = p.kb = (uint32_t)d.tokens;
            p.a[0] = dz, p.b[0] = px.p, p.lda = (uint32_t)(s.ld * 2), p.ldb = px.ld;
            p.m = (uint32_t)round_up(rows, 8), p.n = px.cols;
            const ProductOut out{{(bf16 *)dw + first * odw.ld, nullptr}, part_dw, {odw.ld, 0}, 0x80000000u, (uint32_t)rows, (uint32_t)d.dim, false, lead};
            if ((rc = product<true, false, true>(s.dw, p, out, st)) != AR_OK) return rc;
        }
    }
    return dx && s.pieces > 1 ? run_join<true>(to_dx, (uint32_t)d.tokens, s.dx.splits, st) : AR_OK;
}

}  // namespace
}  // namespace ar

extern "C" int ar_vocab_loss(const ar_vocab_desc *desc, const void *x, const void *w, const void *target, float *loss, float *lse,
                             void *workspace, size_t workspace_bytes, void *stream)
{
    return ar::ops_ret(loss ? ar::vocab_loss(desc, x, w, target, loss, lse, workspace, workspace_bytes, stream)
                            : desc && desc->tokens == 0 ? ar::check_vocab(desc) : AR_ERR_ARG);
}

extern "C" int ar_vocab_loss_part(const ar_vocab_desc *desc, const void *x, const void *w, const void *target, float *part, void *workspace,
                                  size_t workspace_bytes, void *stream)
{
    return ar::ops_ret(ar::vocab_loss(desc, x, w, target, nullptr, part, workspace, workspace_bytes, stream));
}

extern "C" int ar_vocab_loss_join(const ar_vocab_desc *desc, size_t ranks, const float *parts, const void *target, float *loss, float *lse,
                                  void *stream)
{
    return ar::ops_ret(ar::vocab_join(desc, ranks, parts, target, loss, lse, stream));
}

extern "C" size_t ar_vocab_loss_workspace(const ar_vocab_desc *desc, const void *x, const void *w)
{
    return ar::check_vocab(desc) == AR_OK && desc->tokens ? ar::vocab_need(*desc, ar::vocab_mats(*desc, x, w, nullptr)) : 0;
}

extern "C" int ar_vocab_loss_backward(const ar_vocab_desc *desc, const float *dloss, size_t dloss_stride, const void *x, const void *w,
                                      const void *target, const float *lse, void *dx, void *dw, void *workspace, size_t workspace_bytes,
                                      void *stream)
{
    return ar::ops_ret(ar::vocab_backward(desc, dloss, dloss_stride, x, w, target, lse, dx, dw, workspace, workspace_bytes, stream));
}

extern "C" size_t ar_vocab_loss_backward_workspace(const ar_vocab_desc *desc, const void *x, const void *w, int dx, int dw)
{
    return ar::check_vocab(desc) == AR_OK && desc->tokens ? ar::vocab_backward_need(*desc, ar::vocab_mats(*desc, x, w, nullptr), dx, dw) : 0;
}
