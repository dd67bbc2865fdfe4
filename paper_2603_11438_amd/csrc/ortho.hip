// Newton-Schulz orthogonalisation (gfx950): steps of three matrix products,
//     A = X X^T,  B = b A + c A A,  X = a X + B X   (ar_ops.h),
// on the matrix units through gemm_nt.h, with fp16 operands and fp32 sums.
//
// Operands.  A value v is held as hi = fp16(v s) and lo = fp16(v s - hi) with a
// power of two s chosen from a bound on |v|: 11 bits, or 22 with lo.
//   fp32 matrices: products of hi and lo, hi hi + hi lo + lo hi, and X also in
//   fp32 for the a X term.
//   bf16 matrices: products of hi alone, one third of the work.  What a single
//   plane would lose is kept out of the products, or kept from adding up: X itself
//   has both planes for the a X term (a strong direction's rounding error would
//   otherwise swamp weak directions, which the steps amplify up to a^steps = 485
//   times); the diagonals of A and B, on which most of their norm sits, stay in
//   fp32, A's from the rows of both planes: with A = D + O, D diagonal,
//     A A = D D + D O + O D + O O,   a X + B X = (a + diag B) X + (B - diag B) X;
//   and values among equals are rounded at random (round_alike).
//   The result's error before its rounding to bf16 (1.7e-3 of its norm, up to
//   3.9e-3), with every rounding modelled in 64 bits: 0.2e-3 to 0.9e-3 of its norm
//   for matrices of full rank, up to 1.8e-3 for those of low rank, up to 2.8e-3 where
//   rows hold few magnitudes or few elements (identity, constant, signs, blocks of
//   ones, repeated columns: 50 kinds in all).  Without these measures up to 1.8e-2.
//   Small matrices, whose few singular values do not average such errors, take
//   two planes in bf16 too.
//
// A and B are symmetric: only tiles on and below the diagonal are computed and
// written to both places.  Tall matrices are transposed on the way in and out.
//
// Five steps of 4096 x 4096 bf16: 1600 us, 860 TFLOP/s (a step's A 84 us, B 88, X
// 150, of which 40 the epilogue's bytes); six of 1410 x 700 bf16: 250 us; 1024 x
// 4096 fp32: 395 us, 530 TFLOP/s of fp16 products; 128 x 384 fp32: 97 us.  The small
// ones are bound by no unit (matrix units busy 11 to 45 % of the cycles, the LDS 30 to
// 45 %) but by what one or two rounds of tiles leave in the open: first loads,
// epilogues, launches.
#include <type_traits>

#include "gemm_nt.h"

#pragma clang fp contract(fast)

namespace ar {
namespace dev {

constexpr uint32_t kNormParts = 256;  // partial sums of squares of a matrix, at most

// Scales of one step: X in (2^14 for the input), A, B, and the factor that the
// step's X planes stand to the true X (1 but for the first step).
struct Scales {
    float x, a, b, tau;
};

// One matrix' part of the workspace, in bytes.
struct OrthoSpace {
    size_t x[2], x_lo, xf, a, a_lo, b, b_lo, diag_a, diag_b, squares, part, scales, norms, bytes;
};

struct OrthoArgs {
    const void *in;
    void *out;
    char *ws;
    OrthoSpace at;
    uint64_t ld_in, ld_out, stride_in, stride_out;
    uint32_t m, n, mp, np;       // rows <= columns, and both in multiples of 64
    uint32_t batch, norm_parts, step, steps;
    uint32_t strips;             // of X's columns: one plane keeps a row's sum of squares in so many parts
    int tall;                    // the matrix is the transpose
    float a, b, c, eps, scale;
    // bound of |X| after k steps, and of its growth from |X| = tau, for
    // singular values up to 1 (tau)
    float bound[AR_ORTHO_MAX_STEPS + 1], growth[AR_ORTHO_MAX_STEPS + 1];
    float abs_b[AR_ORTHO_MAX_STEPS], abs_c[AR_ORTHO_MAX_STEPS];
};

// ---- the norm ---------------------------------------------------------------

// Sums of squares in fp64: any fp32 matrix' norm is in range.  One wave a row.
template <typename T> __global__ __launch_bounds__(256) void ortho_norm_kernel(const OrthoArgs o)
{
    constexpr int VEC = 16 / (int)sizeof(T);
    __shared__ double sums[4];
    const uint32_t rows = o.tall ? o.n : o.m, cols = o.tall ? o.m : o.n;
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    const T *in = (const T *)o.in + blockIdx.y * o.stride_in;
    double sum = 0.0;
    for (uint32_t r = blockIdx.x * 4 + wave; r < rows; r += gridDim.x * 4) {
        const T *row = in + (uint64_t)r * o.ld_in;
        for (uint32_t c = lane * VEC; c < cols; c += 64 * VEC) {
            float v[VEC];
            if (c + VEC <= cols) load_vec<T, VEC>(row + c, v);
            else load_part<T, VEC>(row + c, (int)(cols - c), v);
#pragma unroll
            for (int k = 0; k < VEC; ++k) sum += (double)v[k] * (double)v[k];
        }
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
    if (lane == 0) sums[wave] = sum;
    __syncthreads();
    if (threadIdx.x == 0)
        ((double *)(o.ws + blockIdx.y * o.at.bytes + o.at.norms))[blockIdx.x] = sums[0] + sums[1] + sums[2] + sums[3];
}

// 2^(14 - e) for the least e with bound <= 2^e, the exponent kept within what
// an fp32 scale and its inverse hold.
__device__ __forceinline__ float scale_for(float bound)
{
    int e = bound > 0.0f ? ilogbf(bound) + 1 : -100;
    e = e < -100 ? -100 : e > 100 ? 100 : e;
    return ldexpf(1.0f, 14 - e);
}

// X's planes from the input: X = M / 2^e with the norm of M between 2^(e-1) and
// 2^e, which is exact; the rest of the normalisation is the first step's tau.
// Tiles of 64 x 64.
template <typename T, int PLANES> __global__ __launch_bounds__(256) void ortho_enter_kernel(const OrthoArgs o)
{
    __shared__ float tile[64][65];
    __shared__ double total[4];
    char *ws = o.ws + blockIdx.z * o.at.bytes;
    const double *parts = (const double *)(ws + o.at.norms);
    double sum = threadIdx.x < o.norm_parts ? parts[threadIdx.x] : 0.0;
#pragma unroll
    for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
    if ((threadIdx.x & 63u) == 0) total[threadIdx.x >> 6] = sum;
    __syncthreads();
    const double norm = sqrt(total[0] + total[1] + total[2] + total[3]);
    int e = 0;
    if (norm > 0.0) frexp(norm, &e);  // norm = f 2^e, f in [1/2, 1)
    const bool finite = norm <= 1.7976931348623157e308;
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x <= o.steps) {
        const int k = (int)threadIdx.x;
        const float tau = !finite ? __builtin_nanf("") : norm > 0.0 ? (float)(ldexp(1.0, e) / (norm + (double)o.eps)) : 1.0f;
        const float bound = fminf(o.bound[k], tau * o.growth[k]);
        const float sq = bound * bound;
        Scales s;
        s.x = k == 0 ? 16384.0f : scale_for(bound);
        s.a = scale_for(sq);
        s.b = k < (int)o.steps ? scale_for(o.abs_b[k] * sq + o.abs_c[k] * sq * sq) : 1.0f;
        s.tau = k == 0 ? tau : 1.0f;
        ((Scales *)(ws + o.at.scales))[k] = s;
    }
    // the tile of the input that becomes rows i0.., columns j0.. of X
    const uint32_t i0 = blockIdx.y * 64, j0 = blockIdx.x * 64;
    const uint32_t r0 = o.tall ? j0 : i0, c0 = o.tall ? i0 : j0, rows = o.tall ? o.n : o.m, cols = o.tall ? o.m : o.n;
    const T *in = (const T *)o.in + blockIdx.z * o.stride_in;
    for (uint32_t k = threadIdx.x; k < 512; k += 256) {
        const uint32_t r = k / 8, c = k % 8 * 8;
        float v[8];
        const T *from = in + (uint64_t)(r0 + r) * o.ld_in + c0 + c;
        if (r0 + r < rows && c0 + c + 8 <= cols) load_vec<T, 8>(from, v);
        else load_part<T, 8>(from, r0 + r < rows && c0 + c < cols ? (int)(cols - c0 - c) : 0, v);
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            // in two factors: 2^(14-e) alone may leave fp32's range
            const float x = finite ? ldexpf(ldexpf(v[q], -e / 2), 14 - e + e / 2) : __builtin_nanf("");
            if (o.tall) tile[c + q][r] = x;
            else tile[r][c + q] = x;
        }
    }
    __syncthreads();
    for (uint32_t k = threadIdx.x; k < 512; k += 256) {
        const uint32_t r = k / 8, c = k % 8 * 8;
        f16x8 h, l;
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const float x = tile[r][c + q];
            h[q] = (f16)x, l[q] = (f16)(x - (float)h[q]);
        }
        const size_t x_at = ((size_t)(i0 + r) * o.np + j0 + c) * 2;
        *(f16x8 *)(ws + o.at.x[0] + x_at) = h;
        *(f16x8 *)(ws + o.at.x[0] + o.at.x_lo + x_at) = l;
        if (PLANES == 2) store_vec<float, 8>((float *)(ws + o.at.xf + x_at * 2), &tile[r][c]);
    }
}

// ---- the products -----------------------------------------------------------

// Writes a wave's 32 x COLS block transposed: value(j, r) as in stage_rows,
// row(c): where column c goes (its element of the block's first row) or null;
// `rows` of the 32 are written.
template <typename O, int COLS, typename V, typename R>
__device__ __forceinline__ void store_32_cols(char *lds, uint32_t rows, V value, R row)
{
    constexpr int E = sizeof(O), PER = 16 / E, PITCH = 32 * E + 16, LANES = 32 / PER;
    const uint32_t lane = threadIdx.x & 63u;
#pragma unroll
    for (int j = 0; j < COLS / 32; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r)
            *(O *)(lds + (j * 32 + r / 4 * 8 + (lane >> 5) * 4 + r % 4) * PITCH + (lane & 31u) * E) = (O)value(j, r);
    asm volatile("" ::: "memory");
    const uint32_t c = lane % LANES * PER;
    static_assert(64 % LANES == 0 && COLS % (64 / LANES) == 0, "whole waves");
#pragma unroll
    for (int k0 = 0; k0 < COLS; k0 += 64 / LANES) {
        const uint32_t k = k0 + lane / LANES;
        O *to = row(k);
        const O *from = (const O *)(lds + k * PITCH) + c;
        if (to) {
            if (c + PER <= rows) {
                typedef O OV __attribute__((ext_vector_type(PER)));
                typedef O OU __attribute__((ext_vector_type(PER), aligned(E)));
                *(OU *)(to + c) = *(const OV *)from;
            } else {
                for (uint32_t q = c; q < rows; ++q) to[q] = from[q - c];
            }
        }
    }
    asm volatile("" ::: "memory");
}
template <typename O, int COLS> constexpr int kStageColBytes = COLS * (32 * (int)sizeof(O) + 16);

// A wave's place in its tile.
template <typename S> struct WaveAt {
    uint32_t row0, col0, row, half;
    __device__ __forceinline__ WaveAt(const TileAt at)
    {
        const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        row0 = at.m * S::BM + wave / S::WN * S::MT * 32, col0 = at.n * S::BN + wave % S::WN * S::NT * 32;
        row = lane & 31u, half = (lane >> 5) * 4;
    }
    __device__ __forceinline__ uint32_t i(int bi) const { return row0 + bi * 32 + row; }
    __device__ __forceinline__ uint32_t j(int bj, int r) const { return col0 + bj * 32 + r / 4 * 8 + half + r % 4; }
};

// Whether among four neighbouring elements of a row two have the same magnitude, to
// 18 bits, and it is not zero.
__device__ __forceinline__ bool two_alike(const float *v)
{
    uint32_t m[4];
    bool same = false;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t found = (__builtin_bit_cast(uint32_t, v[k]) + 32) >> 6 & 0x1ffffffu;
        m[k] = found > (uint32_t)k ? found : (uint32_t)k;  // zeros differ from each other
#pragma unroll
        for (int h = 0; h < k; ++h) same |= m[h] == m[k];
    }
    return same;
}

// 32 rows of a wave's block on their way into a product's only plane.  The plane's 11
// bits are the nearest, left to the caller's conversion, but where many neighbours
// are alike: there a value goes up or down at random, in proportion.  Equal values'
// rounding errors are equal: in a matrix of few magnitudes they add up over its rows
// and columns instead of averaging, and the steps amplify them (a constant 572 x
// 2158: off by 9.7e-3 of its norm, so by 4e-4).  Elsewhere the nearest value errs less.
// Each block of 32 x 32 is judged by its first eight columns, which costs next to
// nothing (a hash and comparisons for every four elements: 3 to 6 % of a call).  The
// random bits come from an element's place and `salt` alone.  w.j: column.
template <int NT, typename W> __device__ __forceinline__ void round_alike(float (&v)[NT][16], uint32_t i, const W &w, uint32_t salt)
{
#pragma unroll
    for (int bj = 0; bj < NT; ++bj) {
        if (__builtin_popcountll(__builtin_amdgcn_ballot_w64(two_alike(v[bj]))) < 8) continue;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            // odd numbers: leading bits of square roots of primes; eight bits for each of four elements
            uint32_t x = i * 0x6a09e667u + w.j(bj, q * 4) / 4 * 0xbb67ae85u + salt * 0x3c6ef373u;
            x ^= x >> 16, x *= 0x510e527fu, x ^= x >> 13, x *= 0x9b05688du, x ^= x >> 16;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                // a float's bits behind an fp16's ten; an infinity or NaN keeps what it is
                float &e = v[bj][q * 4 + k];
                e = __builtin_bit_cast(float, (__builtin_bit_cast(uint32_t, e) + ((x >> (8 * k) & 255u) << 5) + 16) & ~0x1fffu);
            }
        }
    }
}
enum { kSaltX, kSaltA, kSaltB, kSalts };  // and the step

// The planes of a scaled matrix from 32 rows of a wave's block, for rows and
// columns up to the padded sizes; MIRROR: also transposed, for a symmetric one.
// high(j, r): what the first plane holds.
template <typename S, int PLANES, bool MIRROR, typename H>
__device__ __forceinline__ void store_planes(char *stage, const float (&v)[S::NT][16], H high, uint32_t first, uint32_t col0, char *hi,
                                             size_t lo, uint32_t rows, uint32_t cols)
{
    constexpr int COLS = S::NT * 32;
    if (first >= rows || col0 >= cols) return;
#pragma unroll
    for (int plane = 0; plane < PLANES; ++plane) {
        f16 *to = (f16 *)(hi + plane * lo);
        stage_rows<f16, COLS>(stage, [&](int j, int r) { return plane == 0 ? high(j, r) : v[j][r] - high(j, r); });
        write_rows<f16, COLS>(stage, to + (uint64_t)first * cols + col0, cols, 0, rows - first, cols - col0);
        if (MIRROR) write_columns<f16, COLS>(stage, to + (uint64_t)col0 * cols + first, cols, rows - first, cols - col0);
    }
}

// What an epilogue adds to its sums, from N planes of a padded matrix: block
// row bi + 1 is loaded while bi is worked on.  Each plane has its own stage, the
// first one also the epilogue's own (free again after the last take).
template <typename S, typename X, int N> struct Ahead {
    static constexpr int COLS = S::NT * 32;
    const X *from;
    size_t lo;  // bytes between planes
    uint32_t rows, cols, row0, col0;
    char *lds;
    RowsAhead<X, COLS> next[N];
    __device__ __forceinline__ void load(int bi)
    {
        const uint32_t first = row0 + bi * 32;
        if (bi >= S::MT || first >= rows || col0 >= cols) return;
#pragma unroll
        for (int n = 0; n < N; ++n) next[n].load((const X *)((const char *)from + n * lo) + (uint64_t)first * cols + col0, cols, cols - col0);
    }
    __device__ __forceinline__ void stage(int bi)
    {
#pragma unroll
        for (int n = 0; n < N; ++n) next[n].stage(lds + n * kStageBytes<X, COLS>);
        load(bi + 1);
    }
    __device__ __forceinline__ void take(int bj, int q, float *out) const
    {
        RowsAhead<X, COLS>::take(lds, bj, q, out);
        if (N == 2) {
            float more[4];
            RowsAhead<X, COLS>::take(lds + kStageBytes<X, COLS>, bj, q, more);
#pragma unroll
            for (int k = 0; k < 4; ++k) out[k] += more[k];
        }
    }
};

template <typename S> constexpr int kOrthoStage = kStageColBytes<float, S::NT * 32> > 2 * kStageBytes<f16, S::NT * 32>
                                                      ? kStageColBytes<float, S::NT * 32> : 2 * kStageBytes<f16, S::NT * 32>;
template <typename S> constexpr int kOrthoLds = S::LDS > 4 * kOrthoStage<S> ? S::LDS : 4 * kOrthoStage<S>;

// The sums of squares of X's rows that the update left, one part for each strip of
// columns, for the block rows of a tile on the diagonal.  Both halves of a wave
// share out a row's parts.  The loads begin with the products (4096 x 4096 bf16:
// behind them 7 us a step more).
template <int N> struct RowSquares {
    static constexpr int EARLY = 16;
    float part[N][EARLY];
    const float *from;
    uint32_t strips, pitch;
    __device__ __forceinline__ void load(const OrthoArgs &o, const char *ws, uint32_t row0)
    {
        from = (const float *)(ws + o.at.squares), strips = o.strips, pitch = o.mp;
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int k = 0; k < EARLY; ++k) part[n][k] = at(row0 + n * 32, k);
    }
    // row l%32 of the block that begins at `first`
    __device__ __forceinline__ float at(uint32_t first, uint32_t k) const
    {
        const uint32_t i = first + (threadIdx.x & 31u), s = 2 * k + (threadIdx.x >> 5 & 1u);
        return i < pitch && s < strips ? from[(uint64_t)s * pitch + i] : 0.0f;
    }
    __device__ __forceinline__ float sum(int n, uint32_t first) const
    {
        float t = 0.0f;
#pragma unroll
        for (int k = 0; k < EARLY; ++k) t += part[n][k];
        for (uint32_t k = EARLY; 2 * k < strips; ++k) t += at(first, k);
        return t + __shfl_xor(t, 32);
    }
};

// 32 rows of A (SECOND false) or B from their sums: written to both places; the
// diagonal goes to its fp32 vector and is zero in the planes.
template <typename S, bool SECOND, typename A, int N>
__device__ __forceinline__ void square_rows(float (&v)[S::NT][16], int bi, const TileAt at, const WaveAt<S> &w, const OrthoArgs &o,
                                            const Scales &s, A &ahead, const RowSquares<N> &squares, char *stage)
{
    constexpr int NT = S::NT, PLANES = S::PLANES;
    char *ws = o.ws + at.batch * o.at.bytes;
    float *diag_a = (float *)(ws + o.at.diag_a), *diag_b = (float *)(ws + o.at.diag_b);
    const float sx = s.tau / s.x, ia = 1.0f / s.a, to = SECOND ? s.b : s.a;  // powers of two but for tau
    const uint32_t i = w.i(bi);
    const float di = SECOND && i < o.m ? diag_a[i] : 0.0f;
    if constexpr (SECOND) ahead.stage(bi);
#pragma unroll
    for (int bj = 0; bj < NT; ++bj)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint32_t j0 = w.j(bj, q * 4);
            float off[4] = {0.0f, 0.0f, 0.0f, 0.0f}, dj[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            if constexpr (SECOND) {
                if (j0 < o.mp) load_vec<float, 4>(diag_a + j0, dj);
                ahead.take(bj, q, off);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t j = j0 + k;
                float x = v[bj][q * 4 + k];
                if (!SECOND) {
                    x = x * sx * sx;
                } else {
                    const float t = off[k] * ia;
                    x = o.b * t + o.c * (x * ia * ia + (di + dj[k]) * t);
                }
                v[bj][q * 4 + k] = i < o.m && j < o.m ? x * to : 0.0f;
            }
        }
    const uint32_t first = w.row0 + bi * 32;
    if (at.m == at.n) {
        // One plane: A's diagonal is the rows' sums of squares, of which the products
        // hold those of X rounded to a plane (the input's plane is exact).
        const bool exact = !SECOND && PLANES == 1 && o.step > 0;
        const float square = exact ? squares.sum(N == 1 ? 0 : bi, first) * sx * sx : 0.0f;
        // the diagonal goes to its vector (off and dj are zero there)
#pragma unroll
        for (int bj = 0; bj < NT; ++bj)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                if (w.j(bj, r) != i) continue;
                const float found = exact ? square : v[bj][r] / to;
                if (i < o.m) (SECOND ? diag_b : diag_a)[i] = SECOND ? o.b * di + found + o.c * di * di : found;
                v[bj][r] = 0.0f;
            }
    }
    char *hi = ws + (SECOND ? o.at.b : o.at.a);
    const size_t lo = SECOND ? o.at.b_lo : o.at.a_lo;
    if (PLANES == 1) round_alike<NT>(v, i, w, o.step * kSalts + (SECOND ? kSaltB : kSaltA));
    auto high = [&](int j, int r) { return (float)(f16)v[j][r]; };
    if (at.m != at.n) store_planes<S, PLANES, true>(stage, v, high, first, w.col0, hi, lo, o.mp, o.mp);
    else store_planes<S, PLANES, false>(stage, v, high, first, w.col0, hi, lo, o.mp, o.mp);
}

// Where a wave's sums of one run of k go: blocks in turn, each four vectors of
// four elements a lane, as the accumulators hold them.
template <typename S> __device__ __forceinline__ float *run_sums(const OrthoArgs &o, const TileAt at, uint32_t tiles, uint32_t split)
{
    const uint64_t tile = (uint64_t)split * (tiles * (tiles + 1) / 2) + at.m * (at.m + 1) / 2 + at.n;
    return (float *)(o.ws + at.batch * o.at.bytes + o.at.part) + (tile * S::WAVES + (threadIdx.x >> 6)) * (S::MT * S::NT * 1024) +
           (threadIdx.x & 63u) * 4;
}

// A = X X^T (SECOND false) or B = b A + c A A (true): tiles on and below the
// diagonal.  A of short rows is split over its long k: the runs' sums go to
// the workspace, for ortho_join_kernel.
template <typename S, bool SECOND>
__global__ __launch_bounds__(S::THREADS) void ortho_square_kernel(const GemmArgs g, const OrthoArgs o)
{
    constexpr int NT = S::NT, PLANES = S::PLANES;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const TileAt at = tile_at_lower(g.tiles_m, g.batch, g.splits);
    const WaveAt<S> w(at);
    const char *ws = o.ws + at.batch * o.at.bytes;
    // what the epilogue begins with is on its way during the products
    const Scales s = ((const Scales *)(ws + o.at.scales))[o.step];
    char *stage = lds + (threadIdx.x >> 6) * kOrthoStage<S>;
    Ahead<S, f16, PLANES> ahead{(const f16 *)(ws + o.at.a), o.at.a_lo, o.mp, o.mp, w.row0, w.col0, stage};
    if (SECOND) ahead.load(0);
    RowSquares<S::MT> squares;
    if (!SECOND && PLANES == 1 && o.step > 0 && at.m == at.n && g.splits == 1) squares.load(o, ws, w.row0);
    f32x16 acc[S::MT][NT];
    gemm_tile<f16, S, false>(g, at, lds, acc);
    if (!SECOND && g.splits > 1) {
        float *to = run_sums<S>(o, at, g.tiles_m, at.split);
        static_for<S::MT>([&](auto block) {
            float v[NT][16];
            take(acc[block.value], v);
#pragma unroll
            for (int bj = 0; bj < NT; ++bj)
#pragma unroll
                for (int q = 0; q < 4; ++q) store_vec<float, 4>(to + ((block.value * NT + bj) * 4 + q) * 256, &v[bj][q * 4]);
        });
        return;
    }
    static_for<S::MT>([&](auto block) {
        float v[NT][16];
        take(acc[block.value], v);
        square_rows<S, SECOND>(v, block.value, at, w, o, s, ahead, squares, stage);
    });
}

// A from the runs' sums, added in their order; a workgroup has one block row of
// each wave's.
template <typename S> __global__ __launch_bounds__(S::THREADS) void ortho_join_kernel(const GemmArgs g, const OrthoArgs o)
{
    constexpr int NT = S::NT;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const TileAt at = tile_at_lower(g.tiles_m, g.batch, 1);
    const WaveAt<S> w(at);
    const Scales s = ((const Scales *)(o.ws + at.batch * o.at.bytes + o.at.scales))[o.step];
    const float *from = run_sums<S>(o, at, g.tiles_m, 0) + blockIdx.y * NT * 1024;
    const uint64_t run = run_sums<S>(o, at, g.tiles_m, 1) - run_sums<S>(o, at, g.tiles_m, 0);
    RowSquares<1> squares;
    if (S::PLANES == 1 && o.step > 0 && at.m == at.n) squares.load(o, o.ws + at.batch * o.at.bytes, w.row0 + blockIdx.y * 32);
    float v[NT][16];
#pragma unroll
    for (int bj = 0; bj < NT; ++bj)
#pragma unroll
        for (int r = 0; r < 16; ++r) v[bj][r] = 0.0f;
#pragma unroll 4
    for (uint32_t split = 0; split < g.splits; ++split) {
#pragma unroll
        for (int bj = 0; bj < NT; ++bj)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float x[4];
                load_vec<float, 4>(from + split * run + (bj * 4 + q) * 256, x);
#pragma unroll
                for (int k = 0; k < 4; ++k) v[bj][q * 4 + k] += x[k];
            }
    }
    int none = 0;
    square_rows<S, false>(v, (int)blockIdx.y, at, w, o, s, none, squares, lds + (threadIdx.x >> 6) * kOrthoStage<S>);
}

// X = a X + B X from the sums of B X (the off-diagonal B); after the last step the
// result in the output's type.  stage: this wave's.
// ahead: X's elements, begun before the products.
template <typename S> using X = typename std::conditional<S::PLANES == 2, float, f16>::type;
template <typename S> using XAhead = Ahead<S, X<S>, S::PLANES == 2 ? 1 : 2>;
template <typename S> __device__ __forceinline__ XAhead<S> x_ahead(const TileAt at, const OrthoArgs &o, char *stage)
{
    const WaveAt<S> w(at);
    const char *ws = o.ws + at.batch * o.at.bytes;
    return XAhead<S>{(const X<S> *)(ws + (S::PLANES == 2 ? o.at.xf : o.at.x[o.step & 1u])), o.at.x_lo, o.mp, o.np, w.row0, w.col0, stage};
}
template <typename S, typename O>
__device__ __forceinline__ void update(f32x16 (&acc)[S::MT][S::NT], const TileAt at, const OrthoArgs &o, const Scales s, const Scales next,
                                       XAhead<S> &ahead, const float *diag_b)
{
    constexpr int NT = S::NT, PLANES = S::PLANES;
    char *stage = ahead.lds;
    const WaveAt<S> w(at);
    char *ws = o.ws + at.batch * o.at.bytes;
    const bool last = o.step + 1 == o.steps;
    const float to = last ? o.scale : next.x, ib = 1.0f / s.b, ix = s.tau / s.x;
    // X's planes are read by other tiles too, so they alternate; its fp32 values are not.
    char *x_next = ws + o.at.x[(o.step + 1) & 1u];
    O *out = (O *)o.out + at.batch * o.stride_out;
    static_for<S::MT>([&](auto block) {
        constexpr int bi = block.value;
        float v[NT][16];
        take(acc[bi], v);
        const uint32_t i = w.i(bi);
        const float d = i < o.m ? o.a + diag_b[i] : 0.0f;
        ahead.stage(bi);
#pragma unroll
        for (int bj = 0; bj < NT; ++bj)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const uint32_t j0 = w.j(bj, q * 4);
                float x[4];
                ahead.take(bj, q, x);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float y = (d * x[k] + v[bj][q * 4 + k] * ib) * ix;
                    v[bj][q * 4 + k] = i < o.m && j0 + k < o.n ? y * to : 0.0f;
                }
            }
        const uint32_t first = w.row0 + bi * 32;
        auto value = [&](int j, int r) { return v[j][r]; };
        if (!last) {
            if (PLANES == 1 && w.col0 < o.np) {
                float square = 0.0f;
#pragma unroll
                for (int bj = 0; bj < NT; ++bj)
#pragma unroll
                    for (int r = 0; r < 16; ++r) square += v[bj][r] * v[bj][r];
                square += __shfl_xor(square, 32);
                if (w.half == 0 && i < o.mp) ((float *)(ws + o.at.squares))[(uint64_t)(w.col0 / (NT * 32)) * o.mp + i] = square;
            }
            float h[NT][16];
#pragma unroll
            for (int bj = 0; bj < NT; ++bj)
#pragma unroll
                for (int r = 0; r < 16; ++r) h[bj][r] = v[bj][r];
            if (PLANES == 1) round_alike<NT>(h, i, w, (o.step + 1) * kSalts + kSaltX);
            store_planes<S, 2, false>(stage, v, [&](int j, int r) { return (float)(f16)h[j][r]; }, first, w.col0, x_next, o.at.x_lo, o.mp, o.np);
            if (PLANES == 2 && first < o.m && w.col0 < o.np) {
                stage_rows<float, NT * 32>(stage, value);
                write_rows<float, NT * 32>(stage, (float *)(ws + o.at.xf) + (uint64_t)first * o.np + w.col0, o.np, 0, o.m - first, o.np - w.col0);
            }
        } else if (first < o.m && w.col0 < o.n) {
            if (o.tall) {
                store_32_cols<O, NT * 32>(stage, o.m - first, value, [&](uint32_t c) {
                    return w.col0 + c < o.n ? out + (uint64_t)(w.col0 + c) * o.ld_out + first : nullptr;
                });
            } else {
                stage_rows<O, NT * 32>(stage, value);
                write_rows<O, NT * 32>(stage, out + (uint64_t)first * o.ld_out + w.col0, o.ld_out, 0, o.m - first, o.n - w.col0);
            }
        }
    });
}

template <typename S, typename O>
__global__ __launch_bounds__(S::THREADS) void ortho_update_kernel(const GemmArgs g, const OrthoArgs o)
{
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const TileAt at = tile_at(g.tiles_m, g.tiles_n, g.batch);
    const Scales *scales = (const Scales *)(o.ws + at.batch * o.at.bytes + o.at.scales);
    const Scales s = scales[o.step], next = scales[o.step + 1];
    XAhead<S> ahead = x_ahead<S>(at, o, lds + (threadIdx.x >> 6) * kOrthoStage<S>);
    ahead.load(0);
    f32x16 acc[S::MT][S::NT];
    gemm_tile<f16, S, false, false, true>(g, at, lds, acc);
    update<S, O>(acc, at, o, s, next, ahead, (const float *)(o.ws + at.batch * o.at.bytes + o.at.diag_b));
}

// A whole step of a small matrix (at most 128 rows) in one kernel: every
// workgroup computes A and B for itself, keeps their planes in LDS, and updates
// 64 columns of X.  Launches are what small matrices spend their time on (128 x
// 384 fp32: a step as three kernels 20 us, as this one 17.5); the repeated
// products cost less.
typedef Shape<1, 2, 2, 64, 2, 4> SmallSquare;  // eight waves: they hide each other's waits
typedef Shape<1, 1, 2, 64, 2, 4> SmallUpdate;
constexpr uint32_t kSmallRows = 128, kSmallBlock = kSmallRows * 128, kSmallPlane = 2 * kSmallBlock;  // k = 64 of a plane; a plane
constexpr uint32_t kSmallX = 2 * kSmallPlane, kSmallStage = kSmallX + 2 * kSmallBlock;  // X's 64 columns; the epilogue
constexpr uint32_t kSmallDiag = kSmallStage + 8 * kOrthoStage<SmallUpdate> > SmallSquare::LDS ? kSmallStage + 8 * kOrthoStage<SmallUpdate> : SmallSquare::LDS;
constexpr uint32_t kSmallLds = kSmallDiag + 2 * kSmallRows * 4;
static_assert(kSmallStage + 8 * kOrthoStage<SmallUpdate> <= kSmallLds - 2 * kSmallRows * 4, "the stages fit");

template <typename O> __global__ __launch_bounds__(512) void ortho_step_kernel(const GemmArgs g, const OrthoArgs o)
{
    extern __shared__ __attribute__((aligned(16))) char lds[];
    float *diag_a = (float *)(lds + kSmallDiag), *diag_b = diag_a + kSmallRows;
    const uint32_t tiles = o.np / 64, lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const TileAt at{blockIdx.x / tiles, 0, blockIdx.x % tiles, 0};
    char *ws = o.ws + at.batch * o.at.bytes;
    const Scales s = ((const Scales *)(ws + o.at.scales))[o.step], following = ((const Scales *)(ws + o.at.scales))[o.step + 1];
    const WaveAt<SmallSquare> w(TileAt{at.batch, 0, 0, 0});
    XAhead<SmallUpdate> ahead = x_ahead<SmallUpdate>(at, o, lds + kSmallStage + wave * kOrthoStage<SmallUpdate>);
    ahead.load(0);
    // where the planes' element (row, column) lies: rows of 64 columns, chunks swizzled as the products read them
    auto place = [&](uint32_t row, uint32_t col) { return col / 64 * kSmallBlock + row * 128 + ((col % 64 / 8) ^ (row >> 1 & 7u)) * 16 + col % 8 * 2; };
    typedef f16 f16x4 __attribute__((ext_vector_type(4)));

    f32x16 acc[1][2];
    gemm_tile<f16, SmallSquare, false>(g, TileAt{at.batch, 0, 0, 0}, lds, acc);

    // X's columns on their way while A and B are made: 128 rows by k, both planes
    {
        const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds + kSmallX;
        Side<SmallUpdate, true, 64> side;  // 64 rows a buffer: two of them
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            side.place(wave, at.n * 64, o.np, [&](uint32_t row, uint32_t) { return row * o.np * 2; });
            if (half * 64u >= o.mp) side.stop_at(wave, 0);
#pragma unroll
            for (int plane = 0; plane < 2; ++plane) {
                const u32x4v from = tile_resource(uniform_address(ws + o.at.x[o.step & 1u] + plane * o.at.x_lo + (size_t)half * 64 * o.np * 2 + at.n * 128));
#pragma unroll
                for (int n = 0; n < side.LOADS; ++n)
                    load_to_lds(lds0 + plane * kSmallBlock + half * (kSmallBlock / 2) + (n * 8 + wave) * 1024, side.off[n], from, 0);
            }
        }
    }

    // The sums scaled by `to` become the planes; the diagonal goes to its vector.
    auto keep = [&](float (&v)[2][16], float *diag, float to, float of_diag) {
        const uint32_t i = w.i(0);
#pragma unroll
        for (int bj = 0; bj < 2; ++bj)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const uint32_t j0 = w.j(bj, q * 4);
                f16x4 h, l;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    float x = i < o.m && j0 + k < o.m ? v[bj][q * 4 + k] : 0.0f;
                    if (j0 + k == i) {
                        diag[i] = x + of_diag;
                        x = 0.0f;
                    }
                    x *= to;
                    h[k] = (f16)x, l[k] = (f16)(x - (float)h[k]);
                }
                *(f16x4 *)(lds + place(i, j0)) = h;
                *(f16x4 *)(lds + kSmallPlane + place(i, j0)) = l;
            }
    };
    const float sx = s.tau / s.x, ia = 1.0f / s.a;
    float v[2][16];
    take(acc[0], v);
#pragma unroll
    for (int bj = 0; bj < 2; ++bj)
#pragma unroll
        for (int r = 0; r < 16; ++r) v[bj][r] = v[bj][r] * sx * sx;
    keep(v, diag_a, s.a, 0.0f);
    __syncthreads();

    // Fragments of the planes: row l%32 from `row0` on, k = 16 * quarter + 8 * (l/32) + 0..7.
    const uint32_t fr = lane & 31u, fc = lane >> 5;
    auto rows = [&](int plane, uint32_t row0, int quarter) {
        return *(const f16x8 *)(lds + plane * kSmallPlane + quarter / 4 * kSmallBlock + (row0 + fr) * 128 +
                                ((2 * (quarter % 4) + fc) ^ (fr >> 1 & 7u)) * 16);
    };
    const uint32_t wm = wave / 2, wn = wave % 2;
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[0][j][r] = 0.0f;
    static_for<8>([&](auto quarter) {
        f16x8 a[2], b[2][2];
#pragma unroll
        for (int plane = 0; plane < 2; ++plane) {
            a[plane] = rows(plane, wm * 32, quarter.value);
#pragma unroll
            for (int j = 0; j < 2; ++j) b[plane][j] = rows(plane, wn * 64 + j * 32, quarter.value);
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            acc[0][j] = Frag<f16>::mfma(b[0][j], a[0], acc[0][j]);
            acc[0][j] = Frag<f16>::mfma(b[1][j], a[0], acc[0][j]);
            acc[0][j] = Frag<f16>::mfma(b[0][j], a[1], acc[0][j]);
        }
    });
    settle(acc);
    // b A + c A A, with A's elements from the planes, before those make room
    take(acc[0], v);
    const float di = diag_a[w.i(0)];
#pragma unroll
    for (int bj = 0; bj < 2; ++bj)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint32_t at_ij = place(w.i(0), w.j(bj, q * 4));
            const f16x4 h = *(const f16x4 *)(lds + at_ij), l = *(const f16x4 *)(lds + kSmallPlane + at_ij);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float t = ((float)h[k] + (float)l[k]) * ia;  // zero on the diagonal
                v[bj][q * 4 + k] = o.b * t + o.c * (v[bj][q * 4 + k] * ia * ia + (di + diag_a[w.j(bj, q * 4 + k)]) * t);
            }
        }
    __syncthreads();
    keep(v, diag_b, s.b, o.b * di + o.c * di * di);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // X's columns
    __syncthreads();

    // B X: 32 rows and 32 columns a wave
    f32x16 sums[1][1];
#pragma unroll
    for (int r = 0; r < 16; ++r) sums[0][0][r] = 0.0f;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
    typedef Side<SmallUpdate, true, 64> SideX;
    const uint32_t tk = 8 * fc + (lane & 15u) / 4, tc = 2 * (lane >> 4 & 1u) + (lane >> 1 & 1u);
    const uint32_t col = tk * 128 + (wn * 4 + tc + SideX::turn(tk)) % 8 * 16 + (lane & 1u) * 8;
    static_for<8>([&](auto quarter) {
        f16x8 a[2], b[2];
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) s16x4 *P;
#pragma unroll
        for (int plane = 0; plane < 2; ++plane) {
            a[plane] = rows(plane, wm * 32, quarter.value);
            const uint32_t from = lds0 + kSmallX + plane * kSmallBlock + quarter.value * 16 * 128 + col;
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(uintptr_t)from);
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(uintptr_t)(from + 4 * 128));
            b[plane] = __builtin_bit_cast(f16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        }
        sums[0][0] = Frag<f16>::mfma(b[0], a[0], sums[0][0]);
        sums[0][0] = Frag<f16>::mfma(b[1], a[0], sums[0][0]);
        sums[0][0] = Frag<f16>::mfma(b[0], a[1], sums[0][0]);
    });
    settle(sums);
    update<SmallUpdate, O>(sums, at, o, s, following, ahead, diag_b);
}

}  // namespace dev

namespace {

using namespace dev;

int check_ortho(const ar_ortho_desc *d)
{
    if (!d) return AR_ERR_ARG;
    if (!known_dtype(d->dtype)) return AR_ERR_UNSUPPORTED;
    if (d->rows < 1 || d->cols < 1 || d->rows > 65536 || d->cols > 65536 || d->batch > 65535) return AR_ERR_ARG;
    if (d->steps < 1 || d->steps > AR_ORTHO_MAX_STEPS) return AR_ERR_ARG;
    if (!isfinite(d->eps) || d->eps < 0.0f || !isfinite(d->scale)) return AR_ERR_ARG;
    for (size_t ld : {d->ld_in, d->ld_out})
        if (ld && (ld < d->cols || ld > kOpsMaxSize / d->rows)) return AR_ERR_ARG;
    for (size_t stride : {d->stride_in, d->stride_out})
        if (stride > kOpsMaxSize) return AR_ERR_ARG;
    return AR_OK;
}

// Bounds of |X| after each step for singular values in [0, 1], with 2 % for
// rounding; false for coefficients that leave what the planes can scale.
bool bounds(const ar_ortho_desc &d, OrthoArgs *o)
{
    double bound = 1.0, growth = 1.0;
    o->bound[0] = 1.0f, o->growth[0] = 1.0f;
    for (int k = 0; k < d.steps; ++k) {
        const double a = d.coefs[3 * k], b = d.coefs[3 * k + 1], c = d.coefs[3 * k + 2];
        if (!isfinite(a) || !isfinite(b) || !isfinite(c)) return false;
        // |p(v)| and |p(v) / v| have their largest values at an end of [0, bound] or at a zero of a derivative
        auto ratio = [&](double v2) { return fabs(a + b * v2 + c * v2 * v2); };
        auto value = [&](double v2) { return sqrt(v2) * ratio(v2); };
        const double top = bound * bound;
        double most = value(top), slope = ratio(0.0) > ratio(top) ? ratio(0.0) : ratio(top);
        auto consider = [&](double v2) {
            if (!(v2 > 0.0 && v2 < top)) return;
            most = value(v2) > most ? value(v2) : most;
            slope = ratio(v2) > slope ? ratio(v2) : slope;
        };
        if (c != 0.0) {
            const double disc = 9.0 * b * b - 20.0 * a * c;  // of a + 3 b w + 5 c w w, w = v v
            if (disc >= 0.0) {
                consider((-3.0 * b + sqrt(disc)) / (10.0 * c));
                consider((-3.0 * b - sqrt(disc)) / (10.0 * c));
            }
            consider(-b / (2.0 * c));
        } else if (b != 0.0) {
            consider(-a / (3.0 * b));
        }
        bound = 1.02 * most, growth *= 1.02 * slope;
        if (!(bound <= 4096.0)) return false;
        if (growth > 1e30) growth = 1e30;
        o->bound[k + 1] = (float)bound, o->growth[k + 1] = (float)growth;
        o->abs_b[k] = (float)fabs(b), o->abs_c[k] = (float)fabs(c);
    }
    return true;
}

// Whether the products take two planes: fp32, and bf16 with a short side of at
// most 256, where three products cost little beside the launches (see above).
bool two_planes(const ar_ortho_desc &d)
{
    return d.dtype == AR_FLOAT32 || (d.rows < d.cols ? d.rows : d.cols) <= 256;
}

OrthoSpace ortho_space(const ar_ortho_desc &d, uint32_t mp, uint32_t np)
{
    OrthoSpace s{};
    const bool two = two_planes(d);
    const size_t m = d.rows < d.cols ? d.rows : d.cols;
    const Cut c = a_cut(two ? 2 : 1, m, np, d.batch);
    const size_t side = kTiles[0][c.tile].side, tiles = (m + side - 1) / side;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += round_up(bytes, 256);
        return here;
    };
    const size_t x = (size_t)mp * np * 2, sq = (size_t)mp * mp * 2;
    s.x[0] = take(2 * x), s.x[1] = take(2 * x), s.xf = take(two ? 2 * x : 0);
    s.a = take(two ? 2 * sq : sq), s.b = take(two ? 2 * sq : sq);
    s.x_lo = x, s.a_lo = s.b_lo = sq;
    s.diag_a = take(mp * 4), s.diag_b = take(mp * 4);
    s.squares = take(two ? 0 : (size_t)np / 32 * mp * 4);  // strips of 32 columns at least
    s.part = take(c.splits > 1 ? c.splits * (tiles * (tiles + 1) / 2) * side * side * 4 : 0);
    s.scales = take(sizeof(Scales) * (AR_ORTHO_MAX_STEPS + 1));
    s.norms = take(sizeof(double) * kNormParts);
    s.bytes = at;
    return s;
}

// The shapes of kTiles' tiles.
template <int PLANES, int TILE> struct ShapeOf;
template <> struct ShapeOf<1, 0> { typedef Shape<1, 1, 1, 64, 4> type; };
template <> struct ShapeOf<1, 1> { typedef Shape<2, 2, 1, 64, 2> type; };
template <> struct ShapeOf<1, 2> { typedef Shape<3, 3, 1, 64, 2> type; };
template <> struct ShapeOf<1, 3> { typedef Shape<4, 4, 1, 64, 2> type; };
template <> struct ShapeOf<2, 0> { typedef Shape<1, 1, 2, 64, 3> type; };
template <> struct ShapeOf<2, 1> { typedef Shape<2, 2, 2, 64, 2> type; };
template <> struct ShapeOf<2, 2> { typedef Shape<3, 3, 2, 32, 2> type; };
template <> struct ShapeOf<2, 3> { typedef Shape<4, 4, 2, 32, 2> type; };

template <typename S, bool SECOND> int launch_square(GemmArgs &g, const OrthoArgs &o, hipStream_t st)
{
    g.tiles_m = g.tiles_n = (o.m + S::BM - 1) / S::BM;
    static OncePerDevice once;
    int rc = allow_lds(once, (const void *)ortho_square_kernel<S, SECOND>, kOrthoLds<S>);
    if (rc != AR_OK) return rc;
    const uint32_t tiles = g.tiles_m * (g.tiles_m + 1) / 2 * o.batch;
    hipLaunchKernelGGL((ortho_square_kernel<S, SECOND>), dim3(tiles * g.splits), dim3(S::THREADS), kOrthoLds<S>, st, g, o);
    rc = launch_status();
    if (rc != AR_OK || SECOND || g.splits == 1) return rc;
    constexpr int LDS = S::WAVES * kOrthoStage<S>;
    static OncePerDevice also;
    if ((rc = allow_lds(also, (const void *)ortho_join_kernel<S>, LDS)) != AR_OK) return rc;
    hipLaunchKernelGGL((ortho_join_kernel<S>), dim3(tiles, S::MT), dim3(S::THREADS), LDS, st, g, o);
    return launch_status();
}
template <int PLANES, bool SECOND> int square(GemmArgs &g, const OrthoArgs &o, hipStream_t st)
{
    const Cut c = SECOND ? b_cut(PLANES, o.m, o.mp, o.batch) : a_cut(PLANES, o.m, o.np, o.batch);
    g.splits = c.splits;
    switch (c.tile) {
    case 0: return launch_square<typename ShapeOf<PLANES, 0>::type, SECOND>(g, o, st);
    case 1: return launch_square<typename ShapeOf<PLANES, 1>::type, SECOND>(g, o, st);
    case 2: return launch_square<typename ShapeOf<PLANES, 2>::type, SECOND>(g, o, st);
    default: return launch_square<typename ShapeOf<PLANES, 3>::type, SECOND>(g, o, st);
    }
}

template <typename S, typename O> int launch_update(GemmArgs &g, OrthoArgs &o, hipStream_t st)
{
    o.strips = (o.np + S::NT * 32 - 1) / (S::NT * 32);
    g.tiles_m = (o.m + S::BM - 1) / S::BM, g.tiles_n = (o.n + S::BN - 1) / S::BN;
    static OncePerDevice once;
    const int rc = allow_lds(once, (const void *)ortho_update_kernel<S, O>, kOrthoLds<S>);
    if (rc != AR_OK) return rc;
    hipLaunchKernelGGL((ortho_update_kernel<S, O>), dim3(g.tiles_m * g.tiles_n * o.batch), dim3(S::THREADS), kOrthoLds<S>, st, g, o);
    return launch_status();
}
template <int PLANES, typename O> int update_step(GemmArgs &g, OrthoArgs &o, hipStream_t st)
{
    switch (x_cut(PLANES, o.m, o.n, o.mp, o.batch).tile) {
    case 0: return launch_update<typename ShapeOf<PLANES, 0>::type, O>(g, o, st);
    case 1: return launch_update<typename ShapeOf<PLANES, 1>::type, O>(g, o, st);
    case 2: return launch_update<typename ShapeOf<PLANES, 2>::type, O>(g, o, st);
    default: return launch_update<typename ShapeOf<PLANES, 3>::type, O>(g, o, st);
    }
}

// A product in the workspace; the second planes lie a_lo and b_lo behind the first.
void operands(GemmArgs *g, const OrthoArgs &o, size_t a, size_t a_lo, uint32_t lda, size_t b, size_t b_lo, uint32_t ldb, uint32_t k,
              uint32_t m, uint32_t n)
{
    *g = GemmArgs{};
    g->segments = 1, g->steps = k / kStepK, g->ka = g->kb = k;
    g->a[0] = o.ws + a, g->b[0] = o.ws + b, g->a_lo = a_lo, g->b_lo = b_lo;
    g->lda = lda * 2, g->ldb = ldb * 2;
    g->m = m, g->n = n, g->batch_a = g->batch_b = o.at.bytes, g->batch = o.batch, g->splits = 1;
}

template <typename O, int PLANES> int run_ortho(OrthoArgs &o, const float *coefs, hipStream_t st)
{
    hipLaunchKernelGGL((ortho_norm_kernel<O>), dim3(o.norm_parts, o.batch), dim3(256), 0, st, o);
    int rc = launch_status();
    if (rc != AR_OK) return rc;
    hipLaunchKernelGGL((ortho_enter_kernel<O, PLANES>), dim3(o.np / 64, o.mp / 64, o.batch), dim3(256), 0, st, o);
    if ((rc = launch_status()) != AR_OK) return rc;
    // One kernel a step for short rows of few columns: beyond about 1024 the
    // repeated A costs more than the launches.
    const bool small = PLANES == 2 && o.mp <= kSmallRows && o.np <= 1024;
    for (o.step = 0; o.step < o.steps; ++o.step) {
        o.a = coefs[3 * o.step], o.b = coefs[3 * o.step + 1], o.c = coefs[3 * o.step + 2];
        GemmArgs g;
        const size_t x = o.at.x[o.step & 1u];
        operands(&g, o, x, o.at.x_lo, o.np, x, o.at.x_lo, o.np, o.np, o.m, o.m);
        if constexpr (PLANES == 2) {
            if (small) {
                static OncePerDevice once;
                if ((rc = allow_lds(once, (const void *)ortho_step_kernel<O>, kSmallLds)) != AR_OK) return rc;
                hipLaunchKernelGGL((ortho_step_kernel<O>), dim3(o.np / 64 * o.batch), dim3(512), kSmallLds, st, g, o);
                if ((rc = launch_status()) != AR_OK) return rc;
                continue;
            }
        }
        if ((rc = square<PLANES, false>(g, o, st)) != AR_OK) return rc;
        operands(&g, o, o.at.a, o.at.a_lo, o.mp, o.at.a, o.at.a_lo, o.mp, o.mp, o.m, o.m);
        if ((rc = square<PLANES, true>(g, o, st)) != AR_OK) return rc;
        operands(&g, o, o.at.b, o.at.b_lo, o.mp, x, o.at.x_lo, o.np, o.mp, o.m, o.np);
        if ((rc = update_step<PLANES, O>(g, o, st)) != AR_OK) return rc;
    }
    return AR_OK;
}

int ortho(const ar_ortho_desc *desc, const void *in, void *out, void *ws, size_t ws_bytes, void *stream)
{
    int rc = check_ortho(desc);
    if (rc != AR_OK) return rc;
    const ar_ortho_desc &d = *desc;
    OrthoArgs o{};
    if (!d.coefs || !bounds(d, &o)) return AR_ERR_ARG;
    if (d.batch == 0) return AR_OK;
    const size_t e = elem_bytes(d.dtype), ld_in = d.ld_in ? d.ld_in : d.cols, ld_out = d.ld_out ? d.ld_out : d.cols;
    const size_t si = d.stride_in ? d.stride_in : d.rows * ld_in, so = d.stride_out ? d.stride_out : d.rows * ld_out;
    // matrices of a batch must not share elements: one after another, or side by side in shared rows
    auto apart = [&](size_t stride, size_t ld) {
        return d.batch == 1 || stride >= (d.rows - 1) * ld + d.cols || (stride >= d.cols && stride * (d.batch - 1) + d.cols <= ld);
    };
    if (!apart(si, ld_in) || !apart(so, ld_out)) return AR_ERR_ARG;
    if (!in || !out || (uintptr_t)in % e || (uintptr_t)out % e) return AR_ERR_ARG;
    const Batch bi{mat(in, d.rows, d.cols, ld_in, d.dtype), d.batch, si}, bo{mat(out, d.rows, d.cols, ld_out, d.dtype), d.batch, so};
    if (!(bi.first.same(bo.first) && (d.batch == 1 || si == so)) && meet(bi, bo)) return AR_ERR_ARG;
    const size_t need = ar_orthogonalize_workspace(desc);
    if (!ws || ws_bytes < need) return AR_ERR_SCRATCH;
    if ((uintptr_t)ws % 256 != 0) return AR_ERR_ARG;
    const Batch bw{Mat{ws, 1, need, need, 1}, 1, need};
    if (meet(bw, bi) || meet(bw, bo)) return AR_ERR_ARG;

    o.tall = d.rows > d.cols;
    o.m = (uint32_t)(o.tall ? d.cols : d.rows), o.n = (uint32_t)(o.tall ? d.rows : d.cols);
    o.mp = (uint32_t)round_up(o.m, kStepK), o.np = (uint32_t)round_up(o.n, kStepK);
    o.in = in, o.out = out, o.ws = (char *)ws, o.at = ortho_space(d, o.mp, o.np);
    o.ld_in = ld_in, o.ld_out = ld_out, o.stride_in = si, o.stride_out = so;
    o.batch = (uint32_t)d.batch, o.steps = (uint32_t)d.steps, o.eps = d.eps, o.scale = d.scale;
    const size_t parts = (d.rows + 3) / 4;
    o.norm_parts = (uint32_t)(parts < kNormParts ? parts : kNormParts);
    hipStream_t st = (hipStream_t)stream;
    if (d.dtype == AR_FLOAT32) return run_ortho<float, 2>(o, d.coefs, st);
    return two_planes(d) ? run_ortho<bf16, 2>(o, d.coefs, st) : run_ortho<bf16, 1>(o, d.coefs, st);
}

}  // namespace
}  // namespace ar

extern "C" int ar_orthogonalize(const ar_ortho_desc *desc, const void *in, void *out, void *workspace, size_t workspace_bytes,
                                void *stream)
{
    return ar::ops_ret(ar::ortho(desc, in, out, workspace, workspace_bytes, stream));
}

extern "C" size_t ar_orthogonalize_workspace(const ar_ortho_desc *desc)
{
    if (ar::check_ortho(desc) != AR_OK) return 0;
    const size_t m = desc->rows < desc->cols ? desc->rows : desc->cols, n = desc->rows < desc->cols ? desc->cols : desc->rows;
    return desc->batch * ar::ortho_space(*desc, (uint32_t)ar::round_up(m, ar::dev::kStepK), (uint32_t)ar::round_up(n, ar::dev::kStepK)).bytes;
}
