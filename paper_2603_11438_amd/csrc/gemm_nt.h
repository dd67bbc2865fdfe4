// Matrix products C[m][n] = sum_k A[m][k] B[k][n] on gfx950's matrix units, for
// kernels that bring their own epilogue.
//
// Operands are 16-bit and row-major, rows 16-byte aligned.  Each lies either by
// rows, A[m][k] or B[n][k] with k contiguous, or by k, A[k][m] or B[k][n]; then
// fragments are transposed on their way out of LDS, four k at a time.  What lies
// behind the last k of an operand is not read: those lanes' loads are out of
// their resource's range and bring zeros.  A product may run over several (A, B)
// pairs ("segments") of one k length one after another, all into
// the same sums ([dG dU] times [Wg; Wu]).  Operands in two planes, hi and lo,
// are multiplied as hi hi + hi lo + lo hi.
//
// A workgroup, mostly of four waves, one per SIMD, owns a tile; each wave holds MT x NT
// accumulators of 32 x 32 in registers.  k advances in stages of BK through
// BUFS LDS buffers.  Loads go from memory straight into LDS (16 bytes a lane).
// Once every wave has read the last fragments of a buffer its next loads
// begin, spread over the products of a stage: issued at once they would fill
// the way to the L2 (64 bytes a cycle for a compute unit) and hold up the
// products behind them.  Fragments for the next quarter of a stage (k = 16) are
// read while the matrix units work on this one, across stages too.
//
// A row's 16-byte chunks are stored in the order chunk ^ (row >> 1 & 7) (rows of
// 64 bytes: row >> 2 & 3), by permuting which chunk a lane loads: the sixteen
// rows' equal chunks that a read touches together then lie in sixteen different
// groups of four banks (SQ_LDS_BANK_CONFLICT: 0 where no epilogue is staged, else
// up to 2 % of the cycles; with row & 7 a read took twice as long).  By k, row k's
// chunks are rotated by 4 (k & 3) (64 columns: by 4 (k >> 1 & 1)): a transposing
// read takes 64 bytes of each of four rows.
//
// Rate, bf16, 8192 x 8192 x 8192: 856 us, 1284 TFLOP/s with the 256 x 256 tile and two
// buffers, at 1.75 GHz: the board's power limit has the clock.  With every load an L2
// hit the same kernel takes 794 us, so the rest is misses that a stage's lead does
// not cover.  A third buffer for A (AHEAD) makes the waits 15 % of the cycles, from 25,
// and the clock lower: 2 to 3 % less time (4096 x 4096 x 131072: 3540 us, from 3630), but
// paired and with all data in the cache 1 to 3 % more (`pair_ahead`).
// Smaller tiles: 128 x 128 1020 us, 64 x 64 1525 us.
#pragma once

#include <type_traits>
#include <utility>

#include "gemm_cut.h"
#include "ops_common.h"

namespace ar {
namespace dev {

typedef _Float16 f16;
typedef f16 f16x8 __attribute__((ext_vector_type(8)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4v __attribute__((ext_vector_type(4)));

template <typename T> struct Frag;
template <> struct Frag<f16> {
    typedef f16x8 type;
    static __device__ __forceinline__ f32x16 mfma(type a, type b, f32x16 c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
    }
};
template <> struct Frag<bf16> {
    typedef bf16x8 type;
    static __device__ __forceinline__ f32x16 mfma(type a, type b, f32x16 c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
    }
};

constexpr int kMaxSegments = 2;
// Rows of one tile are reached by 32-bit offsets from the tile's first row.
inline bool gemm_reaches(uint64_t row_bytes, uint64_t k_bytes) { return row_bytes * 256 + k_bytes < (1ull << 31); }

struct GemmArgs {
    const void *a[kMaxSegments], *b[kMaxSegments];
    const void *b2;             // paired operands: the second of each pair of columns (one segment)
    uint64_t a_lo, b_lo;        // two planes: bytes from the hi plane to the lo plane (one segment)
    uint32_t segments, steps;   // steps of 64 per segment, the last one not always whole
    uint32_t ka, kb;            // each operand's k of a segment (by rows: a multiple of 8)
    uint32_t lda, ldb, ldb2;    // bytes
    uint32_t m, n;              // of the result (paired: of each; by k: multiples of 8 that can be read)
    uint32_t tiles_m, tiles_n;
    uint64_t batch_a, batch_b;  // bytes between the matrices of a batch
    uint32_t batch;
    uint32_t splits;            // runs of stages that k is split into; 1: not split
};

// A load from this offset on is out of range: it touches no memory and brings zeros.
constexpr uint32_t kOutOfRange = 0x80000000u;

// a: wave-uniform
__device__ __forceinline__ u32x4v tile_resource(uint64_t a)
{
    u32x4v r;
    r.x = (uint32_t)a;
    r.y = (uint32_t)(a >> 32) & 0xffffu;
    r.z = kOutOfRange;  // offsets stay below 2^31 (gemm_reaches); rows are clamped to the matrix
    r.w = 0x00020000u;
    return r;
}

// 64 lanes' 16 bytes each into 1 KiB of LDS from `lds` on, in lane order.  The
// load has no output register: it is complete when vmcnt says so.  m0, which names
// the place in LDS, cannot be declared as written: the compiler takes it for its own
// and ignores it in a clobber list.  So nothing else may use it, and nothing does: a
// test holds that against the built code.  (Given back by each load, it would cost 1 %
// of the products' time.)
__device__ __forceinline__ void load_to_lds(uint32_t lds, uint32_t offset, u32x4v resource, uint32_t soffset)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                 :
                 : "s"(lds), "v"(offset), "s"(resource), "s"(soffset)
                 : "memory");
}

// Which tile a workgroup takes.  Consecutive workgroups go to the eight XCDs in
// turn; each XCD gets a run of neighbouring tiles, ordered in groups of
// kGroupRows tile rows, so that the operand rows its workgroups share stay in
// its L2.
constexpr uint32_t kGroupRows = 8;
struct TileAt {
    uint32_t batch, m, n;
    uint32_t split;  // which run of k
};
__device__ __forceinline__ uint32_t xcd_run(uint32_t id, uint32_t total)
{
    const uint32_t q = total / 8, r = total % 8, x = id % 8;
    return x * q + (x < r ? x : r) + id / 8;
}
__device__ __forceinline__ TileAt tile_at(uint32_t tiles_m, uint32_t tiles_n, uint32_t batch)
{
    const uint32_t per = tiles_m * tiles_n;
    uint32_t t = xcd_run(blockIdx.x, per * batch);
    TileAt at;
    at.split = blockIdx.y;
    at.batch = t / per;
    t %= per;
    const uint32_t group = t / (kGroupRows * tiles_n), first = group * kGroupRows;
    const uint32_t rows = tiles_m - first < kGroupRows ? tiles_m - first : kGroupRows;
    t -= first * tiles_n;
    at.m = first + t % rows;
    at.n = t / rows;
    return at;
}
// Tiles on and below the diagonal, by rows; with k split, the runs one after
// another, so that an XCD reads few of them.
__device__ __forceinline__ TileAt tile_at_lower(uint32_t tiles, uint32_t batch, uint32_t splits)
{
    const uint32_t per = tiles * (tiles + 1) / 2;
    uint32_t t = xcd_run(blockIdx.x, per * batch * splits);
    TileAt at;
    at.split = t / (per * batch);
    t %= per * batch;
    at.batch = t / per;
    t %= per;
    uint32_t m = (uint32_t)((sqrtf(8.0f * (float)t + 1.0f) - 1.0f) * 0.5f);
    while (m * (m + 1) / 2 > t) --m;
    while ((m + 1) * (m + 2) / 2 <= t) ++m;
    at.m = m;
    at.n = t - m * (m + 1) / 2;
    return at;
}

// f(0), f(1), .. f(N - 1) with the index as a constant.
template <int N, typename F, int... I> __device__ __forceinline__ void static_for_(F &&f, std::integer_sequence<int, I...>)
{
    (f(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F> __device__ __forceinline__ void static_for(F &&f)
{
    static_for_<N>(f, std::make_integer_sequence<int, N>{});
}
// How many of `most` things that come at `things` in `steps` steps are due before step k.
constexpr int upto(int k, int steps, int things, int most)
{
    const int n = (k * things + steps - 1) / steps;
    return n < most ? n : most;
}

// The shape of a workgroup's tile and pipeline: WM x 2 waves of MT x NT blocks of
// 32 x 32, PLANES planes of each operand, k in stages of BK through BUFS buffers, or
// with AHEAD through one more for A.
template <int MT_, int NT_, int PLANES_, int BK_, int BUFS_, int WM_ = 2, bool AHEAD_ = false> struct Shape {
    static constexpr int MT = MT_, NT = NT_, PLANES = PLANES_, BK = BK_, BUFS = BUFS_;
    static constexpr bool AHEAD = AHEAD_;
    static constexpr int WM = WM_, WN = 2, WAVES = WM * WN, THREADS = 64 * WAVES, BM = WM * MT * 32, BN = WN * NT * 32;
    static constexpr int ROW = BK * 2;                        // bytes of a row in a buffer
    static constexpr int PLANE = (BM + BN) * ROW;             // A's rows, then B's
    static constexpr int BUF = PLANES * PLANE, LDS = BUFS * BUF + (AHEAD ? BM * ROW : 0);
    static_assert(!AHEAD || (PLANES == 1 && BUFS == 2 && LDS <= 160 * 1024), "one plane, and room for it");
    static_assert(BM * ROW % (1024 * WAVES) == 0 && BN * ROW % (1024 * WAVES) == 0, "whole loads");
};

// Makes the accumulators safe to read by take().  Nothing in the hardware holds
// up a read of a register that a matrix instruction is still writing, and the
// compiler, which otherwise counts the cycles in between, does not look into
// take()'s instructions: the wait has to stand here (19 cycles at most), behind
// every product, which the operands see to.
template <int MT, int NT> __device__ __forceinline__ void settle(f32x16 (&acc)[MT][NT])
{
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) asm volatile("" : "+a"(acc[i][j]));
    asm volatile("s_nop 15\n\ts_nop 7" : "+a"(acc[MT - 1][NT - 1]));
}

// A block row of the accumulators in ordinary registers.  The reads stay where
// they are written: moved up as one, all accumulators together would not fit.
template <int NT> __device__ __forceinline__ void take(const f32x16 (&acc)[NT], float (&v)[NT][16])
{
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(v[j][r]) : "a"(acc[j][r]));
}

// One operand of a tile: which of its bytes each lane loads, and where its
// fragments lie in LDS.  R: rows (by rows) or columns (by k) of the tile; X:
// those of a wave, in blocks of 32.
template <typename S, bool BYK, int R> struct Side {
    static constexpr int CHUNKS = BYK ? R / 8 : S::ROW / 16;  // of 16 bytes in a row of the buffer
    static constexpr int LOADS = R * S::ROW / 1024 / S::WAVES;
    uint32_t off[LOADS];  // a lane's loads: bytes from the tile's first element
    uint64_t base;        // the tile's first element; by k, of this stage

    static __device__ __forceinline__ uint32_t turn(uint32_t k) { return CHUNKS == 8 ? (k >> 1 & 1u) * 4 : (k & 3u) * 4; }
    static __device__ __forceinline__ uint32_t swizzle(uint32_t row) { return CHUNKS == 8 ? row >> 1 & 7u : row >> 2 & 3u; }

    // first: the tile's first row or column, of `count`
    template <typename RowOf> __device__ __forceinline__ void place(uint32_t wave, uint32_t first, uint32_t count, RowOf row_of)
    {
        const uint32_t lane = threadIdx.x & 63u;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const uint32_t q = (i * S::WAVES + wave) * 64 + lane, row = q / CHUNKS, at = q % CHUNKS;
            if (BYK) {
                // columns past the end repeat the last eight
                uint32_t c = (at + CHUNKS - turn(row) % CHUNKS) % CHUNKS;
                c = first / 8 + c < count / 8 ? c : count / 8 - 1 - first / 8;
                off[i] = row_of(row, 0u) + c * 16;
            } else {
                off[i] = row_of(row, first) + (at ^ swizzle(row)) * 16;
            }
        }
    }

    // Puts the lanes that would load from k = `left` of the stage on out of range.
    __device__ __forceinline__ void stop_at(uint32_t wave, int left)
    {
        const uint32_t lane = threadIdx.x & 63u;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const uint32_t q = (i * S::WAVES + wave) * 64 + lane, row = q / CHUNKS, k = BYK ? row : ((q % CHUNKS) ^ swizzle(row)) * 8;
            if ((int)k >= left) off[i] = kOutOfRange;
        }
    }
};

__device__ __forceinline__ uint64_t uniform_address(const void *p)
{
    const uint64_t a = (uint64_t)p;
    // the builtin returns int: without the casts the low half's sign would fill the high half
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)a);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(a >> 32));
    return (uint64_t)hi << 32 | lo;
}

// The products of one tile.  acc[i][j][r], lane l: row i*32 + l%32 of the wave's
// rows, column j*32 + 8*(r/4) + 4*(l/32) + r%4 of its columns (B's fragment is
// the instruction's first operand, so a lane holds four neighbouring columns).
//
// ABYK, BBYK: the operand lies by k.  PAIRED (B by rows): of a wave's NT*32 rows
// of B the first half comes from b, the second half from b2, both at the same
// rows: the wave then holds both products of the same columns.
//
// With k split, a workgroup adds up run at.split of g.splits of the stages
// (never empty: there are at least as many steps as splits).
template <typename T, typename S, bool PAIRED, bool ABYK, bool BBYK>
__device__ __forceinline__ void gemm_tile_even(const GemmArgs &g, const TileAt at, char *lds, f32x16 (&acc)[S::MT][S::NT])
{
    constexpr int MT = S::MT, NT = S::NT, PLANES = S::PLANES, KQ = S::BK / 16, BUFS = S::BUFS;
    typedef Side<S, ABYK, S::BM> SideA;
    typedef Side<S, BBYK, S::BN> SideB;
    constexpr int LOADS_A = SideA::LOADS, LOADS_B = SideB::LOADS, LOADS_PLANE = LOADS_A + LOADS_B, LOADS = PLANES * LOADS_PLANE;
    static_assert((PLANES == 1 || !PAIRED) && (!PAIRED || !BBYK), "pairs have one plane and lie by rows");
    constexpr uint32_t A_BYTES = S::BM * S::ROW;
    typedef typename Frag<T>::type F;
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t wm = wave / S::WN, wn = wave % S::WN;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
    const uint32_t m0 = at.m * S::BM, n0 = at.n * (PAIRED ? S::BN / 2 : S::BN);
    constexpr int HALF = NT * 16;  // paired: columns of a wave

    SideA sa;
    SideB sb;
    auto place = [&]() {
        sa.place(wave, m0, g.m, [&](uint32_t row, uint32_t first) {
            return ABYK ? row * g.lda : ((first + row < g.m ? first + row : g.m - 1) - first) * g.lda;
        });
        sb.place(wave, n0, g.n, [&](uint32_t row, uint32_t first) {
            if (BBYK) return row * g.ldb;
            uint32_t ld = g.ldb, r = row;
            if (PAIRED) {
                const uint32_t in = row % (2 * HALF);
                ld = in < HALF ? g.ldb : g.ldb2;
                r = row / (2 * HALF) * HALF + in % HALF;
            }
            return ((first + r < g.n ? first + r : g.n - 1) - first) * ld;
        });
    };
    place();
    const uint32_t per = g.steps * (kStepK / S::BK), all = g.segments * per;
    const uint32_t begin = (uint32_t)((uint64_t)all * at.split / g.splits);
    const uint32_t total = (uint32_t)((uint64_t)all * (at.split + 1) / g.splits) - begin;
    uint32_t segment = begin / per, step = begin % per, loaded = 0;  // of the next load
    // by rows a stage is reached by `kbyte` behind the base, by k the base moves on
    u32x4v ra, rb, rb2, ra_lo, rb_lo;
    auto point = [&]() {
        ra = tile_resource(sa.base), rb = tile_resource(sb.base);
        if (PLANES == 2) ra_lo = tile_resource(sa.base + g.a_lo), rb_lo = tile_resource(sb.base + g.b_lo);
    };
    auto enter = [&]() {
        sa.base = uniform_address((const char *)g.a[segment] + at.batch * g.batch_a +
                                  (ABYK ? (uint64_t)step * S::BK * g.lda + m0 * 2 : (uint64_t)m0 * g.lda));
        sb.base = uniform_address((const char *)g.b[segment] + at.batch * g.batch_b +
                                  (BBYK ? (uint64_t)step * S::BK * g.ldb + n0 * 2 : (uint64_t)n0 * g.ldb));
        point();
    };
    auto mask = [&]() {
        if ((step + 1) * S::BK > g.ka) sa.stop_at(wave, (int)g.ka - (int)(step * S::BK));
        if ((step + 1) * S::BK > g.kb) sb.stop_at(wave, (int)g.kb - (int)(step * S::BK));
    };
    enter();
    mask();
    if (PAIRED) rb2 = tile_resource(uniform_address((const char *)g.b2 + (uint64_t)n0 * g.ldb2));
    uint32_t put = lds0 + wave * 1024, kbyte = step * S::ROW, slot = 0;
    auto load_one = [&](int n) {
        const int i = n % LOADS_PLANE, plane = n / LOADS_PLANE;
        if (i < LOADS_A) {
            load_to_lds(put + plane * S::PLANE + i * S::WAVES * 1024, sa.off[i], plane ? ra_lo : ra, ABYK ? 0u : kbyte);
        } else {
            const int k = i - LOADS_A;
            // a load of the four waves covers 32 rows (or 64): all of one half
            static_assert(!PAIRED || HALF % (S::WAVES * 1024 / S::ROW) == 0, "loads do not straddle halves");
            const bool second = PAIRED && k * S::WAVES * (1024 / S::ROW) % (2 * HALF) >= HALF;
            load_to_lds(put + plane * S::PLANE + A_BYTES + k * S::WAVES * 1024, sb.off[k], plane ? rb_lo : second ? rb2 : rb,
                        BBYK ? 0u : kbyte);
        }
    };
    auto next_stage = [&]() {
        ++loaded;
        slot = slot + 1 == BUFS ? 0 : slot + 1;
        put = lds0 + slot * S::BUF + wave * 1024;
        kbyte += S::ROW;
        if (++step == per) {
            step = 0, kbyte = 0;
            ++segment;  // never past the last: stages end there
            enter();
            place();
        } else if (ABYK || BBYK) {
            if (ABYK) sa.base += (uint64_t)S::BK * g.lda;
            if (BBYK) sb.base += (uint64_t)S::BK * g.ldb;
            point();
        }
        mask();
    };

    // Fragments: lane l holds row (by k: column) l%32 of a block and k = 16 *
    // quarter + 8 * (l/32) + 0..7.  By k they come as two transposing reads,
    // each of four k: sixteen lanes address four rows of sixteen columns.
    const uint32_t fr = lane & 31u, fc = lane >> 5;
    const uint32_t rows_a = (wm * MT * 32 + fr) * S::ROW, rows_b = A_BYTES + (wn * NT * 32 + fr) * S::ROW;
    const uint32_t tk = 8 * fc + (lane & 15u) / 4, tc = 2 * (lane >> 4 & 1u) + (lane >> 1 & 1u), te = (lane & 1u) * 8;
    uint32_t cols_a[MT], cols_b[NT];
    if (ABYK)
#pragma unroll
        for (int i = 0; i < MT; ++i)
            cols_a[i] = tk * (S::BM * 2) + ((wm * MT + i) * 4 + tc + SideA::turn(tk)) % SideA::CHUNKS * 16 + te;
    if (BBYK)
#pragma unroll
        for (int j = 0; j < NT; ++j)
            cols_b[j] = A_BYTES + tk * (S::BN * 2) + ((wn * NT + j) * 4 + tc + SideB::turn(tk)) % SideB::CHUNKS * 16 + te;
    auto transposed = [&](uint32_t at_byte, uint32_t pitch) {
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) s16x4 *P;
        const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(uintptr_t)(lds0 + at_byte));
        const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(uintptr_t)(lds0 + at_byte + 4 * pitch));
        return __builtin_bit_cast(F, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    constexpr int READS_PLANE = MT + NT, READS = PLANES * READS_PLANE;
    F fa[2][PLANES][MT], fb[2][PLANES][NT];
    auto read_one = [&](uint32_t at_buf, int quarter, int to, int n) {
        const int i = n % READS_PLANE, plane = n / READS_PLANE;
        const uint32_t o = at_buf + plane * S::PLANE;
        if (i < MT) {
            if (ABYK) fa[to][plane][i] = transposed(o + quarter * 16 * (S::BM * 2) + cols_a[i], S::BM * 2);
            else fa[to][plane][i] = *(const F *)(lds + o + rows_a + i * 32 * S::ROW + ((2 * quarter + fc) ^ SideA::swizzle(fr)) * 16);
        } else {
            const int j = i - MT;
            if (BBYK) fb[to][plane][j] = transposed(o + quarter * 16 * (S::BN * 2) + cols_b[j], S::BN * 2);
            else fb[to][plane][j] = *(const F *)(lds + o + rows_b + j * 32 * S::ROW + ((2 * quarter + fc) ^ SideB::swizzle(fr)) * 16);
        }
    };
    // product k of a quarter: with two planes three rounds over the accumulators
    auto multiply = [&](int from, int k) {
        const int i = k % (MT * NT) / NT, j = k % NT, round = k / (MT * NT);
        acc[i][j] = Frag<T>::mfma(fb[from][round == 1 ? PLANES - 1 : 0][j], fa[from][round == 2 ? PLANES - 1 : 0][i], acc[i][j]);
    };

#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;

    // A stage's loads are spread over SPREAD quarters, from the one behind the
    // barrier that frees its buffer on.
    constexpr int SPREAD = BUFS == 2 ? KQ - 1 : KQ, PER_Q = (LOADS + SPREAD - 1) / SPREAD;
    // Past the last stage the loads go on, into buffers that are not read
    // again, so that one constant count says which have landed.
    auto step_stage = [&]() {
        if (loaded + 1 < total) {
            next_stage();
        } else {
            slot = slot + 1 == BUFS ? 0 : slot + 1;
            put = lds0 + slot * S::BUF + wave * 1024;
        }
    };
    static_for<BUFS - 1>([&](auto) {
        static_for<LOADS>([&](auto i) { load_one(i.value); });
        step_stage();
    });
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((BUFS - 2) * LOADS) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    static_for<READS>([&](auto i) { read_one(0, 0, 0, i.value); });
    static_for<(PER_Q < LOADS ? PER_Q : LOADS)>([&](auto i) { load_one(i.value); });
    uint32_t buf = 0;
    for (uint32_t t = 0; t < total; ++t) {
        const uint32_t next = buf + S::BUF == S::LDS ? 0 : buf + S::BUF;
        static_for<KQ>([&](auto quarter) {
            constexpr int q = quarter.value, from = q & 1, to = from ^ 1;
            constexpr bool last = q == KQ - 1;
            if (last && t + 1 < total) {
                // This wave has its last fragments of the buffer, and its loads
                // of the next stage have landed; past the barrier that holds for
                // every wave.
                asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((BUFS - 2) * LOADS) : "memory");
                __builtin_amdgcn_s_barrier();
                asm volatile("" ::: "memory");
                step_stage();
            }
            constexpr int PRODUCTS = MT * NT * (PLANES == 2 ? 3 : 1), FIRST = (q + 1) % KQ * PER_Q;
            constexpr int HERE = (q + 1) % KQ >= SPREAD || FIRST >= LOADS ? 0 : LOADS - FIRST < PER_Q ? LOADS - FIRST : PER_Q;
            static_for<PRODUCTS>([&](auto product) {
                // reads go with the first half of the products, loads with all of them
                constexpr int k = product.value, r0 = upto(k, PRODUCTS, 2 * READS, READS), r1 = upto(k + 1, PRODUCTS, 2 * READS, READS);
                constexpr int l0 = upto(k, PRODUCTS, HERE, HERE), l1 = upto(k + 1, PRODUCTS, HERE, HERE);
                static_for<r1 - r0>([&](auto n) { read_one(last ? next : buf, last ? 0 : q + 1, to, r0 + n.value); });
                static_for<l1 - l0>([&](auto n) { load_one(FIRST + l0 + n.value); });
                __builtin_amdgcn_sched_barrier(0);
                multiply(from, k);
                __builtin_amdgcn_sched_barrier(0);
            });
        });
        buf = next;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    settle(acc);
}

// The same with a third buffer for A: what a stage needs of B is loaded in the first half
// of the one before, and of A in the second half of the one before that, so that the last
// loads that a barrier waits for are half a stage old, not a quarter.  (Two buffers of both
// are 128 KiB of a compute unit's 160 with the 256 x 256 tile: three of both do not fit.)
template <typename T, typename S, bool PAIRED, bool ABYK, bool BBYK>
__device__ __forceinline__ void gemm_tile_ahead(const GemmArgs &g, const TileAt at, char *lds, f32x16 (&acc)[S::MT][S::NT])
{
    constexpr int MT = S::MT, NT = S::NT, KQ = S::BK / 16;
    typedef Side<S, ABYK, S::BM> SideA;
    typedef Side<S, BBYK, S::BN> SideB;
    constexpr int LOADS_A = SideA::LOADS, LOADS_B = SideB::LOADS, LOADS = LOADS_A + LOADS_B;
    static_assert(!PAIRED || !BBYK, "pairs lie by rows");
    constexpr uint32_t A_BYTES = S::BM * S::ROW, B_BYTES = S::BN * S::ROW, B_AT = 3 * A_BYTES;
    typedef typename Frag<T>::type F;
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t wm = wave / S::WN, wn = wave % S::WN;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
    const uint32_t m0 = at.m * S::BM, n0 = at.n * (PAIRED ? S::BN / 2 : S::BN);
    constexpr int HALF = NT * 16;  // paired: columns of a wave

    const uint32_t per = g.steps * (kStepK / S::BK), all = g.segments * per;
    const uint32_t begin = (uint32_t)((uint64_t)all * at.split / g.splits);
    const uint32_t total = (uint32_t)((uint64_t)all * (at.split + 1) / g.splits) - begin;

    // where an operand's next loads are, and where in LDS they go
    struct Next {
        uint32_t segment, step, loaded, kbyte, slot, put;
        u32x4v from;
    };
    SideA sa;
    SideB sb;
    Next na{begin / per, begin % per, 0, begin % per * S::ROW, 0, lds0 + wave * 1024}, nb = na;
    nb.put += B_AT;
    u32x4v rb2;
    auto place_a = [&]() {
        sa.place(wave, m0, g.m, [&](uint32_t row, uint32_t first) {
            return ABYK ? row * g.lda : ((first + row < g.m ? first + row : g.m - 1) - first) * g.lda;
        });
        sa.base = uniform_address((const char *)g.a[na.segment] + at.batch * g.batch_a +
                                  (ABYK ? (uint64_t)na.step * S::BK * g.lda + m0 * 2 : (uint64_t)m0 * g.lda));
    };
    auto place_b = [&]() {
        sb.place(wave, n0, g.n, [&](uint32_t row, uint32_t first) {
            if (BBYK) return row * g.ldb;
            uint32_t ld = g.ldb, r = row;
            if (PAIRED) {
                const uint32_t in = row % (2 * HALF);
                ld = in < HALF ? g.ldb : g.ldb2;
                r = row / (2 * HALF) * HALF + in % HALF;
            }
            return ((first + r < g.n ? first + r : g.n - 1) - first) * ld;
        });
        sb.base = uniform_address((const char *)g.b[nb.segment] + at.batch * g.batch_b +
                                  (BBYK ? (uint64_t)nb.step * S::BK * g.ldb + n0 * 2 : (uint64_t)n0 * g.ldb));
    };
    auto ready_a = [&]() {
        na.from = tile_resource(sa.base);
        if ((na.step + 1) * S::BK > g.ka) sa.stop_at(wave, (int)g.ka - (int)(na.step * S::BK));
    };
    auto ready_b = [&]() {
        nb.from = tile_resource(sb.base);
        if ((nb.step + 1) * S::BK > g.kb) sb.stop_at(wave, (int)g.kb - (int)(nb.step * S::BK));
    };
    place_a(), place_b(), ready_a(), ready_b();
    if (PAIRED) rb2 = tile_resource(uniform_address((const char *)g.b2 + (uint64_t)n0 * g.ldb2));
    // Past the last stage the loads go on, into buffers that are not read again, so that
    // one constant count says which have landed.
    auto next_a = [&]() {
        na.slot = na.slot == 2 ? 0 : na.slot + 1;
        na.put = lds0 + na.slot * A_BYTES + wave * 1024;
        if (++na.loaded >= total) return;
        na.kbyte += S::ROW;
        if (++na.step == per) na.step = 0, na.kbyte = 0, ++na.segment, place_a();
        else if (ABYK) sa.base += (uint64_t)S::BK * g.lda;
        ready_a();
    };
    auto next_b = [&]() {
        nb.slot ^= 1;
        nb.put = lds0 + B_AT + nb.slot * B_BYTES + wave * 1024;
        if (++nb.loaded >= total) return;
        nb.kbyte += S::ROW;
        if (++nb.step == per) nb.step = 0, nb.kbyte = 0, ++nb.segment, place_b();
        else if (BBYK) sb.base += (uint64_t)S::BK * g.ldb;
        ready_b();
    };
    auto load_a = [&](int i) { load_to_lds(na.put + i * S::WAVES * 1024, sa.off[i], na.from, ABYK ? 0u : na.kbyte); };
    auto load_b = [&](int k) {
        // a load of the four waves covers 32 rows (or 64): all of one half
        static_assert(!PAIRED || HALF % (S::WAVES * 1024 / S::ROW) == 0, "loads do not straddle halves");
        const bool second = PAIRED && k * S::WAVES * (1024 / S::ROW) % (2 * HALF) >= HALF;
        load_to_lds(nb.put + k * S::WAVES * 1024, sb.off[k], second ? rb2 : nb.from, BBYK ? 0u : nb.kbyte);
    };
    auto load_one = [&](int n) {  // B's, then A's
        if (n < LOADS_B) load_b(n);
        else load_a(n - LOADS_B);
    };

    // Fragments, as above.
    const uint32_t fr = lane & 31u, fc = lane >> 5;
    const uint32_t rows_a = (wm * MT * 32 + fr) * S::ROW, rows_b = B_AT + (wn * NT * 32 + fr) * S::ROW;
    const uint32_t tk = 8 * fc + (lane & 15u) / 4, tc = 2 * (lane >> 4 & 1u) + (lane >> 1 & 1u), te = (lane & 1u) * 8;
    uint32_t cols_a[MT], cols_b[NT];
    if (ABYK)
#pragma unroll
        for (int i = 0; i < MT; ++i)
            cols_a[i] = tk * (S::BM * 2) + ((wm * MT + i) * 4 + tc + SideA::turn(tk)) % SideA::CHUNKS * 16 + te;
    if (BBYK)
#pragma unroll
        for (int j = 0; j < NT; ++j)
            cols_b[j] = B_AT + tk * (S::BN * 2) + ((wn * NT + j) * 4 + tc + SideB::turn(tk)) % SideB::CHUNKS * 16 + te;
    auto transposed = [&](uint32_t at_byte, uint32_t pitch) {
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) s16x4 *P;
        const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(uintptr_t)(lds0 + at_byte));
        const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(uintptr_t)(lds0 + at_byte + 4 * pitch));
        return __builtin_bit_cast(F, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    constexpr int READS = MT + NT;
    F fa[2][MT], fb[2][NT];
    auto read_one = [&](uint32_t at_a, uint32_t at_b, int quarter, int to, int n) {
        if (n < MT) {
            if (ABYK) fa[to][n] = transposed(at_a + quarter * 16 * (S::BM * 2) + cols_a[n], S::BM * 2);
            else fa[to][n] = *(const F *)(lds + at_a + rows_a + n * 32 * S::ROW + ((2 * quarter + fc) ^ SideA::swizzle(fr)) * 16);
        } else {
            const int j = n - MT;
            if (BBYK) fb[to][j] = transposed(at_b + quarter * 16 * (S::BN * 2) + cols_b[j], S::BN * 2);
            else fb[to][j] = *(const F *)(lds + at_b + rows_b + j * 32 * S::ROW + ((2 * quarter + fc) ^ SideB::swizzle(fr)) * 16);
        }
    };

#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;

    constexpr int PER_Q = (LOADS + KQ - 1) / KQ;
    static_for<LOADS_A>([&](auto i) { load_a(i.value); });
    static_for<LOADS_B>([&](auto i) { load_b(i.value); });
    next_a(), next_b();
    static_for<LOADS_A>([&](auto i) { load_a(i.value); });
    next_a();
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LOADS_A) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    static_for<READS>([&](auto i) { read_one(0, 0, 0, 0, i.value); });
    static_for<PER_Q>([&](auto i) { load_one(i.value); });
    uint32_t buf_a = 0, buf_b = 0;
    for (uint32_t t = 0; t < total; ++t) {
        const uint32_t then_a = buf_a == 2 * A_BYTES ? 0 : buf_a + A_BYTES, then_b = B_BYTES - buf_b;
        static_for<KQ>([&](auto quarter) {
            constexpr int q = quarter.value, from = q & 1, to = from ^ 1;
            constexpr bool last = q == KQ - 1;
            if (last && t + 1 < total) {
                // This wave has its last fragments of the buffers, and its loads of the
                // next stage have landed, A's behind them not; past the barrier that holds
                // for every wave.
                asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(LOADS_A) : "memory");
                __builtin_amdgcn_s_barrier();
                asm volatile("" ::: "memory");
                next_a(), next_b();
            }
            constexpr int PRODUCTS = MT * NT, FIRST = (q + 1) % KQ * PER_Q;
            constexpr int HERE = FIRST >= LOADS ? 0 : LOADS - FIRST < PER_Q ? LOADS - FIRST : PER_Q;
            static_for<PRODUCTS>([&](auto product) {
                constexpr int k = product.value, r0 = upto(k, PRODUCTS, 2 * READS, READS), r1 = upto(k + 1, PRODUCTS, 2 * READS, READS);
                constexpr int l0 = upto(k, PRODUCTS, HERE, HERE), l1 = upto(k + 1, PRODUCTS, HERE, HERE);
                static_for<r1 - r0>([&](auto n) { read_one(last ? then_a : buf_a, last ? then_b : buf_b, last ? 0 : q + 1, to, r0 + n.value); });
                static_for<l1 - l0>([&](auto n) { load_one(FIRST + l0 + n.value); });
                __builtin_amdgcn_sched_barrier(0);
                acc[k / NT][k % NT] = Frag<T>::mfma(fb[from][k % NT], fa[from][k / NT], acc[k / NT][k % NT]);
                __builtin_amdgcn_sched_barrier(0);
            });
        });
        buf_a = then_a, buf_b = then_b;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    settle(acc);
}

template <typename T, typename S, bool PAIRED, bool ABYK = false, bool BBYK = false>
__device__ __forceinline__ void gemm_tile(const GemmArgs &g, const TileAt at, char *lds, f32x16 (&acc)[S::MT][S::NT])
{
    if constexpr (S::AHEAD) gemm_tile_ahead<T, S, PAIRED, ABYK, BBYK>(g, at, lds, acc);
    else gemm_tile_even<T, S, PAIRED, ABYK, BBYK>(g, at, lds, acc);
}

// 32 rows of a wave's results in its own part of LDS, so that a row's bytes can
// leave together.  value(j, r): the lane's value at column j*32 + 8*(r/4) +
// 4*(l/32) + r%4 of COLS, row l%32.
template <typename O, int COLS> constexpr int kStagePitch = COLS * (int)sizeof(O) + 16;
template <typename O, int COLS> constexpr int kStageBytes = 32 * kStagePitch<O, COLS>;
template <typename O, int COLS, typename V> __device__ __forceinline__ void stage_rows(char *lds, V value)
{
    constexpr int E = sizeof(O), PITCH = kStagePitch<O, COLS>;
    const uint32_t lane = threadIdx.x & 63u;
    typedef O O4 __attribute__((ext_vector_type(4)));
    char *at = lds + (lane & 31u) * PITCH + (lane >> 5) * 4 * E;
    asm volatile("" ::: "memory");
#pragma unroll
    for (int j = 0; j < COLS / 32; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            O4 v;
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = (O)value(j, q * 4 + k);
            *(O4 *)(at + (j * 32 + q * 8) * E) = v;
        }
    asm volatile("" ::: "memory");
}

// 32 rows of a padded matrix on their way to the lanes that hold their
// elements' sums: loaded by rows, a whole row's bytes together, and later staged
// in LDS.  Rows of at least `cols` elements (a multiple of 8); 0: no rows.
template <typename O, int COLS> struct RowsAhead {
    static constexpr int PER = 16 / (int)sizeof(O), LANES = COLS / PER, N = 32 * LANES / 64;
    u32x4v v[N];
    __device__ __forceinline__ void load(const O *from, uint64_t ld, uint32_t cols)
    {
        const uint32_t lane = threadIdx.x & 63u;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const uint32_t r = (n * 64 + lane) / LANES, c = (n * 64 + lane) % LANES * PER;
            if (c < cols) v[n] = *(const u32x4v *)(from + r * ld + c);
        }
    }
    __device__ __forceinline__ void stage(char *lds) const
    {
        const uint32_t lane = threadIdx.x & 63u;
        asm volatile("" ::: "memory");
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const uint32_t r = (n * 64 + lane) / LANES, c = (n * 64 + lane) % LANES * PER;
            *(u32x4v *)(lds + r * kStagePitch<O, COLS> + c * sizeof(O)) = v[n];
        }
        asm volatile("" ::: "memory");
    }
    // the staged elements of columns j*32 + 8*q + 4*(l/32) on, row l%32
    static __device__ __forceinline__ void take(const char *lds, int j, int q, float *out)
    {
        const uint32_t lane = threadIdx.x & 63u;
        typedef O O4 __attribute__((ext_vector_type(4)));
        const O4 x = *(const O4 *)(lds + (lane & 31u) * kStagePitch<O, COLS> + (j * 32 + q * 8 + (lane >> 5) * 4) * sizeof(O));
#pragma unroll
        for (int k = 0; k < 4; ++k) out[k] = (float)x[k];
    }
};

// Writes staged rows to `out` and the rows behind it: of the 32 rows those in
// [from, until), of the columns the first `cols`.
template <typename O, int COLS>
__device__ __forceinline__ void write_rows(const char *lds, O *out, uint64_t ld, uint32_t from, uint32_t until, uint32_t cols)
{
    constexpr int E = sizeof(O), PITCH = kStagePitch<O, COLS>, PER = 16 / E, LANES = COLS / PER;  // of a row
    static_assert(COLS % PER == 0 && 32 * LANES % 64 == 0, "whole rows and waves");
    typedef O OV __attribute__((ext_vector_type(PER)));
    typedef O OU __attribute__((ext_vector_type(PER), aligned(E)));
    const uint32_t lane = threadIdx.x & 63u;
    const bool whole = from == 0 && until >= 32 && cols >= COLS;
#pragma unroll
    for (int k0 = 0; k0 < 32 * LANES; k0 += 64) {
        const uint32_t r = (k0 + lane) / LANES, c = (k0 + lane) % LANES * PER;
        O *to = out + r * ld + c;
        const char *at = lds + r * PITCH + c * E;
        if (whole) {
            *(OU *)to = *(const OV *)at;
        } else if (r >= from && r < until) {
            if (c + PER <= cols) *(OU *)to = *(const OV *)at;
            else
                for (uint32_t k = c; k < cols; ++k) to[k - c] = ((const O *)at)[k - c];
        }
    }
}

// Writes staged rows of a 16-bit type transposed: column c to row c of `out`, for
// the first `cols` columns, `rows` of the 32 elements (a multiple of 8, or all).
template <typename O, int COLS>
__device__ __forceinline__ void write_columns(const char *lds, O *out, uint64_t ld, uint32_t rows, uint32_t cols)
{
    static_assert(sizeof(O) == 2, "a 16-bit type");
    constexpr int PITCH = kStagePitch<O, COLS>;
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef short s16x8 __attribute__((ext_vector_type(8)));
    typedef s16x8 Out __attribute__((aligned(2)));
    typedef __attribute__((address_space(3))) s16x4 *P;
    const uint32_t lane = threadIdx.x & 63u, r8 = (lane >> 4) * 8;
    // sixteen lanes: rows r8..r8+3 of sixteen columns, then the next four rows
    const uint32_t from = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char *)lds +
                          (r8 + (lane & 15u) / 4) * PITCH + (lane & 3u) * 8;
#pragma unroll
    for (int c0 = 0; c0 < COLS; c0 += 16) {
        const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(uintptr_t)(from + c0 * 2));
        const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(uintptr_t)(from + c0 * 2 + 4 * PITCH));
        const uint32_t c = c0 + (lane & 15u);
        if (c < cols && r8 < rows) *(Out *)(out + c * ld + r8) = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    }
}

}  // namespace dev
}  // namespace ar
