// Matrix products C[m][n] = sum_k A[m][k] B[n][k] on gfx950's matrix units, for
// kernels that bring their own epilogue.
//
// Both operands are row-major with k contiguous ("NT"), 16-bit, rows 16-byte
// aligned, k a multiple of 64; callers lay out what is not so.  A product may
// run over several (A, B) pairs ("segments") of one k length one after another,
// all into the same sums ([dG dU] times [Wg; Wu]).  Operands in two planes, hi
// and lo, are multiplied as hi hi + hi lo + lo hi.
//
// A workgroup of four waves, one per SIMD, owns a tile; each wave holds MT x NT
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
// groups of four banks (SQ_LDS_BANK_CONFLICT: 0; with row & 7 a read took
// twice as long).
//
// Rate, bf16, 8192 x 8192 x 8192: 856 us, 1284 TFLOP/s with the 256 x 256 tile,
// at 1.75 GHz: the board's power limit has the clock.  With every load an L2 hit
// the same kernel takes 794 us, so the rest is misses that a stage's lead does
// not cover.  Smaller tiles: 128 x 128 1020 us, 64 x 64 1525 us.
#pragma once

#include <type_traits>
#include <utility>

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
constexpr int kStepK = 64;  // k is a multiple of this

// Rows of one tile are reached by 32-bit offsets from the tile's first row.
inline bool gemm_reaches(uint64_t row_bytes, uint64_t k_bytes) { return row_bytes * 256 + k_bytes < (1ull << 31); }

struct GemmArgs {
    const void *a[kMaxSegments], *b[kMaxSegments];
    const void *b2;             // paired operands: the second of each pair of columns (one segment)
    uint64_t a_lo, b_lo;        // two planes: bytes from the hi plane to the lo plane (one segment)
    uint32_t segments, steps;   // steps of 64 per segment
    uint32_t lda, ldb, ldb2;    // bytes
    uint32_t m, n;              // rows of A and of B (paired: of each)
    uint32_t tiles_m, tiles_n;
    uint64_t batch_a, batch_b;  // bytes between the matrices of a batch
    uint32_t batch;
    uint32_t splits;            // runs of stages that k is split into (grid.y); 1: not split
};

__device__ __forceinline__ u32x4v tile_resource(const void *p)
{
    const uint64_t a = (uint64_t)p;
    u32x4v r;
    r.x = __builtin_amdgcn_readfirstlane((uint32_t)a);
    r.y = __builtin_amdgcn_readfirstlane((uint32_t)(a >> 32) & 0xffffu);
    r.z = 0x80000000u;  // offsets stay below 2^31 (gemm_reaches); rows are clamped to the matrix
    r.w = 0x00020000u;
    return r;
}

// 64 lanes' 16 bytes each into 1 KiB of LDS from `lds` on, in lane order.  The
// load has no output register: it is complete when vmcnt says so.  Nothing else
// in these kernels uses m0.
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
    at.batch = t / per;
    t %= per;
    const uint32_t group = t / (kGroupRows * tiles_n), first = group * kGroupRows;
    const uint32_t rows = tiles_m - first < kGroupRows ? tiles_m - first : kGroupRows;
    t -= first * tiles_n;
    at.m = first + t % rows;
    at.n = t / rows;
    return at;
}
// Tiles on and below the diagonal, by rows.
__device__ __forceinline__ TileAt tile_at_lower(uint32_t tiles, uint32_t batch)
{
    const uint32_t per = tiles * (tiles + 1) / 2;
    uint32_t t = xcd_run(blockIdx.x, per * batch);
    TileAt at;
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

// The shape of a workgroup's tile and pipeline: 2 x 2 waves of MT x NT blocks of
// 32 x 32, PLANES planes of each operand, k in stages of BK through BUFS buffers.
template <int MT_, int NT_, int PLANES_, int BK_, int BUFS_> struct Shape {
    static constexpr int MT = MT_, NT = NT_, PLANES = PLANES_, BK = BK_, BUFS = BUFS_;
    static constexpr int WM = 2, WN = 2, WAVES = WM * WN, THREADS = 64 * WAVES, BM = WM * MT * 32, BN = WN * NT * 32;
    static constexpr int ROW = BK * 2;                        // bytes of a row in a buffer
    static constexpr int PLANE = (BM + BN) * ROW;             // A's rows, then B's
    static constexpr int BUF = PLANES * PLANE, LDS = BUFS * BUF;
    static constexpr int ROWS_PER_LOAD = 1024 / ROW, LOADS_A = BM / ROWS_PER_LOAD / WAVES, LOADS_B = BN / ROWS_PER_LOAD / WAVES;
    static constexpr int LOADS_PLANE = LOADS_A + LOADS_B, LOADS = PLANES * LOADS_PLANE;  // of a wave and stage
    static_assert(BM % (ROWS_PER_LOAD * WAVES) == 0 && BN % (ROWS_PER_LOAD * WAVES) == 0, "whole loads");
};

// The products of one tile.  acc[i][j][r], lane l: row i*32 + l%32 of the wave's
// rows, column j*32 + 8*(r/4) + 4*(l/32) + r%4 of its columns (B's fragment is
// the instruction's first operand, so a lane holds four neighbouring columns).
//
// PAIRED: of a wave's NT*32 rows of B the first half comes from b, the second
// half from b2, both at the same rows: the wave then holds both products of the
// same columns.
//
// With k split, workgroup blockIdx.y of g.splits adds up its run of the stages
// (never empty: there are at least as many steps as splits).
template <typename T, typename S, bool PAIRED>
__device__ __forceinline__ void gemm_tile(const GemmArgs &g, const TileAt at, char *lds, f32x16 (&acc)[S::MT][S::NT])
{
    constexpr int MT = S::MT, NT = S::NT, PLANES = S::PLANES, LOADS_A = S::LOADS_A, LOADS_B = S::LOADS_B, LOADS = S::LOADS;
    constexpr int LOADS_PLANE = S::LOADS_PLANE, RPL = S::ROWS_PER_LOAD;
    static_assert(PLANES == 1 || !PAIRED, "pairs have one plane");
    constexpr int CHUNKS = S::ROW / 16, KQ = S::BK / 16, BUFS = S::BUFS;
    constexpr uint32_t A_BYTES = S::BM * S::ROW;
    typedef typename Frag<T>::type F;
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t wm = wave / S::WN, wn = wave % S::WN;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
    auto swizzle = [](uint32_t row) { return CHUNKS == 8 ? (row >> 1) & 7u : (row >> 2) & 3u; };

    // Loads of this wave: RPL rows each, from row RPL * (WAVES * i + wave) of the tile on.
    const uint32_t lrow = lane / CHUNKS;
    const uint32_t m0 = at.m * S::BM, n0 = at.n * (PAIRED ? S::BN / 2 : S::BN);
    constexpr int HALF = NT * 16;  // paired: columns of a wave
    uint32_t off[LOADS_PLANE];
#pragma unroll
    for (int i = 0; i < LOADS_A; ++i) {
        const uint32_t t = (i * S::WAVES + wave) * RPL + lrow, r = m0 + t;
        off[i] = ((r < g.m ? r : g.m - 1) - m0) * g.lda + ((lane % CHUNKS) ^ swizzle(t)) * 16;
    }
#pragma unroll
    for (int i = 0; i < LOADS_B; ++i) {
        const uint32_t t = (i * S::WAVES + wave) * RPL + lrow;
        uint32_t r = t, ld = g.ldb;
        if (PAIRED) {
            const uint32_t in = t % (2 * HALF);
            ld = in < HALF ? g.ldb : g.ldb2;
            r = t / (2 * HALF) * HALF + in % HALF;
        }
        r += n0;
        off[LOADS_A + i] = ((r < g.n ? r : g.n - 1) - n0) * ld + ((lane % CHUNKS) ^ swizzle(t)) * 16;
    }
    const uint32_t per = g.steps * (64 / S::BK), all = g.segments * per;
    const uint32_t begin = (uint32_t)((uint64_t)all * blockIdx.y / g.splits);
    const uint32_t total = (uint32_t)((uint64_t)all * (blockIdx.y + 1) / g.splits) - begin;
    uint32_t segment = begin / per, step = begin % per, loaded = 0;  // of the next load
    u32x4v ra, rb, rb2;  // rb2: the second of a pair; ra_lo, rb_lo: the lo planes
    auto enter = [&]() {
        ra = tile_resource((const char *)g.a[segment] + at.batch * g.batch_a + (uint64_t)m0 * g.lda);
        rb = tile_resource((const char *)g.b[segment] + at.batch * g.batch_b + (uint64_t)n0 * g.ldb);
    };
    enter();
    rb2 = PAIRED ? tile_resource((const char *)g.b2 + (uint64_t)n0 * g.ldb2) : rb;
    u32x4v ra_lo = ra, rb_lo = rb;
    if (PLANES == 2) {
        ra_lo = tile_resource((const char *)g.a[0] + g.a_lo + at.batch * g.batch_a + (uint64_t)m0 * g.lda);
        rb_lo = tile_resource((const char *)g.b[0] + g.b_lo + at.batch * g.batch_b + (uint64_t)n0 * g.ldb);
    }
    uint32_t put = lds0 + wave * 1024, kbyte = step * S::ROW, slot = 0;
    auto load_one = [&](int n) {
        const int i = n % LOADS_PLANE, plane = n / LOADS_PLANE;
        if (i < LOADS_A) {
            load_to_lds(put + plane * S::PLANE + i * S::WAVES * 1024, off[i], plane ? ra_lo : ra, kbyte);
        } else {
            const int k = i - LOADS_A;
            const bool second = PAIRED && (((k * S::WAVES + wave) * RPL) % (2 * HALF)) >= HALF;
            load_to_lds(put + plane * S::PLANE + A_BYTES + k * S::WAVES * 1024, off[i], plane ? rb_lo : second ? rb2 : rb, kbyte);
        }
    };
    auto next_stage = [&]() {
        ++loaded;
        slot = slot + 1 == BUFS ? 0 : slot + 1;
        put = lds0 + slot * S::BUF + wave * 1024;
        kbyte += S::ROW;
        if (++step == per) {
            step = 0, kbyte = 0;
            if (++segment < g.segments) enter();
        }
    };

    const uint32_t fr = lane & 31u, fc = lane >> 5, sw = swizzle(fr);
    const char *pa = lds + (wm * MT * 32 + fr) * S::ROW, *pb = lds + A_BYTES + (wn * NT * 32 + fr) * S::ROW;
    constexpr int READS_PLANE = MT + NT, READS = PLANES * READS_PLANE;
    F fa[2][PLANES][MT], fb[2][PLANES][NT];
    auto read_one = [&](uint32_t at_buf, int quarter, int to, int n) {
        const int i = n % READS_PLANE, plane = n / READS_PLANE;
        const uint32_t o = at_buf + plane * S::PLANE + (((2 * quarter + fc) ^ sw) * 16);
        if (i < MT) fa[to][plane][i] = *(const F *)(pa + o + i * 32 * S::ROW);
        else fb[to][plane][i - MT] = *(const F *)(pb + o + (i - MT) * 32 * S::ROW);
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

// Writes 32 rows of a wave's results through its own part of LDS, so that a
// row's bytes leave together.  value(j, r): the lane's value at column
// j*32 + 8*(r/4) + 4*(l/32) + r%4 of COLS, row l%32.  row(r): where row r goes
// (its first column), or null for none; `cols` columns are written.
template <typename O, int COLS, typename V, typename R>
__device__ __forceinline__ void store_32_rows(char *lds, uint32_t cols, V value, R row)
{
    constexpr int E = sizeof(O), PITCH = COLS * E + 16, PER = 16 / E;  // elements a lane stores at once
    constexpr int LANES = COLS / PER;  // of a row
    static_assert(COLS % PER == 0 && 32 * LANES % 64 == 0, "whole rows and waves");
    const uint32_t lane = threadIdx.x & 63u;
    typedef O O4 __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int j = 0; j < COLS / 32; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            O4 v;
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = (O)value(j, q * 4 + k);
            *(O4 *)(lds + (lane & 31u) * PITCH + (j * 32 + q * 8 + (lane >> 5) * 4) * E) = v;
        }
    asm volatile("" ::: "memory");
#pragma unroll
    for (int k0 = 0; k0 < 32 * LANES; k0 += 64) {
        const uint32_t r = (k0 + lane) / LANES, c = (k0 + lane) % LANES * PER;
        O *to = row(r);
        const O *from = (const O *)(lds + r * PITCH) + c;
        if (to) {
            if (c + PER <= cols) {
                typedef O OV __attribute__((ext_vector_type(PER)));
                typedef O OU __attribute__((ext_vector_type(PER), aligned(E)));
                *(OU *)(to + c) = *(const OV *)from;
            } else {
                for (uint32_t k = c; k < cols; ++k) to[k] = from[k - c];
            }
        }
    }
    asm volatile("" ::: "memory");
}
template <typename O, int COLS> constexpr int kStageBytes = 32 * (COLS * (int)sizeof(O) + 16);

}  // namespace dev
}  // namespace ar
