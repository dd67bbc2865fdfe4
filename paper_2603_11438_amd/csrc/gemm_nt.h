// Matrix products C[m][n] = sum_k A[m][k] B[n][k] on gfx950's matrix units, for
// kernels that bring their own epilogue.
//
// Both operands are row-major with k contiguous ("NT"), 16-bit, rows 16-byte
// aligned, k a multiple of 64; callers lay out what is not so.  A product may
// run over several (A, B) pairs ("segments") of one k length one after another,
// all into the same sums: planes of a split operand, or [dG dU] times [Wg; Wu].
//
// A workgroup of four waves, one per SIMD, owns a tile of MT*64 x NT*64; each
// wave holds MT x NT accumulators of 32 x 32 in registers.  With MT = NT = 4 a
// step of k = 16 costs a wave 8 KiB of LDS reads for 512 cycles of matrix work:
// at 128 bytes a cycle the four waves' reads and the tile's writes fill three
// quarters of the LDS' time, where eight waves of half the tile fill all of it.
//
// k advances in steps of 64 (128 bytes of a row) through two LDS buffers.
// Loads go from memory straight into LDS (16 bytes a lane) and are issued a
// whole step ahead: once every wave has read the last fragments of a buffer,
// the step after next is loaded into it.  Fragments for the next quarter of a
// step are read while the matrix units work on this one, across steps too.
//
// A row's eight 16-byte chunks are stored in the order chunk ^ (row & 7), by
// permuting which chunk a lane loads: eight rows' equal chunks, which one read
// touches together, then lie in eight different bank groups.
#pragma once

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

constexpr int kMaxSegments = 3;
constexpr int kStepK = 64;
constexpr uint32_t kRowBytes = kStepK * 2;  // of a row in one LDS buffer

// Rows of one tile are reached by 32-bit offsets from the tile's first row.
inline bool gemm_reaches(uint64_t row_bytes, uint64_t k_bytes) { return row_bytes * 256 + k_bytes < (1ull << 31); }

struct GemmArgs {
    const void *a[kMaxSegments], *b[kMaxSegments];
    const void *b2;             // paired operands: the second of each pair of columns (one segment)
    uint32_t segments, steps;   // steps of 64 per segment
    uint32_t lda, ldb, ldb2;    // bytes
    uint32_t m, n;              // rows of A and of B (paired: of each)
    uint32_t tiles_m, tiles_n;
    uint64_t batch_a, batch_b;  // bytes between the matrices of a batch
    uint32_t batch;
    uint32_t splits;            // runs of steps that k is split into (grid.y); 1: not split
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

template <int MT, int NT> constexpr int kGemmLds = 2 * (MT + NT) * 64 * (int)kRowBytes;

// The products of one tile.  acc[i][j][r], lane l: row i*32 + l%32 of the wave's
// rows, column j*32 + 8*(r/4) + 4*(l/32) + r%4 of its columns (B's fragment is
// the instruction's first operand, so a lane holds four neighbouring columns).
//
// PAIRED: of a wave's NT*32 rows of B the first half comes from b, the second
// half from b2, both at the same rows: the wave then holds both products of the
// same columns.
//
// With k split, workgroup blockIdx.y of g.splits adds up its run of the steps
// (never empty: there are at least as many steps as splits).
template <typename T, int MT, int NT, bool PAIRED>
__device__ __forceinline__ void gemm_tile(const GemmArgs &g, const TileAt at, char *lds, f32x16 (&acc)[MT][NT])
{
    constexpr int BM = MT * 64, BN = NT * 64, LOADS_A = BM / 32, LOADS_B = BN / 32;
    constexpr uint32_t A_BYTES = BM * kRowBytes, BUF = (BM + BN) * kRowBytes;
    typedef typename Frag<T>::type F;
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t wm = wave >> 1, wn = wave & 1u;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;

    // Loads of this wave: eight rows each, row 8 * (4 * i + wave) of the tile on.
    const uint32_t row8 = lane >> 3, chunk = ((lane & 7u) ^ row8) * 16;
    const uint32_t m0 = at.m * BM, n0 = at.n * (PAIRED ? BN / 2 : BN);
    uint32_t off_a[LOADS_A], off_b[LOADS_B];
#pragma unroll
    for (int i = 0; i < LOADS_A; ++i) {
        const uint32_t r = m0 + (i * 4 + wave) * 8 + row8;
        off_a[i] = ((r < g.m ? r : g.m - 1) - m0) * g.lda + chunk;
    }
    constexpr int HALF = NT * 16;  // paired: columns of a wave
#pragma unroll
    for (int i = 0; i < LOADS_B; ++i) {
        uint32_t r = (i * 4 + wave) * 8 + row8;
        uint32_t ld = g.ldb;
        if (PAIRED) {
            const uint32_t in = r % (2 * HALF);
            ld = in < HALF ? g.ldb : g.ldb2;
            r = r / (2 * HALF) * HALF + in % HALF;
        }
        r += n0;
        off_b[i] = ((r < g.n ? r : g.n - 1) - n0) * ld + chunk;
    }
    const uint32_t all = g.segments * g.steps;
    const uint32_t begin = (uint32_t)((uint64_t)all * blockIdx.y / g.splits);
    const uint32_t total = (uint32_t)((uint64_t)all * (blockIdx.y + 1) / g.splits) - begin;
    uint32_t segment = begin / g.steps, step = begin % g.steps;  // of the next load
    u32x4v ra, rb, rb2;
    auto enter = [&]() {
        ra = tile_resource((const char *)g.a[segment] + at.batch * g.batch_a + (uint64_t)m0 * g.lda);
        rb = tile_resource((const char *)g.b[segment] + at.batch * g.batch_b + (uint64_t)n0 * g.ldb);
    };
    enter();
    rb2 = PAIRED ? tile_resource((const char *)g.b2 + (uint64_t)n0 * g.ldb2) : rb;
    auto load = [&](uint32_t buf) {
        const uint32_t base = lds0 + buf * BUF + wave * 1024, k = step * kRowBytes;
#pragma unroll
        for (int i = 0; i < LOADS_A; ++i) load_to_lds(base + i * 4096, off_a[i], ra, k);
#pragma unroll
        for (int i = 0; i < LOADS_B; ++i) {
            // rows (4 * i + wave) * 8: the halves of a pair change every HALF / 8 loads
            const bool second = PAIRED && (((i * 4 + wave) * 8) % (2 * HALF)) >= HALF;
            load_to_lds(base + A_BYTES + i * 4096, off_b[i], second ? rb2 : rb, k);
        }
        if (++step == g.steps) {
            step = 0;
            if (++segment < g.segments) enter();
        }
    };

    // Fragment reads: row l%32 of a 32-row block, chunk 2 * quarter + l/32.
    const uint32_t fr = lane & 31u, fc = lane >> 5, sw = fr & 7u;
    const uint32_t row_a = (wm * MT * 32 + fr) * kRowBytes, row_b = A_BYTES + (wn * NT * 32 + fr) * kRowBytes;
    F fa[2][MT], fb[2][NT];
    auto read = [&](uint32_t buf, int quarter, int to) {
        const char *p = lds + buf * BUF + (((2 * quarter + fc) ^ sw) * 16);
#pragma unroll
        for (int i = 0; i < MT; ++i) fa[to][i] = *(const F *)(p + row_a + i * 32 * kRowBytes);
#pragma unroll
        for (int j = 0; j < NT; ++j) fb[to][j] = *(const F *)(p + row_b + j * 32 * kRowBytes);
    };
    auto multiply = [&](int from) {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) acc[i][j] = Frag<T>::mfma(fb[from][j], fa[from][i], acc[i][j]);
    };

#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;

    load(0);
    if (total > 1) load(1);
    if (total > 1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LOADS_A + LOADS_B) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    read(0, 0, 0);
    for (uint32_t t = 0; t < total; ++t) {
        const uint32_t buf = t & 1u;
        read(buf, 1, 1);
        multiply(0);
        read(buf, 2, 0);
        multiply(1);
        read(buf, 3, 1);
        multiply(0);
        if (t + 1 < total) {
            // This wave has its last fragments of the buffer, and its loads of
            // the next step (issued a step ago) have landed; past the barrier
            // that holds for every wave.
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            if (t + 2 < total) load(buf);
            read(buf ^ 1u, 0, 0);
        }
        multiply(1);
    }
    // Every wave is done with the buffers: the epilogue may use them.
    __syncthreads();
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
