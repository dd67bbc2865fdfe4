// Attention over packed sequences (gfx950), forward and backward (formulas and
// layouts in ar_ops.h).
//
// The queries of one key head and its group of heads are the rows of a tile: row
// r is query r / group of the sequence, head r % group of the group.  Single
// queries of many heads then share a read of the keys, and a prompt's tile has
// the rows of few positions, so little of it is masked.
//
// Everything is computed transposed, S^T = K Q^T and O^T = V^T P^T, so that a lane
// holds one query: the row's maximum and sum are sums in the lane and one exchange
// with lane ^ 32.  The instruction's sums lie so that eight neighbouring ones are,
// rounded, a fragment of P^T for the next product, if V's keys are taken in the same
// order (4 h + 0..3, 8 + 4 h + 0..3 for lane half h): P never leaves its lane.
//
// What bounds it, 32 heads over 8 of 128, bf16.  Prompts, 16384 tokens in four: 765 us,
// 1050 TFLOP/s, the board's power (matrix units busy 57 % of the cycles, vector units 51 %,
// at 1.7 GHz).  Single tokens over 160 to 15000 keys, 32 of them: 193 us, 5.0 TB/s of the
// cache.  Training, 2 x 4096: 1235 us; dq 1050 TFLOP/s as the forward, dk and dv 1000.
#include <type_traits>

#include "gemm_nt.h"

#pragma clang fp contract(fast)

namespace ar {
namespace dev {

constexpr int kKeys = 64;   // keys, or queries, of a stage
constexpr int kRows = 128;  // rows of a workgroup's tile: 32 for each of four waves
constexpr float kLog2e = 1.4426950408889634f;

// One of q, k, v, o and their gradients: element d of head h of token t lies at
// t * ld + h * hs + d.
template <typename T> struct Heads {
    T *p;
    uint64_t ld, hs;
    __device__ __forceinline__ T *at(uint64_t token, uint64_t head) const { return p + token * ld + head * hs; }
};

struct AttnArgs {
    Heads<const bf16> q, k, v, dout;
    Heads<bf16> o, dq, dk, dv;
    const int32_t *starts_q, *starts_k;  // null: one sequence
    float *lse;                          // [head][token]; null: not kept
    const float *delta;                  // [head][token]
    float *part, *part_lse;              // with keys split: [split][token][head][dim], [split][token][head]
    uint32_t sequences, tokens_q, tokens_k, heads, kv_heads, group;
    uint32_t dim, dim_in;  // dim_in: a multiple of eight, up to which the inputs can be read
    uint32_t slots, splits;
    uint32_t causal, rest;  // rest: rows of no sequence are set to zero
    float scale;
};

__device__ __forceinline__ uint32_t uniform(uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); }

// Where sequence i begins, kept inside the tokens whatever the array holds.
__device__ __forceinline__ uint32_t start_of(const int32_t *starts, uint32_t i, uint32_t tokens)
{
    if (!starts) return i ? tokens : 0u;
    const int32_t s = starts[i];
    return s < 0 ? 0u : (uint32_t)s < tokens ? (uint32_t)s : tokens;
}

// A sequence's part of the tokens, and which of its tiles a slot stands for.
// Tiles are not counted on the host, which does not know the lengths: sequence i
// has the slots from floor(start_i * per / rows) + i on, which are enough for its
// tiles (of `rows` rows, `per` for each token) and do not meet the next one's.
struct Place {
    uint32_t q0, lq, k0, lk, tile;
    bool some;
};
__device__ __forceinline__ Place find_place(const AttnArgs &a, uint32_t slot, bool by_keys, uint32_t per, uint32_t rows)
{
    const uint32_t lane = threadIdx.x & 63u;
    const int32_t *starts = by_keys ? a.starts_k : a.starts_q;
    const uint32_t tokens = by_keys ? a.tokens_k : a.tokens_q;
    auto first_slot = [&](uint32_t i) { return (uint64_t)start_of(starts, i, tokens) * per / rows + i; };
    uint32_t lo = 0, hi = a.sequences;  // the last sequence whose slots begin at `slot` or before
    Place p{};
    do {
        const uint32_t step = (hi - lo + 63) / 64, i = lo + lane * step;
        const uint32_t below = (uint32_t)__popcll(__ballot(i < hi && first_slot(i) <= slot));
        if (below == 0) return p;
        lo += (below - 1) * step;
        hi = lo + step < hi ? lo + step : hi;
    } while (hi - lo > 1);
    lo = uniform(lo);
    const uint64_t before = first_slot(lo);
    const uint32_t qa = start_of(a.starts_q, lo, a.tokens_q), qb = start_of(a.starts_q, lo + 1, a.tokens_q);
    const uint32_t ka = start_of(a.starts_k, lo, a.tokens_k), kb = start_of(a.starts_k, lo + 1, a.tokens_k);
    p.q0 = uniform(qa), p.lq = uniform(qb > qa ? qb - qa : 0), p.k0 = uniform(ka), p.lk = uniform(kb > ka ? kb - ka : 0);
    if (before > slot) return p;
    p.tile = uniform(slot - (uint32_t)before);
    p.some = (uint64_t)p.tile * rows < (uint64_t)(by_keys ? p.lk : p.lq) * per;
    return p;
}

// Zeros in the rows of no sequence, by the workgroups behind the tiles'.
constexpr uint32_t kRestGroups = 128;
template <typename T> __device__ void clear_rest(const Heads<T> &x, const int32_t *starts, uint32_t sequences, uint32_t tokens,
                                                uint32_t heads, uint32_t dim, uint32_t group)
{
    const uint32_t a = start_of(starts, 0, tokens), b = start_of(starts, starts ? sequences : 1, tokens), rest = a + (tokens - b);
    if (b < a) return;
    constexpr int V = sizeof(T) == 2 ? 8 : 4;
    const float zeros[V] = {};
    const uint32_t per = (dim + V - 1) / V;
    const uint64_t each = (uint64_t)heads * per, n = rest * each;
    for (uint64_t i = (uint64_t)group * 256 + threadIdx.x; i < n; i += kRestGroups * 256) {
        const uint32_t t = (uint32_t)(i / each), c = (uint32_t)(i % each), d = c % per * V;
        T *to = x.at(t < a ? t : b + (t - a), c / per) + d;
        if (d + V <= dim) store_vec<T, V>(to, zeros);
        else store_part<T, V>(to, (int)(dim - d), zeros);
    }
}

// A stage's rows, 64 of DP elements, in LDS: read by rows and transposed.  Row r's
// 16-byte chunks lie in the order chunk ^ turn(r): sixteen rows' equal chunks are in
// sixteen groups of four banks, and so are the four chunks of four rows that a
// transposing read touches together.
template <int DP> struct Stage {
    static constexpr int CHUNKS = DP / 8, ROW = DP * 2, BYTES = kKeys * ROW, LOADS = BYTES / 4096;
    static __device__ __forceinline__ uint32_t turn(uint32_t r)
    {
        return DP == 128 ? (r & 3u) << 2 | (r >> 2 & 3u) : (r >> 1 & 1u) << 2 | (r >> 2 & 3u);
    }
    uint32_t off[LOADS];
    uint64_t next, step;  // the next stage's first row; bytes from a stage to the one behind it
    __device__ __forceinline__ void place(uint32_t wave, const void *first, uint64_t ld, uint32_t dim)
    {
        const uint32_t lane = threadIdx.x & 63u;
        next = uniform_address(first), step = kKeys * ld * 2;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const uint32_t n = (i * 4 + wave) * 64 + lane, r = n / CHUNKS, c = (n % CHUNKS) ^ turn(r);
            off[i] = c * 8 < dim ? r * (uint32_t)ld * 2 + c * 16 : kOutOfRange;
        }
    }
    // rows from `left` on are zeros
    __device__ __forceinline__ void load(uint32_t lds, uint32_t wave, uint32_t left)
    {
        const u32x4v from = tile_resource(next);
        next += step;
        if (left >= kKeys) {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) load_to_lds(lds + (i * 4 + wave) * 1024, off[i], from, 0u);
        } else {
            const uint32_t lane = threadIdx.x & 63u;
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const uint32_t r = ((i * 4 + wave) * 64 + lane) / CHUNKS;
                load_to_lds(lds + (i * 4 + wave) * 1024, r < left ? off[i] : kOutOfRange, from, 0u);
            }
        }
    }
};

// Addresses of a lane's fragments in a stage.  By rows: lane l has row l % 32 of a
// block of 32 and elements 16 c + 8 (l / 32) + 0..7.  Transposed: element l % 32 of a
// block of 32 and rows 16 c + 4 (l / 32) + 0..3 and 8 + 4 (l / 32) + 0..3.
template <int DP> struct Reads {
    uint32_t by_row[DP / 16], across[DP / 32][2];
    __device__ __forceinline__ void place(uint32_t lds)
    {
        const uint32_t lane = threadIdx.x & 63u, h = lane >> 5, r = lane & 31u;
        // The compiler would take an address apart again, for parts that several share, and
        // add them up for every read; as they are, a read's constant goes into the instruction.
#pragma unroll
        for (int c = 0; c < DP / 16; ++c) {
            by_row[c] = lds + r * Stage<DP>::ROW + ((2 * c + h) ^ Stage<DP>::turn(r)) * 16;
            asm("" : "+v"(by_row[c]));
        }
#pragma unroll
        for (int b = 0; b < DP / 32; ++b)
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const uint32_t k = 8 * s + 4 * h + (lane & 15u) / 4, c = 4 * b + 2 * (lane >> 4 & 1u) + (lane >> 1 & 1u);
                across[b][s] = lds + k * Stage<DP>::ROW + (c ^ Stage<DP>::turn(k)) * 16 + (lane & 1u) * 8;
                asm("" : "+v"(across[b][s]));
            }
    }
    typedef __attribute__((address_space(3))) const char *P;
    // block: of 32 rows; c: of 16 elements; at: bytes from the stage that `place` was told
    __device__ __forceinline__ bf16x8 rows(int block, int c, int at) const
    {
        return *(__attribute__((address_space(3))) const bf16x8 *)((P)(uintptr_t)by_row[c] + (block * 32 * Stage<DP>::ROW + at));
    }
    // block: of 32 elements; c: of 16 rows
    __device__ __forceinline__ bf16x8 columns(int block, int c, int at) const
    {
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) s16x4 *V;
        const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((V)((P)(uintptr_t)across[block][0] + (c * 16 * Stage<DP>::ROW + at)));
        const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((V)((P)(uintptr_t)across[block][1] + (c * 16 * Stage<DP>::ROW + at)));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
    }
};

// The fragment of a lane's row, elements 16 c + 8 (l / 32) + 0..7.
template <int DP> __device__ __forceinline__ void load_row(const bf16 *row, uint32_t dim, bf16x8 (&f)[DP / 16])
{
    const uint32_t h = threadIdx.x >> 5 & 1u;
#pragma unroll
    for (int c = 0; c < DP / 16; ++c) {
        const uint32_t d = c * 16 + h * 8;
        f[c] = bf16x8{};
        if (d < dim) f[c] = *(const bf16x8 *)(row + d);
    }
}

// Eight neighbouring sums of a lane, rounded: a fragment of the next product.
__device__ __forceinline__ bf16x8 rounded(const f32x16 &v, int from)
{
    bf16x8 f;
#pragma unroll
    for (int k = 0; k < 8; ++k) f[k] = (bf16)v[from + k];
    return f;
}

// A lane's value and that of lane ^ 32.
struct Halves {
    float a, b;
};
__device__ __forceinline__ Halves halves(float v)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, v);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return {__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1])};
}

// Keeps the operations that make a value before the ones written behind this: the
// compiler's barriers hold no operations that touch no memory.
template <typename T> __device__ __forceinline__ void here_now(T &v) { asm volatile("" : "+v"(v)); }

// One product, then so many reads of LDS for a later one and vector and transcendental
// operations of what is independent of it, N times over: the matrix unit takes 32 cycles
// for a product.
template <int N, int READS, int VECTOR, int TRANS> __device__ __forceinline__ void interleave()
{
    static_for<N>([](auto) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        if constexpr (READS) __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
        if constexpr (VECTOR) __builtin_amdgcn_sched_group_barrier(0x002, VECTOR, 0);
        if constexpr (TRANS) __builtin_amdgcn_sched_group_barrier(0x400, TRANS, 0);
    });
}

// A lane's row of O^T (or of a gradient), times `by`: elements 32 b + 8 q + 4 (l / 32)
// + 0..3 of row l % 32.
template <int DP, typename O> __device__ __forceinline__ void store_row(O *row, uint32_t dim, const f32x16 (&acc)[DP / 32], float by)
{
    typedef O O4 __attribute__((ext_vector_type(4)));
    typedef O4 Out __attribute__((aligned(sizeof(O))));
    const uint32_t h = threadIdx.x >> 5 & 1u;
#pragma unroll
    for (int b = 0; b < DP / 32; ++b)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint32_t d = b * 32 + q * 8 + h * 4;
            O4 v;
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = (O)(acc[b][q * 4 + k] * by);
            if (d + 4 <= dim) {
                *(Out *)(row + d) = v;
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (d + k < dim) row[d + k] = v[k];
            }
        }
}

// What the rows of a wave's tile may see.
struct Rows {
    uint32_t row, query, head;  // of the lane; rows past the last one repeat it
    uint32_t limit;             // keys that the lane's row sees
    uint32_t least, most;       // of the wave's rows
    bool real;                  // there is such a row
};
__device__ __forceinline__ Rows rows_of(const AttnArgs &a, const Place &p, uint32_t first, uint32_t kv_head)
{
    const uint32_t lane = threadIdx.x & 63u, count = p.lq * a.group;
    auto limit = [&](uint32_t query) {
        const int64_t n = a.causal ? (int64_t)query + 1 + p.lk - p.lq : (int64_t)p.lk;
        return n > 0 ? (uint32_t)n : 0u;
    };
    Rows r;
    r.row = first + (lane & 31u);
    r.real = r.row < count;
    r.row = r.real ? r.row : count - 1;
    r.query = r.row / a.group;
    r.head = kv_head * a.group + (r.row - r.query * a.group);
    r.limit = limit(r.query);
    r.least = uniform(limit((first < count ? first : count - 1) / a.group));
    r.most = uniform(limit((first + 31 < count ? first + 31 : count - 1) / a.group));
    if (first >= count) r.most = 0;  // nothing to do for this wave
    return r;
}

// Sums that are more than this far (powers of two) below the running maximum's new
// value are what makes the kept sums be scaled down: up to there P grows to 2^8,
// which costs none of its bits.
constexpr float kSlack = 8.0f;

// 128 rows, four waves of 32, 64 KiB of LDS for two stages of K and V: two workgroups to a
// compute unit, so that a SIMD has two waves (64 rows a wave, one on a SIMD: prompts 940 us
// in place of 770; 256 rows a workgroup: 769 and 775, and slower where rows are few).
template <int DP> __global__ __launch_bounds__(256, 2) void attention_kernel(const AttnArgs a)
{
    typedef Stage<DP> S;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const uint32_t wave = uniform(threadIdx.x >> 6), h = threadIdx.x >> 5 & 1u;
    const uint32_t tiles = a.slots * a.kv_heads * a.splits;
    if (blockIdx.x >= tiles) {
        clear_rest(a.o, a.starts_q, a.sequences, a.tokens_q, a.heads, a.dim, blockIdx.x - tiles);
        if (a.lse) clear_rest(Heads<float>{a.lse, 1, a.tokens_q}, a.starts_q, a.sequences, a.tokens_q, a.heads, 1, blockIdx.x - tiles);
        return;
    }
    // a key head's workgroups on one XCD where the heads come to eight; the last
    // tiles of a sequence, which see the most keys, first
    const uint32_t kv_head = blockIdx.x % a.kv_heads, rest = blockIdx.x / a.kv_heads, split = rest % a.splits;
    const Place p = find_place(a, a.slots - 1 - rest / a.splits, false, a.group, kRows);
    if (!p.some) return;
    const Rows r = rows_of(a, p, p.tile * kRows + wave * 32, kv_head);
    const bool idle = r.most == 0;
    const uint32_t last = (p.tile + 1) * kRows < p.lq * a.group ? (p.tile + 1) * kRows - 1 : p.lq * a.group - 1;
    const int64_t sees = a.causal ? (int64_t)(last / a.group) + 1 + p.lk - p.lq : (int64_t)p.lk;
    const uint32_t stages = sees > 0 ? ((uint32_t)sees + kKeys - 1) / kKeys : 0;
    const uint32_t begin = (uint32_t)((uint64_t)stages * split / a.splits), end = (uint32_t)((uint64_t)stages * (split + 1) / a.splits);

    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
    S ks, vs;
    ks.place(wave, a.k.at(p.k0 + begin * kKeys, kv_head), a.k.ld, a.dim_in);
    vs.place(wave, a.v.at(p.k0 + begin * kKeys, kv_head), a.v.ld, a.dim_in);
    Reads<DP> at;
    at.place(lds0);
    // the stages of keys in turn
    auto load_k = [&](uint32_t t, uint32_t buf) { ks.load(lds0 + buf * 2 * S::BYTES, wave, p.lk - t * kKeys); };
    auto load_v = [&](uint32_t t, uint32_t buf) { vs.load(lds0 + buf * 2 * S::BYTES + S::BYTES, wave, p.lk - t * kKeys); };
    bf16x8 q[DP / 16];
    load_row<DP>(a.q.at(p.q0 + r.query, r.head), a.dim_in, q);
    f32x16 o[DP / 32], x{}, y;
#pragma unroll
    for (int b = 0; b < DP / 32; ++b) o[b] = f32x16{};
    float top = -INFINITY, part[4] = {0.0f, 0.0f, 0.0f, 0.0f};  // top: in units of S, times c once used
    const float c = a.scale * kLog2e;

    // Blocks of 32 keys, in a pipeline: while the softmax of block n is computed, the
    // matrix unit has P V of block n - 1 and Q K^T of block n + 1.  x: P of block n - 1,
    // then S of block n + 1; y: S of block n, then P.  Half 0 and 1 of a stage: block n is
    // the stage's first or second.
    auto products_o = [&](const f32x16 &x, int V, int block) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const bf16x8 w = rounded(x, k * 8);
#pragma unroll
            for (int d = 0; d < DP / 32; ++d) o[d] = Frag<bf16>::mfma(at.columns(d, block * 2 + k, V), w, o[d]);
        }
#pragma unroll
        for (int k = 0; k < 16; ++k) part[k & 3] += x[k];
    };
    auto products_s = [&](f32x16 &x, int K, int block) {
        x = f32x16{};
#pragma unroll
        for (int d = 0; d < DP / 16; ++d) x = Frag<bf16>::mfma(at.rows(block, d, K), q[d], x);
    };
    auto step = [&](uint32_t n, f32x16 &x, f32x16 &y, auto buffer, auto half) {
        constexpr int HERE = buffer.value * 2 * S::BYTES, THERE = (1 - buffer.value) * 2 * S::BYTES;
        constexpr int V = (half.value ? HERE : THERE) + S::BYTES, K = half.value ? THERE : HERE, B = 1 - half.value;
        if (idle) return;
        if (n * 32 + 32 > r.least) {
            const int32_t left = (int32_t)(r.limit - n * 32 - 4 * h);
#pragma unroll
            for (int k = 0; k < 16; ++k) y[k] = 8 * (k / 4) + k % 4 < left ? y[k] : -INFINITY;
        }
        __builtin_amdgcn_sched_barrier(0);
        products_o(x, V, B);
        float m = y[0];
#pragma unroll
        for (int k = 1; k < 16; ++k) m = __builtin_elementwise_maximum(m, y[k]);
        const Halves both = halves(m);
        m = __builtin_elementwise_maximum(both.a, both.b);
        __builtin_amdgcn_sched_group_barrier(0x100, 8, 0);
        interleave<DP / 16, 2, 5, 0>();
        __builtin_amdgcn_sched_barrier(0);
        const bool rises = m * c > top * c + kSlack;
        if (__any(rises)) {
            // a row's bits do not depend on the others: a lane whose maximum stays goes on as it was
            const float next = rises ? m : top, to = next == -INFINITY ? 0.0f : next;
            const float by = __builtin_amdgcn_exp2f((top - to) * c);
            top = next;
#pragma unroll
            for (int k = 0; k < 4; ++k) part[k] *= by;
#pragma unroll
            for (int b = 0; b < DP / 32; ++b)
#pragma unroll
                for (int k = 0; k < 16; ++k) o[b][k] *= by;
        }
        const float base = top == -INFINITY ? 0.0f : top * c;
        __builtin_amdgcn_sched_barrier(0);
        products_s(x, K, B);
#pragma unroll
        for (int k = 0; k < 16; ++k) y[k] = __builtin_amdgcn_exp2f(y[k] * c - base);
        __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
        interleave<DP / 16, 1, 16 / (DP / 16), 16 / (DP / 16)>();
        __builtin_amdgcn_sched_barrier(0);
    };
    auto settled = [&]() {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    if (begin < end) {
        // P of no block, times zeros
        typedef float f32x4 __attribute__((ext_vector_type(4)));
#pragma unroll
        for (int i = 0; i < S::BYTES / 2 / 4096; ++i) *(f32x4 *)(lds + 3 * S::BYTES + S::BYTES / 2 + (i * 256 + threadIdx.x) * 16) = f32x4{};
        load_k(begin, 0), load_v(begin, 0);
        if (begin + 1 < end) load_k(begin + 1, 1);
        settled();
        products_s(y, 0, 0);
    }
    auto stage = [&](uint32_t t, auto buffer) {
        constexpr int B = buffer.value;
        step(2 * t, x, y, buffer, std::integral_constant<int, 0>{});
        settled();
        if (t + 2 < end) load_k(t + 2, B);
        if (t + 1 < end) load_v(t + 1, 1 - B);
        step(2 * t + 1, y, x, buffer, std::integral_constant<int, 1>{});
    };
    for (uint32_t t = begin; t < end; t += 2) {
        stage(t, std::integral_constant<int, 0>{});
        if (t + 1 < end) stage(t + 1, std::integral_constant<int, 1>{});
    }
    if (begin < end && !idle) {
        // the last block of the last stage
        if ((end - begin) & 1u) products_o(x, S::BYTES, 1);
        else products_o(x, 3 * S::BYTES, 1);
    }
    const Halves both = halves((part[0] + part[1]) + (part[2] + part[3]));
    const float sum = both.a + both.b;
    if (!r.real) return;
    const float by = sum == 0.0f ? 0.0f : 1.0f / sum;
    const float lse = sum == 0.0f ? -INFINITY : top * a.scale + __logf(sum);
    const uint64_t token = p.q0 + r.query;
    if (a.splits > 1) {
        const uint64_t at_row = ((uint64_t)split * a.tokens_q + token) * a.heads + r.head;
        store_row<DP>(a.part + at_row * a.dim, a.dim, o, by);
        if (h == 0) a.part_lse[at_row] = lse;
    } else {
        store_row<DP>(a.o.at(token, r.head), a.dim, o, by);
        if (a.lse && h == 0) a.lse[(uint64_t)r.head * a.tokens_q + token] = lse;
    }
}

// The forward pass where there are few rows, single tokens in a serving loop or a short
// prompt: bound by the bytes of K and V, and by latency where those are few.  A tile has 32
// rows, and each wave of the workgroup every fourth block of 32 keys, which it loads into a
// part of LDS of its own and waits for alone; at the end the waves' sums are joined through
// LDS.  A place in LDS is loaded again as soon as it has been read, K's while V is used, so
// one place each is enough with dim above 64, and two workgroups fit a compute unit: with two
// places each and one workgroup 504 tiles of 1200 keys took 34 us, so 26; dim 64, four places
// and one workgroup, two and two: 23, 17 us (by tiles of 128 rows 34 and 32).  32 heads over
// 8 of 128, by tiles of 128 rows and so: 1 query of 16000 keys 37 and 31 us, 32 of 160 to
// 15000 210 and 195 us.
constexpr int kFewRows = 32;
template <int DP> struct Few {
    static constexpr int BLOCK = 32 * DP * 2, DEPTH = DP == 128 ? 1 : 2;  // bytes of a block of K or V; blocks of a wave
    static constexpr int WAVE = 2 * DEPTH * BLOCK, SUMS = 4 * (DP + 2) * 32 * (int)sizeof(float), LDS = 4 * WAVE > SUMS ? 4 * WAVE : SUMS;
    static constexpr int LOADS = BLOCK / 1024;
};
template <int DP> __global__ __launch_bounds__(256, 2) void attention_few_kernel(const AttnArgs a)
{
    typedef Few<DP> F;
    typedef Stage<DP> S;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const uint32_t wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63u, h = lane >> 5;
    const uint32_t tiles = a.slots * a.kv_heads * a.splits;
    if (blockIdx.x >= tiles) {
        clear_rest(a.o, a.starts_q, a.sequences, a.tokens_q, a.heads, a.dim, blockIdx.x - tiles);
        if (a.lse) clear_rest(Heads<float>{a.lse, 1, a.tokens_q}, a.starts_q, a.sequences, a.tokens_q, a.heads, 1, blockIdx.x - tiles);
        return;
    }
    const uint32_t kv_head = blockIdx.x % a.kv_heads, rest = blockIdx.x / a.kv_heads, split = rest % a.splits;
    const Place p = find_place(a, a.slots - 1 - rest / a.splits, false, a.group, kFewRows);
    if (!p.some) return;
    const Rows r = rows_of(a, p, p.tile * kFewRows, kv_head);
    const uint32_t blocks = (r.most + 31) / 32;
    const uint32_t begin = (uint32_t)((uint64_t)blocks * split / a.splits), end = (uint32_t)((uint64_t)blocks * (split + 1) / a.splits);

    // this wave's loads: 1 KiB each, of K and then of V
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds + wave * F::WAVE;
    uint32_t off_k[F::LOADS], off_v[F::LOADS];
#pragma unroll
    for (int i = 0; i < F::LOADS; ++i) {
        const uint32_t n = i * 64 + lane, row = n / S::CHUNKS, c = (n % S::CHUNKS) ^ S::turn(row);
        off_k[i] = c * 8 < a.dim_in ? row * (uint32_t)a.k.ld * 2 + c * 16 : kOutOfRange;
        off_v[i] = c * 8 < a.dim_in ? row * (uint32_t)a.v.ld * 2 + c * 16 : kOutOfRange;
    }
    uint64_t next_k = uniform_address(a.k.at(p.k0 + (begin + wave) * 32, kv_head)), next_v = uniform_address(a.v.at(p.k0 + (begin + wave) * 32, kv_head));
    auto load = [&](uint32_t n, uint32_t to, uint64_t &next, uint64_t ld, const uint32_t *off) {
        const uint32_t left = p.lk - n * 32;
        const u32x4v from = tile_resource(next);
        next += 4 * 32 * ld * 2;
#pragma unroll
        for (int i = 0; i < F::LOADS; ++i) load_to_lds(lds0 + to + i * 1024, (i * 64 + lane) / S::CHUNKS < left ? off[i] : kOutOfRange, from, 0u);
    };
    auto load_k = [&](uint32_t n, uint32_t slot) { load(n, slot * 2 * F::BLOCK, next_k, a.k.ld, off_k); };
    auto load_v = [&](uint32_t n, uint32_t slot) { load(n, slot * 2 * F::BLOCK + F::BLOCK, next_v, a.v.ld, off_v); };
    Reads<DP> at;
    at.place(lds0);
    bf16x8 q[DP / 16];
    load_row<DP>(a.q.at(p.q0 + r.query, r.head), a.dim_in, q);
    f32x16 o[DP / 32];
#pragma unroll
    for (int b = 0; b < DP / 32; ++b) o[b] = f32x16{};
    const float c = a.scale * kLog2e;
    float top = -INFINITY, part[4] = {0.0f, 0.0f, 0.0f, 0.0f};

    // Of the loads that are on their way, all but the newest DEPTH - 1 of K and of V and one
    // more are there; where so many were not begun, all are.
    auto landed = [&](bool all_begun) {
        if (all_begun) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(F::LOADS * (2 * F::DEPTH - 1)) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    };
    auto block = [&](uint32_t n, auto slot) {
        constexpr int K = slot.value * 2 * F::BLOCK, V = K + F::BLOCK;
        landed(n + 4 * (F::DEPTH - 1) < end);
        f32x16 s{};
#pragma unroll
        for (int d = 0; d < DP / 16; ++d) s = Frag<bf16>::mfma(at.rows(0, d, K), q[d], s);
        const uint32_t ahead = n + 4 * F::DEPTH;
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // K's reads are done
        if (ahead < end) load_k(ahead, slot.value);
        if (n * 32 + 32 > r.least) {
            const int32_t left = (int32_t)(r.limit - n * 32 - 4 * h);
#pragma unroll
            for (int k = 0; k < 16; ++k) s[k] = 8 * (k / 4) + k % 4 < left ? s[k] : -INFINITY;
        }
        float m = s[0];
#pragma unroll
        for (int k = 1; k < 16; ++k) m = __builtin_elementwise_maximum(m, s[k]);
        const Halves both = halves(m);
        m = __builtin_elementwise_maximum(both.a, both.b);
        const bool rises = m * c > top * c + kSlack;
        if (__any(rises)) {
            const float next = rises ? m : top, to = next == -INFINITY ? 0.0f : next;
            const float by = __builtin_amdgcn_exp2f((top - to) * c);
            top = next;
#pragma unroll
            for (int k = 0; k < 4; ++k) part[k] *= by;
#pragma unroll
            for (int b = 0; b < DP / 32; ++b)
#pragma unroll
                for (int k = 0; k < 16; ++k) o[b][k] *= by;
        }
        const float base = top == -INFINITY ? 0.0f : top * c;
#pragma unroll
        for (int k = 0; k < 16; ++k) s[k] = __builtin_amdgcn_exp2f(s[k] * c - base), part[k & 3] += s[k];
        landed(ahead < end);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const bf16x8 w = rounded(s, k * 8);
#pragma unroll
            for (int d = 0; d < DP / 32; ++d) o[d] = Frag<bf16>::mfma(at.columns(d, k, V), w, o[d]);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // V's are
        if (ahead < end) load_v(ahead, slot.value);
    };
    static_for<F::DEPTH>([&](auto slot) {
        const uint32_t n = begin + wave + 4 * slot.value;
        if (n < end) load_k(n, slot.value), load_v(n, slot.value);
    });
    for (uint32_t n = begin + wave; n < end; n += 4 * F::DEPTH)
        static_for<F::DEPTH>([&](auto slot) {
            if (n + 4 * slot.value < end) block(n + 4 * slot.value, slot);
        });

    // the waves' sums: element d of row r at d * 32 + r, then the maxima and the sums
    __syncthreads();
    float *mine = (float *)lds + wave * (DP + 2) * 32;
    const uint32_t row = lane & 31u;
#pragma unroll
    for (int b = 0; b < DP / 32; ++b)
#pragma unroll
        for (int k = 0; k < 16; ++k) mine[(b * 32 + 8 * (k / 4) + 4 * h + k % 4) * 32 + row] = o[b][k];
    const Halves sums = halves((part[0] + part[1]) + (part[2] + part[3]));
    if (h == 0) mine[DP * 32 + row] = top, mine[(DP + 1) * 32 + row] = sums.a + sums.b;
    __syncthreads();
    // eight threads a row, each with an eighth of its elements
    constexpr int EACH = DP / 8;
    const uint32_t to_row = threadIdx.x & 31u, d0 = threadIdx.x / 32 * EACH, index = p.tile * kFewRows + to_row;
    if (index >= p.lq * a.group) return;
    const float *all = (const float *)lds + to_row;
    float most = -INFINITY, by[4], sum = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) most = fmaxf(most, all[(w * (DP + 2) + DP) * 32]);
    const float base = most == -INFINITY ? 0.0f : most;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        by[w] = __builtin_amdgcn_exp2f((all[(w * (DP + 2) + DP) * 32] - base) * c);
        sum += by[w] * all[(w * (DP + 2) + DP + 1) * 32];
    }
    const float inverse = sum == 0.0f ? 0.0f : 1.0f / sum;
    float v[EACH];
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
        v[k] = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; ++w) v[k] += by[w] * all[(w * (DP + 2) + d0 + k) * 32];
        v[k] *= inverse;
    }
    const uint32_t query = index / a.group, head = kv_head * a.group + (index - query * a.group);
    const uint64_t token = p.q0 + query;
    const float lse = sum == 0.0f ? -INFINITY : base * a.scale + __logf(sum);
    const int have = (int)a.dim - (int)d0;
    if (a.splits > 1) {
        const uint64_t at_row = ((uint64_t)split * a.tokens_q + token) * a.heads + head;
        float *out = a.part + at_row * a.dim + d0;
        if (have >= EACH) store_vec<float, EACH>(out, v);
        else store_part<float, EACH>(out, have, v);
        if (d0 == 0) a.part_lse[at_row] = lse;
    } else {
        bf16 *out = a.o.at(token, head) + d0;
        if (have >= EACH) store_vec<bf16, EACH>(out, v);
        else store_part<bf16, EACH>(out, have, v);
        if (a.lse && d0 == 0) a.lse[(uint64_t)head * a.tokens_q + token] = lse;
    }
}

// Joins the runs of keys of a split call: one wave for each row, lane s with the
// statistics of run s, and the first sums on their way before those are there, so that no
// load waits for another.
constexpr uint32_t kMaxRuns = 64;
__global__ __launch_bounds__(256) void attention_join_kernel(const AttnArgs a)
{
    const uint32_t lane = threadIdx.x & 63u, d = lane * 2;
    const uint64_t rows = (uint64_t)a.tokens_q * a.heads;
    const uint32_t from = start_of(a.starts_q, 0, a.tokens_q), until = start_of(a.starts_q, a.starts_q ? a.sequences : 1, a.tokens_q);
    for (uint64_t i = (uint64_t)blockIdx.x * 4 + uniform(threadIdx.x >> 6); i < rows; i += (uint64_t)gridDim.x * 4) {
        const uint32_t token = (uint32_t)(i / a.heads), head = (uint32_t)(i % a.heads);
        if (token < from || token >= until) continue;
        const float *o = a.part + i * a.dim + d;
        constexpr int FIRST = 16;
        float early[FIRST][2];
        const float lse = lane < a.splits ? a.part_lse[lane * rows + i] : -INFINITY;
#pragma unroll
        for (int s = 0; s < FIRST; ++s) {
            const float *from_run = o + (s < (int)a.splits ? s * rows * a.dim : 0);
            early[s][0] = d < a.dim ? from_run[0] : 0.0f;
            early[s][1] = d + 1 < a.dim ? from_run[1] : 0.0f;
        }
        float top = lse;
#pragma unroll
        for (int m = 32; m; m >>= 1) top = __builtin_elementwise_maximum(top, __shfl_xor(top, m));  // NaN stays
        const float base = top == -INFINITY ? 0.0f : top, w = __expf(lse - base), sum = wave_sum(w);
        float v[2] = {0.0f, 0.0f};
        auto weight = [&](uint32_t s) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, w), (int)s)); };
#pragma unroll
        for (int s = 0; s < FIRST; ++s) {
            if (s >= (int)a.splits) break;
            const float by = weight(s);
            v[0] += by * early[s][0], v[1] += by * early[s][1];
        }
#pragma unroll 8
        for (uint32_t s = FIRST; s < a.splits; ++s) {
            const float by = weight(s);
            const float *from_run = o + s * rows * a.dim;
            if (d < a.dim) v[0] += by * from_run[0];
            if (d + 1 < a.dim) v[1] += by * from_run[1];
        }
        const float by = sum == 0.0f ? 0.0f : 1.0f / sum;
        bf16 *to = a.o.at(token, head) + d;
        if (d < a.dim) to[0] = (bf16)(v[0] * by);
        if (d + 1 < a.dim) to[1] = (bf16)(v[1] * by);
        if (a.lse && lane == 0) a.lse[(uint64_t)head * a.tokens_q + token] = sum == 0.0f ? -INFINITY : base + __logf(sum);
    }
}

// ---- backward -----------------------------------------------------------------

// delta = the sum over a row of dout * o: sixteen lanes a row, a head's rows in turn.
__global__ __launch_bounds__(256) void attention_delta_kernel(const Heads<const bf16> dout, const Heads<const bf16> o, float *delta,
                                                              uint64_t rows, uint32_t tokens, uint32_t dim)
{
    const uint32_t d = (threadIdx.x & 15u) * 8;
    for (uint64_t i0 = (uint64_t)blockIdx.x * 16; i0 < rows; i0 += (uint64_t)gridDim.x * 16) {
        const uint64_t i = i0 + (threadIdx.x >> 4);
        float sum = 0.0f;
        if (i < rows && d < dim) {
            const bf16 *a = dout.at(i % tokens, i / tokens) + d, *b = o.at(i % tokens, i / tokens) + d;
            float x[8], y[8];
            if (d + 8 <= dim) load_vec<bf16, 8>(a, x), load_vec<bf16, 8>(b, y);
            else load_part<bf16, 8>(a, (int)(dim - d), x), load_part<bf16, 8>(b, (int)(dim - d), y);
#pragma unroll
            for (int k = 0; k < 8; ++k) sum += x[k] * y[k];
        }
#pragma unroll
        for (int m = 8; m; m >>= 1) sum += __shfl_xor(sum, m);
        if (i < rows && d == 0) delta[i] = sum;
    }
}

// dQ of a tile of rows, over the keys they see: dS^T = P^T * (V dO^T - delta) and
// dQ^T += K^T dS^T, S^T as in the forward pass.  2 x 4096, 32 heads over 8 of 128: 390 us,
// 1050 TFLOP/s; matrix units busy 59 %, at 1.9 GHz.
template <int DP> __device__ __forceinline__ void backward_rows(const AttnArgs &a, uint32_t group, char *lds)
{
    typedef Stage<DP> S;
    const uint32_t wave = uniform(threadIdx.x >> 6);
    const uint32_t tiles = a.slots * a.kv_heads * a.splits;
    if (group >= tiles) {
        clear_rest(a.dq, a.starts_q, a.sequences, a.tokens_q, a.heads, a.dim, group - tiles);
        return;
    }
    const uint32_t kv_head = group % a.kv_heads, rest = group / a.kv_heads, split = rest % a.splits;
    const Place p = find_place(a, a.slots - 1 - rest / a.splits, false, a.group, kRows);
    if (!p.some) return;
    const Rows r = rows_of(a, p, p.tile * kRows + wave * 32, kv_head);
    const uint32_t last = (p.tile + 1) * kRows < p.lq * a.group ? (p.tile + 1) * kRows - 1 : p.lq * a.group - 1;
    const int64_t sees = a.causal ? (int64_t)(last / a.group) + 1 + p.lk - p.lq : (int64_t)p.lk;
    const uint32_t stages = sees > 0 ? ((uint32_t)sees + kKeys - 1) / kKeys : 0;
    const uint32_t begin = (uint32_t)((uint64_t)stages * split / a.splits), end = (uint32_t)((uint64_t)stages * (split + 1) / a.splits);

    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
    S ks, vs;
    ks.place(wave, a.k.at(p.k0 + begin * kKeys, kv_head), a.k.ld, a.dim_in);
    vs.place(wave, a.v.at(p.k0 + begin * kKeys, kv_head), a.v.ld, a.dim_in);
    Reads<DP> at;
    at.place(lds0);
    auto load = [&](uint32_t t, uint32_t buf) {
        ks.load(lds0 + buf * 2 * S::BYTES, wave, p.lk - t * kKeys);
        vs.load(lds0 + buf * 2 * S::BYTES + S::BYTES, wave, p.lk - t * kKeys);
    };
    bf16x8 q[DP / 16], g[DP / 16];
    load_row<DP>(a.q.at(p.q0 + r.query, r.head), a.dim_in, q);
    load_row<DP>(a.dout.at(p.q0 + r.query, r.head), a.dim_in, g);
    const uint64_t token = p.q0 + r.query;
    const uint64_t stat = (uint64_t)r.head * a.tokens_q + token;
    const float lse = a.lse[stat] * kLog2e, delta = a.delta[stat], c = a.scale * kLog2e;
    f32x16 dq[DP / 32];
#pragma unroll
    for (int b = 0; b < DP / 32; ++b) dq[b] = f32x16{};
    const uint32_t h = threadIdx.x >> 5 & 1u;

    auto stage = [&](uint32_t t, auto buffer) {
        constexpr int K = buffer.value * 2 * S::BYTES, V = K + S::BYTES;
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (t + 1 < end) load(t + 1, 1 - buffer.value);
        if (t * kKeys >= r.most) return;
        const bool masked = t * kKeys + kKeys > r.least;
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            f32x16 s{}, dp{};
#pragma unroll
            for (int d = 0; d < DP / 16; ++d) s = Frag<bf16>::mfma(at.rows(b, d, K), q[d], s);
#pragma unroll
            for (int d = 0; d < DP / 16; ++d) dp = Frag<bf16>::mfma(at.rows(b, d, V), g[d], dp);
#pragma unroll
            for (int k = 0; k < 16; ++k) s[k] = __builtin_amdgcn_exp2f(s[k] * c - lse) * (dp[k] - delta);
            if (masked) {
                const uint32_t from = t * kKeys + b * 32 + 4 * h;
#pragma unroll
                for (int k = 0; k < 16; ++k)
                    if (from + 8 * (k / 4) + k % 4 >= r.limit) s[k] = 0.0f;
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const bf16x8 w = rounded(s, k * 8);
#pragma unroll
                for (int d = 0; d < DP / 32; ++d) dq[d] = Frag<bf16>::mfma(at.columns(d, b * 2 + k, K), w, dq[d]);
            }
        }
    };
    if (begin < end) load(begin, 0);
    for (uint32_t t = begin; t < end; t += 2) {
        stage(t, std::integral_constant<int, 0>{});
        if (t + 1 < end) stage(t + 1, std::integral_constant<int, 1>{});
    }
    if (!r.real) return;
    if (a.splits > 1)
        store_row<DP>(a.part + (((uint64_t)split * a.tokens_q + token) * a.heads + r.head) * a.dim, a.dim, dq, a.scale);
    else
        store_row<DP>(a.dq.at(token, r.head), a.dim, dq, a.scale);
}

// dK and dV of 128 keys of a key head, 32 for each wave, over the queries that see
// them, of every head of the group in turn: a lane holds one key.  dV^T += dO^T P and
// dK^T += Q^T dS with P = e^(Q K^T - lse), dS = P * (dO V^T - delta).  The sums and the
// fragments of K and V, which stay in registers, are 192 of them for 128 elements, so a
// SIMD has one wave, and what the wave does beside products is laid between them by hand.
// 2 x 4096, 32 heads over 8 of 128: 550 us, 1000 TFLOP/s; matrix units busy 50 %, LDS 58 %.
template <int DP> __device__ __forceinline__ void backward_keys(const AttnArgs &a, uint32_t group, char *lds)
{
    typedef Stage<DP> S;
    const uint32_t wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63u, h = lane >> 5;
    const uint32_t tiles = a.slots * a.kv_heads * a.splits;
    if (group >= tiles) {
        clear_rest(a.dk, a.starts_k, a.sequences, a.tokens_k, a.kv_heads, a.dim, group - tiles);
        clear_rest(a.dv, a.starts_k, a.sequences, a.tokens_k, a.kv_heads, a.dim, group - tiles);
        return;
    }
    const uint32_t kv_head = group % a.kv_heads, rest = group / a.kv_heads, split = rest % a.splits;
    // the first tiles, which the most queries see, first
    const Place p = find_place(a, rest / a.splits, true, 1, kRows);
    if (!p.some) return;
    const uint32_t key0 = p.tile * kRows, mine = key0 + wave * 32 + (lane & 31u);
    // query i sees key j where i >= j + lq - lk
    const int32_t shift = a.causal ? (int32_t)p.lq - (int32_t)p.lk : INT32_MIN / 2;
    const int32_t need = (int32_t)mine + shift, wave_needs = (int32_t)(key0 + wave * 32 + 31) + shift;
    const int32_t wave_from = (int32_t)(key0 + wave * 32) + shift;
    const uint32_t first = (int32_t)key0 + shift > 0 ? (uint32_t)((int32_t)key0 + shift) / kKeys * kKeys : 0;
    const uint32_t per = first < p.lq ? (p.lq - first + kKeys - 1) / kKeys : 0;  // stages of a head
    const uint64_t all = (uint64_t)per * a.group;
    const uint32_t begin = (uint32_t)(all * split / a.splits), end = (uint32_t)(all * (split + 1) / a.splits);

    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
    float *stats = (float *)(lds + 4 * S::BYTES);  // of a buffer's queries: lse, -delta
    S qs, gs;
    Reads<DP> at;
    at.place(lds0);
    uint32_t next_head = per ? begin / per : 0, next_query = per ? first + begin % per * kKeys : 0;  // of the next load
    // the statistics of a stage's queries: one value for each of the first threads
    const bool is_delta = threadIdx.x >= kKeys;
    const uint32_t mine_of = threadIdx.x & (kKeys - 1);
    const float *stat = nullptr;
    auto enter = [&]() {
        const uint64_t token = p.q0 + next_query;
        const uint32_t head = kv_head * a.group + next_head;
        qs.place(wave, a.q.at(token, head), a.q.ld, a.dim_in), gs.place(wave, a.dout.at(token, head), a.dout.ld, a.dim_in);
        stat = (is_delta ? a.delta : a.lse) + (uint64_t)head * a.tokens_q + token + mine_of;
    };
    float ahead = 0.0f;
    auto load = [&](uint32_t buf) {
        const uint32_t left = p.lq - next_query;
        // what a row without keys kept is minus infinity; its P is 0, as it is behind the last row
        if (threadIdx.x < 2 * kKeys) {
            ahead = is_delta ? 0.0f : -INFINITY;
            if (mine_of < left) ahead = *stat;
        }
        qs.load(lds0 + buf * 2 * S::BYTES, wave, left);
        gs.load(lds0 + buf * 2 * S::BYTES + S::BYTES, wave, left);
        stat += kKeys, next_query += kKeys;
        if (next_query >= p.lq) {
            next_query = first, ++next_head;
            if (next_head < a.group) enter();
        }
    };
    auto keep = [&](uint32_t buf) {
        const float kept = is_delta ? -ahead : ahead == -INFINITY ? INFINITY : ahead * kLog2e;
        if (threadIdx.x < 2 * kKeys) stats[buf * 2 * kKeys + threadIdx.x] = kept;
    };
    bf16x8 kf[DP / 16], vf[DP / 16];
    const uint32_t key = mine < p.lk ? mine : p.lk - 1;
    load_row<DP>(a.k.at(p.k0 + key, kv_head), a.dim_in, kf);
    load_row<DP>(a.v.at(p.k0 + key, kv_head), a.dim_in, vf);
    f32x16 dk[DP / 32], dv[DP / 32];
#pragma unroll
    for (int b = 0; b < DP / 32; ++b) dk[b] = f32x16{}, dv[b] = f32x16{};
    const float c = a.scale * kLog2e;
    uint32_t query = next_query;  // of this stage
    if (begin < end) enter();

    auto stage = [&](uint32_t t, auto buffer) {
        constexpr int Q = buffer.value * 2 * S::BYTES, G = Q + S::BYTES;
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        const int32_t here = (int32_t)query;
        query += kKeys;
        if (query >= p.lq) query = first;
        const bool more = t + 1 < end;
        if (more) load(1 - buffer.value);
        if (here + kKeys > wave_from) {
            const float *st = stats + buffer.value * 2 * kKeys;
            // Each block of 32 queries in four parts, whose products have the matrix unit while
            // the part's vector operations go on: S; dO V^T - delta, and P; dV and dS; dK.  A
            // part's fragments are read in the one before: it waits once, and not before each
            // product.  (A wave that has a SIMD to itself issues an instruction in about 7
            // cycles, waits among them, and a product takes 32.)
            constexpr int N = DP / 16;  // products of a part
            typedef float f32x4 __attribute__((ext_vector_type(4)));
            bf16x8 f[N], g[N];
            f32x4 lse[4], delta[4];
            auto read_rows = [&](bf16x8 (&to)[N], int b, int at_stage) {
#pragma unroll
                for (int d = 0; d < N; ++d) to[d] = at.rows(b, d, at_stage);
            };
            auto columns = [&](int b, int n, int at_stage) { return at.columns(n % (DP / 32), b * 2 + n / (DP / 32), at_stage); };
            auto read_stats = [&](int b) {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    lse[k] = *(const f32x4 *)(st + b * 32 + 8 * k + 4 * h);
                    delta[k] = *(const f32x4 *)(st + kKeys + b * 32 + 8 * k + 4 * h);
                }
            };
            auto part = []() {
                __builtin_amdgcn_sched_barrier(0);
                __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0) alone
                __builtin_amdgcn_sched_barrier(0);
            };
            read_rows(f, 0, Q);
            read_stats(0);
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                f32x16 s{}, dp;
                part();
                read_rows(g, b, G);
#pragma unroll
                for (int d = 0; d < N; ++d) s = Frag<bf16>::mfma(f[d], kf[d], s);
                interleave<N, 1, 0, 0>();
                here_now(s);
                __builtin_amdgcn_sched_barrier(0);
                if (here + b * 32 < wave_needs) {
                    const int32_t hidden = need - (here + b * 32 + 4 * (int32_t)h);
#pragma unroll
                    for (int k = 0; k < 16; ++k) s[k] = 8 * (k / 4) + k % 4 >= hidden ? s[k] : -INFINITY;
                }
                part();
                here_now(s);
#pragma unroll
                for (int k = 0; k < 16; ++k) dp[k] = delta[k / 4][k % 4];
#pragma unroll
                for (int d = 0; d < N; ++d) {
                    dp = Frag<bf16>::mfma(g[d], vf[d], dp);
                    here_now(dp);
                    f[d] = columns(b, d, G);
#pragma unroll
                    for (int k = 0; k < 16 / N; ++k) {
                        const int n = d * (16 / N) + k;
                        s[n] = __builtin_amdgcn_exp2f(s[n] * c - lse[n / 4][n % 4]);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                const bf16x8 w[2] = {rounded(s, 0), rounded(s, 8)};
                part();
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    dv[n % (DP / 32)] = Frag<bf16>::mfma(f[n], w[n / (DP / 32)], dv[n % (DP / 32)]);
                    here_now(dv[n % (DP / 32)]);
                    g[n] = columns(b, n, Q);
#pragma unroll
                    for (int k = n * (16 / N); k < (n + 1) * (16 / N); ++k) dp[k] *= s[k];
                    __builtin_amdgcn_sched_barrier(0);
                }
                const bf16x8 u[2] = {rounded(dp, 0), rounded(dp, 8)};
                part();
                if (b == 0) read_rows(f, 1, Q), read_stats(1);
#pragma unroll
                for (int n = 0; n < N; ++n) dk[n % (DP / 32)] = Frag<bf16>::mfma(g[n], u[n / (DP / 32)], dk[n % (DP / 32)]);
                interleave<N, 2, 0, 0>();
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        if (more) keep(1 - buffer.value);
    };
    if (begin < end) load(0), keep(0);
    for (uint32_t t = begin; t < end; t += 2) {
        stage(t, std::integral_constant<int, 0>{});
        if (t + 1 < end) stage(t + 1, std::integral_constant<int, 1>{});
    }
    if (mine >= p.lk) return;
    if (a.splits > 1) {
        const uint64_t all_rows = (uint64_t)a.tokens_k * a.kv_heads, row = (uint64_t)(p.k0 + mine) * a.kv_heads + kv_head;
        store_row<DP>(a.part + (split * all_rows + row) * a.dim, a.dim, dk, a.scale);
        store_row<DP>(a.part + ((a.splits + split) * all_rows + row) * a.dim, a.dim, dv, 1.0f);
    } else {
        store_row<DP>(a.dk.at(p.k0 + mine, kv_head), a.dim, dk, a.scale);
        store_row<DP>(a.dv.at(p.k0 + mine, kv_head), a.dim, dv, 1.0f);
    }
}

template <int DP> __global__ __launch_bounds__(256, 2) void attention_dq_kernel(const AttnArgs a)
{
    extern __shared__ __attribute__((aligned(16))) char lds[];
    backward_rows<DP>(a, blockIdx.x, lds);
}
template <int DP> __global__ __launch_bounds__(256, 1) void attention_dkv_kernel(const AttnArgs a)
{
    extern __shared__ __attribute__((aligned(16))) char lds[];
    backward_keys<DP>(a, blockIdx.x, lds);
}
// Both where neither fills the device by itself: the first `groups` workgroups have the
// keys' tiles, which take longer.
template <int DP> __global__ __launch_bounds__(256, 1) void attention_backward_kernel(const AttnArgs keys, const AttnArgs rows, uint32_t groups)
{
    extern __shared__ __attribute__((aligned(16))) char lds[];
    if (blockIdx.x < groups) backward_keys<DP>(keys, blockIdx.x, lds);
    else backward_rows<DP>(rows, blockIdx.x - groups, lds);
}

// Adds the runs of split gradients, in their order: [split][token][head][dim].
struct Runs {
    Heads<bf16> to;
    const float *part;
    const int32_t *starts;
    uint32_t tokens, heads, splits;
};
struct RunsList {
    Runs r[3];
    uint32_t n, sequences, dim;
};
__global__ __launch_bounds__(256) void attention_sum_kernel(const RunsList list)
{
    const Runs o = list.r[blockIdx.y];
    const uint32_t from = start_of(o.starts, 0, o.tokens), until = start_of(o.starts, o.starts ? list.sequences : 1, o.tokens);
    const uint32_t dim = list.dim, per = (dim + 3) / 4;
    const uint64_t rows = (uint64_t)o.tokens * o.heads, n = rows * dim;
    for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < rows * per; i += (uint64_t)gridDim.x * 256) {
        const uint64_t row = i / per;
        const uint32_t token = (uint32_t)(row / o.heads), d = (uint32_t)(i % per) * 4;
        if (token < from || token >= until) continue;
        bf16 *to = o.to.at(token, row % o.heads) + d;
        const float *at = o.part + row * dim + d;
        float v[4] = {0.0f, 0.0f, 0.0f, 0.0f}, w[4];
        if (d + 4 <= dim) {
#pragma unroll 8
            for (uint32_t s = 0; s < o.splits; ++s) {
                load_vec<float, 4>(at + s * n, w);
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] += w[k];
            }
            store_vec<bf16, 4>(to, v);
        } else {
            for (uint32_t k = 0; k < dim - d; ++k) {
                for (uint32_t s = 0; s < o.splits; ++s) v[0] += at[s * n + k];
                to[k] = (bf16)v[0], v[0] = 0.0f;
            }
        }
    }
}

// Copies rows that the kernels cannot read where they lie, with zeros up to a
// multiple of eight elements.
struct HeadsCopy {
    Heads<const bf16> from;
    bf16 *to;
    uint64_t rows;
    uint32_t heads;
};
struct HeadsCopies {
    HeadsCopy c[4];
    uint32_t n, dim;
};
__global__ __launch_bounds__(256) void attention_pack_kernel(const HeadsCopies list)
{
    const HeadsCopy c = list.c[blockIdx.y];
    const uint32_t per = (list.dim + 7) / 8;
    const uint64_t n = c.rows * per;
    for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (uint64_t)gridDim.x * 256) {
        const uint64_t row = i / per;
        const uint32_t d = (uint32_t)(i % per) * 8;
        const bf16 *from = c.from.at(row / c.heads, row % c.heads) + d;
        float v[8];
        if (d + 8 <= list.dim) load_vec<bf16, 8>(from, v);
        else load_part<bf16, 8>(from, (int)(list.dim - d), v);
        store_vec<bf16, 8>(c.to + row * per * 8 + d, v);
    }
}

}  // namespace dev

namespace {

using namespace dev;

// One of the tensors of a call, as the checks see it: a matrix of the tokens' rows
// where a token's heads lie within the stride between tokens, else one of the heads'.
struct Tensor {
    const void *p;
    size_t tokens, heads, dim, ld, hs;
    bool by_token() const { return heads == 1 || ld >= (heads - 1) * hs + dim; }
    Mat mat() const
    {
        if (!tokens || !heads) return Mat{p, 0, 0, 0, 2};
        return by_token() ? Mat{p, tokens, (heads - 1) * hs + dim, ld, 2} : Mat{p, heads, (tokens - 1) * ld + dim, hs, 2};
    }
    // elements of a tensor do not overlap, and are counted in 64 bits
    bool ok() const
    {
        if ((uintptr_t)p % 2 != 0) return false;
        if (!tokens || !heads) return true;
        if (!p || ld < dim || hs < dim || ld > kOpsMaxSize / tokens || hs > kOpsMaxSize / heads) return false;
        return by_token() || tokens == 1 || hs >= (tokens - 1) * ld + dim;
    }
    bool direct() const
    {
        return (uintptr_t)p % 16 == 0 && ld % 8 == 0 && hs % 8 == 0 && dim % 8 == 0 && gemm_reaches(ld * 2, dim * 2);
    }
    size_t copy_bytes() const { return round_up(tokens * heads * round_up(dim, 8) * 2, 256); }
};
template <typename T> Heads<T> heads_of(const Tensor &t) { return {(T *)t.p, t.ld, t.hs}; }

// Whether two tensors may share an element.  As matrices of rows, and where those meet and
// the strides are the same, head by head: parts of one tensor whose heads take turns, as q,
// k and v of (tokens, heads, 3, dim) do, share none.
bool meet(const Tensor &a, const Tensor &b)
{
    if (!meet(a.mat(), b.mat())) return false;
    if (a.ld != b.ld || a.hs != b.hs || a.heads != b.heads) return true;
    auto by_head = [](const Tensor &t) { return Batch{Mat{t.p, t.tokens, t.dim, t.ld, 2}, t.heads, t.hs}; };
    return meet(by_head(a), by_head(b));
}

// `heads` 0: a stride that is not given
Tensor tensor(const void *p, size_t tokens, size_t heads, size_t dim, size_t ld, size_t hs)
{
    hs = hs ? hs : dim;
    return {p, tokens, heads, dim, ld ? ld : heads * hs, hs};
}

constexpr size_t kMostRows = (size_t)1 << 30, kMostSequences = (size_t)1 << 22;  // times the heads

int check_attention(const ar_attention_desc *d)
{
    if (!d) return AR_ERR_ARG;
    if (d->dtype != AR_BFLOAT16) return AR_ERR_UNSUPPORTED;
    if (d->flags & ~(AR_ATTN_CAUSAL | AR_ATTN_CLEAR)) return AR_ERR_ARG;
    if (!(d->scale >= 0x1p-100f && d->scale <= 0x1p100f)) return AR_ERR_ARG;  // with log2(e) in it still a normal number
    if (d->heads < 1 || d->kv_heads < 1 || d->heads > (1u << 16) || d->heads % d->kv_heads || d->dim < 1) return AR_ERR_ARG;
    if (d->dim > 128) return AR_ERR_UNSUPPORTED;
    // rows are counted in 32 bits on the device, and so are a launch's threads, 256 for a tile
    if (d->sequences > kMostSequences / d->heads || d->tokens_q > kMostRows / d->heads || d->tokens_k > kMostRows / d->kv_heads) return AR_ERR_ARG;
    const size_t strides[] = {d->ld_q, d->hs_q, d->ld_k, d->hs_k, d->ld_v, d->hs_v, d->ld_o, d->hs_o, d->ld_dout, d->hs_dout,
                              d->ld_dq, d->hs_dq, d->ld_dk, d->hs_dk, d->ld_dv, d->hs_dv};
    for (size_t s : strides)
        if (s > kOpsMaxSize) return AR_ERR_ARG;
    return AR_OK;
}

struct AttnTensors {
    Tensor q, k, v, o;
};
AttnTensors attn_tensors(const ar_attention_desc &d, const void *q, const void *k, const void *v, const void *o)
{
    return {tensor(q, d.tokens_q, d.heads, d.dim, d.ld_q, d.hs_q), tensor(k, d.tokens_k, d.kv_heads, d.dim, d.ld_k, d.hs_k),
            tensor(v, d.tokens_k, d.kv_heads, d.dim, d.ld_v, d.hs_v), tensor(o, d.tokens_q, d.heads, d.dim, d.ld_o, d.hs_o)};
}

// Tiles that the grid has room for: of queries' rows, and of keys.
size_t row_slots(const ar_attention_desc &d, size_t rows = kRows) { return d.tokens_q * (d.heads / d.kv_heads) / rows + d.sequences; }
size_t key_slots(const ar_attention_desc &d) { return d.tokens_k / kRows + d.sequences; }

// How many runs the stages of each tile are split into: what makes the time of the
// longest tile, whose stages follow one another, and of the join least.  `stages`: of a
// tile, in the mean, half as many again where there are several sequences, some of them
// longer; us: of a stage, alone; bytes: of a run's sums; work: the time of all tiles with
// the device full.  A join takes 5 us, 0.2 for each run and the sums' way to memory and back
// at 3.4 TB/s.  Tiles of one length (one sequence,
// most of its keys seen by every query) come in rounds of `room` workgroups.  No more than
// `most` times that in all: from there on the device is full and the sums are for nothing.
// By sweeps of 1 to 64 runs over twenty sizes, each in one piece, with the best, as
// chosen: forward, 32 heads over 8 of 128, 1 query of 16000 keys 146, 28, 31 us, 32 of
// 7600 327, 194, 195; 8 heads over 1, 512 of 33000 581, 89, 89; dk and dv of 2048 queries,
// 16 heads over 2, 485, 74, 76 us.
uint32_t runs_for(size_t tiles, double stages, double us, double bytes, size_t room, size_t most, const ar_attention_desc &d,
                  double work = 0.0)
{
    const bool alike = d.sequences == 1 && (!(d.flags & AR_ATTN_CAUSAL) || d.tokens_k >= 4 * d.tokens_q);
    if (d.sequences > 1) stages *= 1.5;
    uint32_t best = 1;
    double time = 0;
    for (uint32_t s = 1; s <= kMaxRuns && (s == 1 || (s <= stages && s * tiles <= most * room)); ++s) {
        double t = stages / s * us;
        if (alike) t *= (tiles * s + room - 1) / room;
        else if (t < work + t / 4) t = work + t / 4;
        if (s > 1) t += 5.0 + s * (0.2 + 2.0 * bytes / 3.4e6);
        if (s == 1 || t < time) best = s, time = t;
    }
    return best;
}
double mean_stages(size_t tokens, const ar_attention_desc &d) { return ceil((double)tokens / d.sequences / kKeys); }
double sums_bytes(size_t rows, const ar_attention_desc &d) { return 4.0 * rows * d.dim; }
// Tiles that there are if the lengths are as even as they can be.
size_t tiles_for(size_t rows, const ar_attention_desc &d, size_t each = kRows)
{
    const size_t n = (rows + each - 1) / each;
    return (n > d.sequences ? n : d.sequences) * d.kv_heads;
}
// Whether the forward pass takes its rows 32 at a time: nearly always where a sequence has
// no more than eight, else where such workgroups find room at once, two on a compute unit
// (or little more, if they have much to do), and there is little to compute in all.  Time by
// 32 rows, of that by 128, means over 8 to 32 heads of dim 128, sequences of 100, 300, 500,
// 1000 tiles: even, of 60 keys 0.92, 0.94, 0.98, 1.20, of 1000 keys 0.87, 0.67, 0.74, 1.03, of
// 8000 keys 1.17, 1.23, 1.15, 1.30; uneven, of 1000 keys 0.91, 0.78, 0.79, 0.88; 32 rows each, of
// 1000 keys 0.94, 0.87, 1.07, 1.04; one or eight rows each 0.7 to 1.1.  Of dim 64: one row each
// of 60 keys 0.89, 0.91, 1.01, 1.26, even of 1000 keys 0.70, 0.50, 0.51, 0.93.
bool few_rows(const ar_attention_desc &d)
{
    const size_t rows = d.tokens_q * (d.heads / d.kv_heads), groups = row_slots(d, kFewRows) * d.kv_heads;
    const double stages = mean_stages(d.tokens_k, d);
    const bool some = groups <= 560 || (stages >= 8 && groups <= 700) || (stages >= 16 && d.dim <= 64 && groups <= 1100);
    if (rows <= 8 * d.sequences) return some || stages >= 16 || d.dim > 64;
    return some && tiles_for(rows, d, kFewRows) * stages <= (d.dim <= 64 ? 32000 : 16000);
}
uint32_t forward_splits(const ar_attention_desc &d)
{
    const size_t rows = d.tokens_q * (d.heads / d.kv_heads);
    const bool few = few_rows(d);
    const size_t tiles = tiles_for(rows, d, few ? kFewRows : kRows);
    const double stages = mean_stages(d.tokens_k, d), bytes = sums_bytes(d.tokens_q * d.heads, d);
    // K and V at 4.8 TB/s, or the tiles' stages with the device full
    const double each = few ? d.dim <= 64 ? 0.9e-3 : 1.5e-3 : d.dim <= 64 ? 3e-3 : 4.5e-3;
    const double work = fmax(4.0 * d.tokens_k * d.kv_heads * d.dim / 4.8e6, tiles * stages * each);
    if (few) return runs_for(tiles, stages, d.dim <= 64 ? 0.37 : 0.6, bytes, 512, 4, d, work);
    return runs_for(tiles, stages, d.dim <= 64 ? 0.9 : 1.2, bytes, 512, 4, d, work);
}
uint32_t dq_splits(const ar_attention_desc &d)
{
    return runs_for(tiles_for(d.tokens_q * (d.heads / d.kv_heads), d), mean_stages(d.tokens_k, d), d.dim <= 64 ? 1.3 : 1.8,
                    sums_bytes(d.tokens_q * d.heads, d), 512, 2, d);
}
uint32_t dkv_splits(const ar_attention_desc &d)
{
    return runs_for(tiles_for(d.tokens_k, d), mean_stages(d.tokens_q, d) * (d.heads / d.kv_heads), d.dim <= 64 ? 1.2 : 1.9,
                    2 * sums_bytes(d.tokens_k * d.kv_heads, d), 256, 2, d);
}

size_t part_bytes(uint32_t splits, size_t rows, size_t each) { return splits > 1 ? round_up(splits * rows * each * sizeof(float), 256) : 0; }
size_t forward_part(const ar_attention_desc &d) { return part_bytes(forward_splits(d), d.tokens_q * d.heads, d.dim + 1); }

bool nothing(const ar_attention_desc &d) { return d.sequences == 0 || (d.tokens_q == 0 && d.tokens_k == 0); }

size_t attention_workspace(const ar_attention_desc &d)
{
    if (nothing(d)) return 0;
    const AttnTensors t = attn_tensors(d, nullptr, nullptr, nullptr, nullptr);
    return t.q.copy_bytes() + t.k.copy_bytes() + t.v.copy_bytes() + forward_part(d);
}
size_t attention_need(const ar_attention_desc &d, const AttnTensors &t)
{
    size_t need = forward_part(d);
    for (const Tensor &in : {t.q, t.k, t.v})
        if (!in.direct()) need += in.copy_bytes();
    return need;
}
size_t attention_workspace_for(const ar_attention_desc *desc, const void *q, const void *k, const void *v)
{
    if (check_attention(desc) != AR_OK || nothing(*desc)) return 0;
    return attention_need(*desc, attn_tensors(*desc, q, k, v, nullptr));
}

// A tensor as the kernels read it: itself, or a copy.
Heads<const bf16> readable(const Tensor &t, char *&ws, HeadsCopies *list)
{
    if (t.direct()) return heads_of<const bf16>(t);
    const uint64_t dim = round_up(t.dim, 8);
    list->c[list->n++] = {heads_of<const bf16>(t), (bf16 *)ws, t.tokens * t.heads, (uint32_t)t.heads};
    const Heads<const bf16> to{(const bf16 *)ws, t.heads * dim, dim};
    ws += t.copy_bytes();
    return to;
}
uint32_t groups_for(uint64_t threads)
{
    const uint64_t n = (threads + 255) / 256;
    return (uint32_t)(n < 1 ? 1 : n < 8192 ? n : 8192);
}
int run_copies(const HeadsCopies &list, hipStream_t st)
{
    if (!list.n) return AR_OK;
    uint64_t most = 0;
    for (uint32_t k = 0; k < list.n; ++k) most = list.c[k].rows > most ? list.c[k].rows : most;
    hipLaunchKernelGGL(attention_pack_kernel, dim3(groups_for(most * ((list.dim + 7) / 8)), list.n), dim3(256), 0, st, list);
    return launch_status();
}

AttnArgs attn_args(const ar_attention_desc &d, const int32_t *starts_q, const int32_t *starts_k)
{
    AttnArgs a{};
    a.starts_q = starts_q, a.starts_k = starts_k;
    a.sequences = (uint32_t)d.sequences, a.tokens_q = (uint32_t)d.tokens_q, a.tokens_k = (uint32_t)d.tokens_k;
    a.heads = (uint32_t)d.heads, a.kv_heads = (uint32_t)d.kv_heads, a.group = (uint32_t)(d.heads / d.kv_heads);
    a.dim = (uint32_t)d.dim, a.dim_in = (uint32_t)round_up(d.dim, 8);
    a.causal = d.flags & AR_ATTN_CAUSAL ? 1 : 0, a.rest = d.flags & AR_ATTN_CLEAR ? 1 : 0, a.scale = d.scale;
    return a;
}

uint32_t groups_of(const AttnArgs &a) { return a.slots * a.kv_heads * a.splits + (a.rest ? kRestGroups : 0); }
template <typename K, typename... A> int launch_tiles(OncePerDevice &once, K kernel, uint32_t groups, int lds, hipStream_t st, A... args)
{
    const int rc = allow_lds(once, (const void *)kernel, lds);
    if (rc != AR_OK) return rc;
    hipLaunchKernelGGL(kernel, dim3(groups), dim3(256), lds, st, args...);
    return launch_status();
}
template <int DP> int launch_forward(const AttnArgs &a, hipStream_t st)
{
    static OncePerDevice once;
    return launch_tiles(once, attention_kernel<DP>, groups_of(a), 4 * Stage<DP>::BYTES, st, a);
}
template <int DP> int launch_few(const AttnArgs &a, hipStream_t st)
{
    static OncePerDevice once;
    return launch_tiles(once, attention_few_kernel<DP>, groups_of(a), Few<DP>::LDS, st, a);
}
// keys, rows: null where not wanted
template <int DP> int launch_backward(const AttnArgs *keys, const AttnArgs *rows, bool together, hipStream_t st)
{
    constexpr int ROWS_LDS = 4 * Stage<DP>::BYTES, KEYS_LDS = ROWS_LDS + 4 * kKeys * (int)sizeof(float);
    static OncePerDevice once[3];
    if (together)
        return launch_tiles(once[2], attention_backward_kernel<DP>, groups_of(*keys) + groups_of(*rows), KEYS_LDS, st, *keys, *rows, groups_of(*keys));
    int rc = AR_OK;
    if (keys) rc = launch_tiles(once[0], attention_dkv_kernel<DP>, groups_of(*keys), KEYS_LDS, st, *keys);
    if (rows && rc == AR_OK) rc = launch_tiles(once[1], attention_dq_kernel<DP>, groups_of(*rows), ROWS_LDS, st, *rows);
    return rc;
}

// What both passes refuse of the inputs.
bool inputs_ok(const ar_attention_desc &d, const AttnTensors &t, const int32_t *starts_q, const int32_t *starts_k)
{
    if ((uintptr_t)starts_q % 4 != 0 || (uintptr_t)starts_k % 4 != 0 || !starts_q != !starts_k) return false;
    if (!starts_q && d.sequences != 1) return false;
    return t.q.ok() && t.k.ok() && t.v.ok() && t.o.ok();
}
Mat starts_mat(const int32_t *s, size_t sequences) { return Mat{s, 1, sequences + 1, sequences + 1, 4}; }

int attention(const ar_attention_desc *desc, const void *q, const void *k, const void *v, const int32_t *starts_q,
              const int32_t *starts_k, void *o, float *lse, void *ws, size_t ws_bytes, void *stream)
{
    int rc = check_attention(desc);
    if (rc != AR_OK) return rc;
    const ar_attention_desc &d = *desc;
    if (nothing(d) || d.tokens_q == 0) return AR_OK;
    const AttnTensors t = attn_tensors(d, q, k, v, o);
    if (!inputs_ok(d, t, starts_q, starts_k) || (uintptr_t)lse % 4 != 0) return AR_ERR_ARG;
    const Mat om = t.o.mat(), lm = mat(lse, d.tokens_q, d.heads, 0, AR_FLOAT32);
    for (const Tensor &in : {t.q, t.k, t.v})
        if (meet(t.o, in) || meet(lm, in.mat())) return AR_ERR_ARG;
    for (const Mat &in : {starts_mat(starts_q, d.sequences), starts_mat(starts_k, d.sequences)})
        if (meet(om, in) || meet(lm, in)) return AR_ERR_ARG;
    if (meet(om, lm)) return AR_ERR_ARG;
    const size_t need = attention_need(d, t);
    if (need) {
        if (!ws || ws_bytes < need) return AR_ERR_SCRATCH;
        if ((uintptr_t)ws % 256 != 0) return AR_ERR_ARG;
        const Mat wm{ws, 1, need, need, 1};
        for (const Mat &x : {t.q.mat(), t.k.mat(), t.v.mat(), om, lm, starts_mat(starts_q, d.sequences), starts_mat(starts_k, d.sequences)})
            if (meet(wm, x)) return AR_ERR_ARG;
    }
    hipStream_t st = (hipStream_t)stream;
    char *at = (char *)ws;
    AttnArgs a = attn_args(d, starts_q, starts_k);
    HeadsCopies copies{};
    copies.dim = a.dim;
    a.q = readable(t.q, at, &copies), a.k = readable(t.k, at, &copies), a.v = readable(t.v, at, &copies);
    if ((rc = run_copies(copies, st)) != AR_OK) return rc;
    a.o = heads_of<bf16>(t.o), a.lse = lse;
    const bool few = few_rows(d);
    a.slots = (uint32_t)row_slots(d, few ? kFewRows : kRows), a.splits = forward_splits(d);
    a.part = (float *)at, a.part_lse = a.part + a.splits * d.tokens_q * d.heads * d.dim;
    if (few) rc = d.dim <= 64 ? launch_few<64>(a, st) : launch_few<128>(a, st);
    else rc = d.dim <= 64 ? launch_forward<64>(a, st) : launch_forward<128>(a, st);
    if (rc != AR_OK || a.splits == 1) return rc;
    hipLaunchKernelGGL(attention_join_kernel, dim3(groups_for(d.tokens_q * d.heads * 64)), dim3(256), 0, st, a);
    return launch_status();
}

// ---- backward -------------------------------------------------------------------

// Where the backward pass keeps what; copies lie behind the rest.
struct BackwardSpace {
    size_t rows, keys, copies;  // the runs' sums of dq, and of dk and dv; delta lies at the start
};
BackwardSpace backward_space(const ar_attention_desc &d, bool dq, bool dkv)
{
    BackwardSpace s{};
    s.rows = round_up(d.tokens_q * d.heads * sizeof(float), 256);
    s.keys = s.rows + (dq ? part_bytes(dq_splits(d), d.tokens_q * d.heads, d.dim) : 0);
    s.copies = s.keys + (dkv ? part_bytes(dkv_splits(d), 2 * d.tokens_k * d.kv_heads, d.dim) : 0);
    return s;
}
// Whether dq shares a launch with dk and dv: a workgroup has a unit to itself there, which
// costs dq half of its rate once there are many.  All of a backward pass, in two launches
// and in one: 1000 tokens, 8 heads of 128 56 and 44 us (160 workgroups), 1000 + 333 queries
// over 1500 + 77 keys, 12 heads of 64, 57 and 40 (552); but 4 x 1024, 16 heads of 128, 124 and
// 130 (1024), 2048, 16 heads over 2, 123 and 128 (928).
bool in_one_launch(const ar_attention_desc &d)
{
    return tiles_for(d.tokens_q * (d.heads / d.kv_heads), d) * dq_splits(d) + tiles_for(d.tokens_k, d) * dkv_splits(d) <= 768;
}
size_t backward_bytes(const ar_attention_desc &d)
{
    if (nothing(d)) return 0;
    const AttnTensors t = attn_tensors(d, nullptr, nullptr, nullptr, nullptr);
    return backward_space(d, true, true).copies + 2 * t.q.copy_bytes() + t.k.copy_bytes() + t.v.copy_bytes();
}

int sum_runs(const RunsList &list, hipStream_t st)
{
    if (!list.n) return AR_OK;
    uint64_t most = 0;
    for (uint32_t k = 0; k < list.n; ++k) {
        const uint64_t n = (uint64_t)list.r[k].tokens * list.r[k].heads;
        most = n > most ? n : most;
    }
    hipLaunchKernelGGL(attention_sum_kernel, dim3(groups_for(most * ((list.dim + 3) / 4)), list.n), dim3(256), 0, st, list);
    return launch_status();
}

int attention_backward(const ar_attention_desc *desc, const void *dout, const void *q, const void *k, const void *v, const void *o,
                       const float *lse, const int32_t *starts_q, const int32_t *starts_k, void *dq, void *dk, void *dv, void *ws,
                       size_t ws_bytes, void *stream)
{
    int rc = check_attention(desc);
    if (rc != AR_OK) return rc;
    const ar_attention_desc &d = *desc;
    if (!dk != !dv) return AR_ERR_ARG;
    if (nothing(d) || (!dq && !dk)) return AR_OK;
    const AttnTensors t = attn_tensors(d, q, k, v, o);
    const Tensor g = tensor(dout, d.tokens_q, d.heads, d.dim, d.ld_dout, d.hs_dout);
    if (!inputs_ok(d, t, starts_q, starts_k) || !g.ok() || (uintptr_t)lse % 4 != 0 || (!lse && d.tokens_q)) return AR_ERR_ARG;
    const Tensor out[3] = {tensor(dq, d.tokens_q, d.heads, d.dim, d.ld_dq, d.hs_dq),
                           tensor(dk, d.tokens_k, d.kv_heads, d.dim, d.ld_dk, d.hs_dk),
                           tensor(dv, d.tokens_k, d.kv_heads, d.dim, d.ld_dv, d.hs_dv)};
    const Mat lm = mat(lse, d.tokens_q, d.heads, 0, AR_FLOAT32);
    const Tensor ins[] = {t.q, t.k, t.v, t.o, g};
    const Mat others[] = {lm, starts_mat(starts_q, d.sequences), starts_mat(starts_k, d.sequences)};
    for (int i = 0; i < 3; ++i) {
        if (!out[i].p) continue;
        if (!out[i].ok()) return AR_ERR_ARG;
        for (const Tensor &in : ins)
            if (meet(out[i], in)) return AR_ERR_ARG;
        for (const Mat &in : others)
            if (meet(out[i].mat(), in)) return AR_ERR_ARG;
        for (int j = 0; j < i; ++j)
            if (out[j].p && meet(out[i], out[j])) return AR_ERR_ARG;
    }
    const size_t need = backward_bytes(d);
    if (!ws || ws_bytes < need) return AR_ERR_SCRATCH;
    if ((uintptr_t)ws % 256 != 0) return AR_ERR_ARG;
    const Mat wm{ws, 1, need, need, 1};
    for (const Tensor &in : ins)
        if (meet(wm, in.mat())) return AR_ERR_ARG;
    for (const Mat &in : others)
        if (meet(wm, in)) return AR_ERR_ARG;
    for (const Tensor &to : out)
        if (to.p && meet(wm, to.mat())) return AR_ERR_ARG;

    hipStream_t st = (hipStream_t)stream;
    const BackwardSpace s = backward_space(d, dq != nullptr, dk != nullptr);
    char *at = (char *)ws + s.copies;
    AttnArgs a = attn_args(d, starts_q, starts_k);
    HeadsCopies copies{};
    copies.dim = a.dim;
    a.q = readable(t.q, at, &copies), a.k = readable(t.k, at, &copies), a.v = readable(t.v, at, &copies), a.dout = readable(g, at, &copies);
    if ((rc = run_copies(copies, st)) != AR_OK) return rc;
    a.lse = (float *)lse, a.delta = (float *)ws;
    if (d.tokens_q) {
        const uint64_t rows = (uint64_t)d.tokens_q * d.heads;
        hipLaunchKernelGGL(attention_delta_kernel, dim3(groups_for(rows * 16)), dim3(256), 0, st, heads_of<const bf16>(g),
                           heads_of<const bf16>(t.o), (float *)ws, rows, a.tokens_q, a.dim);
        if ((rc = launch_status()) != AR_OK) return rc;
    }
    const bool with_keys = dk && d.tokens_k, with_rows = dq && d.tokens_q;
    AttnArgs keys = a, rows = a;
    RunsList runs{};
    runs.sequences = a.sequences, runs.dim = a.dim;
    if (with_keys) {
        keys.dk = heads_of<bf16>(out[1]), keys.dv = heads_of<bf16>(out[2]);
        keys.slots = (uint32_t)key_slots(d), keys.splits = dkv_splits(d), keys.part = (float *)((char *)ws + s.keys);
        if (keys.splits > 1) {
            const uint64_t half = (uint64_t)keys.splits * d.tokens_k * d.kv_heads * d.dim;
            runs.r[runs.n++] = {keys.dk, keys.part, starts_k, a.tokens_k, a.kv_heads, keys.splits};
            runs.r[runs.n++] = {keys.dv, keys.part + half, starts_k, a.tokens_k, a.kv_heads, keys.splits};
        }
    }
    if (with_rows) {
        rows.dq = heads_of<bf16>(out[0]);
        rows.slots = (uint32_t)row_slots(d), rows.splits = dq_splits(d), rows.part = (float *)((char *)ws + s.rows);
        if (rows.splits > 1) runs.r[runs.n++] = {rows.dq, rows.part, starts_q, a.tokens_q, a.heads, rows.splits};
    }
    const bool together = with_keys && with_rows && in_one_launch(d);
    rc = d.dim <= 64 ? launch_backward<64>(with_keys ? &keys : nullptr, with_rows ? &rows : nullptr, together, st)
                     : launch_backward<128>(with_keys ? &keys : nullptr, with_rows ? &rows : nullptr, together, st);
    return rc != AR_OK ? rc : sum_runs(runs, st);
}

}  // namespace
}  // namespace ar

extern "C" int ar_attention(const ar_attention_desc *desc, const void *q, const void *k, const void *v, const int32_t *starts_q,
                            const int32_t *starts_k, void *o, float *lse, void *workspace, size_t workspace_bytes, void *stream)
{
    return ar::ops_ret(ar::attention(desc, q, k, v, starts_q, starts_k, o, lse, workspace, workspace_bytes, stream));
}

extern "C" size_t ar_attention_workspace(const ar_attention_desc *desc)
{
    return ar::check_attention(desc) == AR_OK ? ar::attention_workspace(*desc) : 0;
}

extern "C" size_t ar_attention_workspace_for(const ar_attention_desc *desc, const void *q, const void *k, const void *v)
{
    return ar::attention_workspace_for(desc, q, k, v);
}

extern "C" int ar_attention_backward(const ar_attention_desc *desc, const void *dout, const void *q, const void *k, const void *v,
                                     const void *o, const float *lse, const int32_t *starts_q, const int32_t *starts_k, void *dq,
                                     void *dk, void *dv, void *workspace, size_t workspace_bytes, void *stream)
{
    return ar::ops_ret(ar::attention_backward(desc, dout, q, k, v, o, lse, starts_q, starts_k, dq, dk, dv, workspace, workspace_bytes, stream));
}

extern "C" size_t ar_attention_backward_workspace(const ar_attention_desc *desc)
{
    return ar::check_attention(desc) == AR_OK ? ar::backward_bytes(*desc) : 0;
}
