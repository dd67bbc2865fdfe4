// Residual norm (gfx950): the norm of a block's output, its gate, the scaled
// residual and the norm before the next block in one pass over a row, forward
// and backward (formulas in ar_ops.h).
//
// Memory-bound: the forward reads two rows and writes two, the backward reads
// four and writes two.  A row lives in the registers of one workgroup (NV
// vectors of 16 bytes a thread), so it is read once, and both norms are sums
// over the workgroup with one barrier each.  A workgroup takes a run of
// consecutive rows: the weights and the gate stay in its registers, the next
// row's loads are in flight while this one is summed, and the backward's
// parameter gradients add up in registers and leave as one row of partial
// sums per workgroup, which a second kernel adds in a fixed order.  Rows too wide
// for all of that give up the next row first, then keep those sums in LDS.
//
// 16384 x 8192 bf16 forward 191 us, 5.6 TB/s (a large copy 5.2); 8192 x 4096 bf16
// backward with parameter gradients 98 us, 4.1 TB/s; 2049 x 2501 fp32, rows that
// begin at no vector's bound, 20 us, 4.1 TB/s; one row of 4096 3 us, a launch.
// Wide rows backward: 2048 x 8192 fp32 93 us, 4.3 TB/s; 4096 x 12288 bf16 140 us,
// 4.3 TB/s; 2048 x 12288 fp32 130 us, 4.7 TB/s.
#include <type_traits>

#include "ops_common.h"

#pragma clang fp contract(fast)

namespace ar {
namespace dev {

struct NormArgs {
    const void *y, *residual, *post_w, *gate, *pre_w;
    void *s, *x;
    uint64_t rows, rows_per_gate, ld_y, ld_r, ld_s, ld_x;
    uint32_t cols;
    int flags;
    float alpha, eps;
};

struct NormBwdArgs {
    const void *y, *s, *ds, *dx, *post_w, *gate, *pre_w;
    void *dy, *dr, *dgate;
    float *part;         // [workgroup][kParts][cols]
    uint64_t rows, rows_per_gate, ld_y, ld_s, ld_ds, ld_dx, ld_dy, ld_dr;
    uint32_t cols;
    int flags;
    int want;            // kWant*
    int has_ds;          // else ds is s: read, and taken as zero
    float alpha, eps;
};

// Rows of a workgroup's partial sums: both weights' gradients, and the gate's
// for a gate row that began before the workgroup's rows or ends after them.
constexpr int kPartPost = 0, kPartPre = 1, kPartGateHead = 2, kPartGateTail = 3, kParts = 4;
constexpr int kWantPost = 1, kWantPre = 2, kWantGate = 4;

// Rows [first, last) of workgroup w of n.
__device__ __host__ __forceinline__ uint64_t first_row(uint64_t rows, uint32_t w, uint32_t n) { return rows * w / n; }
// The workgroup that holds row t.
__device__ __forceinline__ uint32_t group_of(uint64_t rows, uint64_t t, uint32_t n)
{
    return (uint32_t)(((t + 1) * n - 1) / rows);
}

template <typename T> constexpr int kVec = 16 / (int)sizeof(T);

// One thread's share of a row, vectors threadIdx.x + k * BS, in its own type: the
// next row waits like this while one is worked on.
template <typename T, int NV> struct RawRow {
    typedef T Vec __attribute__((ext_vector_type(kVec<T>)));
    Vec v[NV];
    __device__ __forceinline__ float at(int k, int j) const { return (float)v[k][j]; }
};
template <int NV, int BS, bool TAIL, typename T>
__device__ __forceinline__ void load_raw(const T *p, uint32_t cols, RawRow<T, NV> &out)
{
    constexpr int VEC = kVec<T>;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const uint32_t at = (threadIdx.x + k * BS) * VEC;
        if (at + VEC <= cols) {
            out.v[k] = *(const typename VecOf<T, VEC>::type *)(p + at);
        } else {
#pragma unroll
            for (int j = 0; j < VEC; ++j) out.v[k][j] = TAIL && at + j < cols ? p[at + j] : (T)0.0f;
        }
    }
}

template <typename T, int VEC, int NV, int BS, bool TAIL>
__device__ __forceinline__ void load_row(const T *p, uint32_t cols, float (*out)[VEC])
{
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const uint32_t at = (threadIdx.x + k * BS) * VEC;
        if (at + VEC <= cols) {
            load_vec<T, VEC>(p + at, out[k]);
        } else if (TAIL && at < cols) {
            load_part<T, VEC>(p + at, (int)(cols - at), out[k]);
        } else {
#pragma unroll
            for (int j = 0; j < VEC; ++j) out[k][j] = 0.0f;
        }
    }
}

template <typename T, int VEC, int NV, int BS, bool TAIL>
__device__ __forceinline__ void store_row(T *p, uint32_t cols, const float (*v)[VEC])
{
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const uint32_t at = (threadIdx.x + k * BS) * VEC;
        if (at + VEC <= cols) store_vec<T, VEC>(p + at, v[k]);
        else if (TAIL && at < cols) store_part<T, VEC>(p + at, (int)(cols - at), v[k]);
    }
}

// A weight or gate; absent ones are ones.
template <typename P, int VEC, int NV, int BS, bool TAIL>
__device__ __forceinline__ void load_param(const void *p, uint32_t cols, float (*out)[VEC])
{
    if (p) {
        load_row<P, VEC, NV, BS, TAIL>((const P *)p, cols, out);
    } else {
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int j = 0; j < VEC; ++j) out[k][j] = 1.0f;
    }
}

template <typename T, typename P, int NV, int BS, bool TAIL>
__global__ __launch_bounds__(BS) void norm_kernel(const NormArgs a)
{
    constexpr int VEC = kVec<T>, W = BS / 64;
    __shared__ float slots[2][W];
    uint32_t turn = 0;
    const bool post = (a.flags & AR_NORM_POST) != 0, pre = (a.flags & AR_NORM_PRE) != 0;
    const uint64_t last = first_row(a.rows, blockIdx.x + 1, gridDim.x);
    uint64_t row = first_row(a.rows, blockIdx.x, gridDim.x);
    if (row >= last) return;
    const float inv = 1.0f / (float)a.cols;
    float w1[NV][VEC], w2[NV][VEC], g[NV][VEC];
    RawRow<T, NV> y, r, next_y, next_r;
    load_raw<NV, BS, TAIL>((const T *)a.y + row * a.ld_y, a.cols, next_y);
    load_raw<NV, BS, TAIL>((const T *)a.residual + row * a.ld_r, a.cols, next_r);
    load_param<P, VEC, NV, BS, TAIL>(post ? a.post_w : nullptr, a.cols, w1);
    load_param<P, VEC, NV, BS, TAIL>(a.pre_w, a.cols, w2);
    uint64_t gate_end = 0;  // first row that this gate row does not hold for
    for (; row < last; ++row) {
        if (row >= gate_end) {
            const uint64_t k = row / a.rows_per_gate;
            gate_end = (k + 1) * a.rows_per_gate;
            load_param<P, VEC, NV, BS, TAIL>(a.gate ? (const P *)a.gate + k * a.cols : nullptr, a.cols, g);
        }
        y = next_y, r = next_r;
        if (row + 1 < last) {
            load_raw<NV, BS, TAIL>((const T *)a.y + (row + 1) * a.ld_y, a.cols, next_y);
            load_raw<NV, BS, TAIL>((const T *)a.residual + (row + 1) * a.ld_r, a.cols, next_r);
        }
        float sum[1] = {0.0f}, r1 = 1.0f;
        if (post) {
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int j = 0; j < VEC; ++j) sum[0] += y.at(k, j) * y.at(k, j);
            group_sum<W, 1>(sum, slots, turn);
            r1 = 1.0f / sqrtf(sum[0] * inv + a.eps);
        }
        float v[NV][VEC];
        sum[0] = 0.0f;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                v[k][j] = a.alpha * r.at(k, j) + g[k][j] * (y.at(k, j) * r1 * w1[k][j]);
                sum[0] += v[k][j] * v[k][j];
            }
        store_row<T, VEC, NV, BS, TAIL>((T *)a.s + row * a.ld_s, a.cols, v);
        if (pre) {
            group_sum<W, 1>(sum, slots, turn);
            const float r2 = 1.0f / sqrtf(sum[0] * inv + a.eps);
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int j = 0; j < VEC; ++j) v[k][j] = v[k][j] * r2 * w2[k][j];
            store_row<T, VEC, NV, BS, TAIL>((T *)a.x + row * a.ld_x, a.cols, v);
        }
    }
}

// Rows too long for registers: each pass reads the row again, from the caches
// where it fits them.  A thread meets the same elements in every pass, so the
// outputs may still be the inputs.
constexpr int kLongThreads = 1024;

// f(first column, how many) for this thread's vectors of four columns.
template <typename F> __device__ __forceinline__ void long_row(uint32_t cols, F f)
{
    for (uint32_t i = threadIdx.x * 4; i < cols; i += kLongThreads * 4) f(i, i + 4 <= cols ? 4 : (int)(cols - i));
}
template <typename T> __device__ __forceinline__ void load4(const T *p, uint32_t at, int have, float *out)
{
    if (have == 4) load_vec<T, 4>(p + at, out);
    else load_part<T, 4>(p + at, have, out);
}
template <typename T> __device__ __forceinline__ void store4(T *p, uint32_t at, int have, const float *in)
{
    if (have == 4) store_vec<T, 4>(p + at, in);
    else store_part<T, 4>(p + at, have, in);
}
// A weight or gate; absent ones are ones.
template <typename P> __device__ __forceinline__ void param4(const P *p, uint32_t at, int have, float *out)
{
    if (p) load4(p, at, have, out);
    else out[0] = out[1] = out[2] = out[3] = 1.0f;
}

template <typename T, typename P> __global__ __launch_bounds__(kLongThreads) void norm_long_kernel(const NormArgs a)
{
    constexpr int W = kLongThreads / 64;
    __shared__ float slots[2][W];
    uint32_t turn = 0;
    const bool post = (a.flags & AR_NORM_POST) != 0, pre = (a.flags & AR_NORM_PRE) != 0;
    const float inv = 1.0f / (float)a.cols;
    const P *w1 = post ? (const P *)a.post_w : nullptr, *w2 = (const P *)a.pre_w;
    for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *y = (const T *)a.y + row * a.ld_y, *r = (const T *)a.residual + row * a.ld_r;
        const P *g = a.gate ? (const P *)a.gate + row / a.rows_per_gate * a.cols : nullptr;
        float sum[1] = {0.0f}, r1 = 1.0f, r2 = 1.0f;
        if (post) {
            long_row(a.cols, [&](uint32_t i, int have) {
                float v[4];
                load4(y, i, have, v);
                for (int k = 0; k < 4; ++k) sum[0] += v[k] * v[k];
            });
            group_sum<W, 1>(sum, slots, turn);
            r1 = 1.0f / sqrtf(sum[0] * inv + a.eps);
        }
        auto at = [&](uint32_t i, int have, float *v) {
            float u[4], w[4], h[4];
            load4(y, i, have, v), load4(r, i, have, u), param4(w1, i, have, w), param4(g, i, have, h);
            for (int k = 0; k < 4; ++k) v[k] = a.alpha * u[k] + h[k] * (v[k] * r1 * w[k]);
        };
        if (pre) {
            sum[0] = 0.0f;
            long_row(a.cols, [&](uint32_t i, int have) {
                float v[4];
                at(i, have, v);
                for (int k = 0; k < have; ++k) sum[0] += v[k] * v[k];
            });
            group_sum<W, 1>(sum, slots, turn);
            r2 = 1.0f / sqrtf(sum[0] * inv + a.eps);
        }
        T *s = (T *)a.s + row * a.ld_s, *x = (T *)a.x + row * a.ld_x;
        long_row(a.cols, [&](uint32_t i, int have) {
            float v[4], w[4];
            at(i, have, v);
            if (pre) param4(w2, i, have, w);
            store4(s, i, have, v);
            if (!pre) return;
            for (int k = 0; k < 4; ++k) v[k] = v[k] * r2 * w[k];
            store4(x, i, have, v);
        });
    }
}

// Where a workgroup's sum for the gate row that ends (or pauses) here goes:
// straight to the gradient if all of that gate row's rows were its own, else
// to the head or tail row of its partial sums.
template <typename P> struct GateOut {
    P *whole;
    float *part;
};
template <typename P>
__device__ __forceinline__ GateOut<P> gate_out(const NormBwdArgs &a, float *part, uint64_t k, uint64_t first, uint64_t last)
{
    const uint64_t begin = k * a.rows_per_gate, end = begin + a.rows_per_gate;
    if (begin >= first && end <= last) return {(P *)a.dgate + k * a.cols, nullptr};
    return {nullptr, part + (size_t)(begin < first ? kPartGateHead : kPartGateTail) * a.cols};
}

// Where a workgroup of wide rows finds registers: the next row is loaded only
// when this one is done (kNoneAhead), and the parameter gradients add up in LDS,
// each thread's in slots of its own, without barriers (kSumsInLds).
enum Room { kNextAhead, kNoneAhead, kSumsInLds };

// A parameter gradient's share of a thread.
template <int VEC, int NV, int BS, bool LDS> struct ParamSum {
    float v[NV][VEC];
    __device__ __forceinline__ ParamSum(float *) { clear(); }
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int j = 0; j < VEC; ++j) v[k][j] = 0.0f;
    }
    __device__ __forceinline__ void add(int k, const float *x)
    {
#pragma unroll
        for (int j = 0; j < VEC; ++j) v[k][j] += x[j];
    }
    template <typename O, bool TAIL> __device__ __forceinline__ void store(O *p, uint32_t cols) const
    {
        store_row<O, VEC, NV, BS, TAIL>(p, cols, v);
    }
};
template <int VEC, int NV, int BS> struct ParamSum<VEC, NV, BS, true> {
    static constexpr int N = NV * VEC / 4;  // vectors of four, those of all threads side by side
    typedef float f32x4 __attribute__((ext_vector_type(4)));
    f32x4 *at;
    __device__ __forceinline__ ParamSum(float *lds) : at((f32x4 *)lds + threadIdx.x) { clear(); }
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int n = 0; n < N; ++n) at[n * BS] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    __device__ __forceinline__ void add(int k, const float *x)
    {
#pragma unroll
        for (int n = 0; n < VEC / 4; ++n) at[(k * (VEC / 4) + n) * BS] += f32x4{x[n * 4], x[n * 4 + 1], x[n * 4 + 2], x[n * 4 + 3]};
    }
    template <typename O, bool TAIL> __device__ __forceinline__ void store(O *p, uint32_t cols) const
    {
        float v[NV][VEC];
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int j = 0; j < 4; ++j) v[n / (VEC / 4)][n % (VEC / 4) * 4 + j] = at[n * BS][j];
        store_row<O, VEC, NV, BS, TAIL>(p, cols, v);
    }
};
template <typename T, int NV, int BS> constexpr int kSumsBytes = 3 * NV * kVec<T> * BS * 4;

template <typename T, typename P, int NV, int BS, bool TAIL, Room ROOM = kNextAhead>
__global__ __launch_bounds__(BS) void norm_bwd_kernel(const NormBwdArgs a)
{
    constexpr int VEC = kVec<T>, W = BS / 64;
    __shared__ float slots3[2][W * 3], slots1[2][W];
    uint32_t turn3 = 0, turn1 = 0;
    const bool post = (a.flags & AR_NORM_POST) != 0, pre = (a.flags & AR_NORM_PRE) != 0;
    const uint64_t first = first_row(a.rows, blockIdx.x, gridDim.x), last = first_row(a.rows, blockIdx.x + 1, gridDim.x);
    if (first >= last) return;
    float *part = a.part + (size_t)blockIdx.x * kParts * a.cols;
    const float inv = 1.0f / (float)a.cols;
    extern __shared__ __attribute__((aligned(16))) float sums[];
    typedef ParamSum<VEC, NV, BS, ROOM == kSumsInLds> Sum;
    Sum dw1(sums), dw2(sums + NV * VEC * BS), dg(sums + 2 * NV * VEC * BS);
    float w1[NV][VEC], w2[NV][VEC], g[NV][VEC];
    load_param<P, VEC, NV, BS, TAIL>(post ? a.post_w : nullptr, a.cols, w1);
    load_param<P, VEC, NV, BS, TAIL>(a.pre_w, a.cols, w2);
    RawRow<T, NV> y, z, ds, dx, next_y, next_z, next_ds, next_dx;
    auto load_next = [&](uint64_t row) {
        load_raw<NV, BS, TAIL>((const T *)a.y + row * a.ld_y, a.cols, next_y);
        load_raw<NV, BS, TAIL>((const T *)a.s + row * a.ld_s, a.cols, next_z);
        // absent ones are not used (dx), or read where s is and taken as zero (ds)
        load_raw<NV, BS, TAIL>((const T *)a.ds + row * a.ld_ds, a.cols, next_ds);
        load_raw<NV, BS, TAIL>((const T *)a.dx + row * a.ld_dx, a.cols, next_dx);
    };
    if constexpr (ROOM == kNextAhead) load_next(first);
    uint64_t gate_end = 0;
    for (uint64_t row = first; row < last; ++row) {
        if constexpr (ROOM != kNextAhead) load_next(row);
        if (row >= gate_end) {
            const uint64_t k = row / a.rows_per_gate;
            gate_end = (k + 1) * a.rows_per_gate;
            load_param<P, VEC, NV, BS, TAIL>(a.gate ? (const P *)a.gate + k * a.cols : nullptr, a.cols, g);
        }
        y = next_y, z = next_z, ds = next_ds, dx = next_dx;
        if constexpr (ROOM == kNextAhead) {
            if (row + 1 < last) load_next(row + 1);
        }
        float sum[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                sum[0] += y.at(k, j) * y.at(k, j);
                if (pre) {
                    sum[1] += z.at(k, j) * z.at(k, j);
                    sum[2] += dx.at(k, j) * w2[k][j] * z.at(k, j);
                }
            }
        if (post || pre) group_sum<W, 3>(sum, slots3, turn3);
        const float r1 = post ? 1.0f / sqrtf(sum[0] * inv + a.eps) : 1.0f;
        const float r2 = pre ? 1.0f / sqrtf(sum[1] * inv + a.eps) : 1.0f;
        const float c2 = r2 * r2 * (sum[2] * inv);
        float svy[1] = {0.0f}, out[NV][VEC], v[NV][VEC];
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            float of_w1[VEC], of_w2[VEC], of_g[VEC];
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                float G = a.has_ds ? ds.at(k, j) : 0.0f;
                of_w2[j] = 0.0f;
                if (pre) {
                    G += r2 * (dx.at(k, j) * w2[k][j] - z.at(k, j) * c2);
                    of_w2[j] = dx.at(k, j) * (z.at(k, j) * r2);
                }
                const float unit = y.at(k, j) * r1, dn = G * g[k][j];
                of_g[j] = G * (unit * w1[k][j]);
                of_w1[j] = dn * unit;
                out[k][j] = a.alpha * G;
                v[k][j] = dn * w1[k][j];
                svy[0] += v[k][j] * y.at(k, j);
            }
            dw1.add(k, of_w1), dw2.add(k, of_w2), dg.add(k, of_g);
        }
        store_row<T, VEC, NV, BS, TAIL>((T *)a.dr + row * a.ld_dr, a.cols, out);
        if (post) {
            group_sum<W, 1>(svy, slots1, turn1);
            const float c1 = r1 * r1 * (svy[0] * inv);
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int j = 0; j < VEC; ++j) v[k][j] = r1 * (v[k][j] - y.at(k, j) * c1);
        }
        store_row<T, VEC, NV, BS, TAIL>((T *)a.dy + row * a.ld_dy, a.cols, v);
        if ((a.want & kWantGate) && (row + 1 == gate_end || row + 1 == last)) {
            const GateOut<P> o = gate_out<P>(a, part, row / a.rows_per_gate, first, last);
            if (o.whole) dg.template store<P, TAIL>(o.whole, a.cols);
            else dg.template store<float, TAIL>(o.part, a.cols);
            dg.clear();
        }
    }
    if (a.want & kWantPost) dw1.template store<float, TAIL>(part + (size_t)kPartPost * a.cols, a.cols);
    if (a.want & kWantPre) dw2.template store<float, TAIL>(part + (size_t)kPartPre * a.cols, a.cols);
}

// Rows too long for registers, see norm_long_kernel; the parameter gradients
// add up in the workgroup's rows of partial sums.
template <typename T, typename P> __global__ __launch_bounds__(kLongThreads) void norm_bwd_long_kernel(const NormBwdArgs a)
{
    constexpr int W = kLongThreads / 64;
    __shared__ float slots3[2][W * 3], slots1[2][W];
    uint32_t turn3 = 0, turn1 = 0;
    const bool post = (a.flags & AR_NORM_POST) != 0, pre = (a.flags & AR_NORM_PRE) != 0;
    const uint64_t first = first_row(a.rows, blockIdx.x, gridDim.x), last = first_row(a.rows, blockIdx.x + 1, gridDim.x);
    float *part = a.part + (size_t)blockIdx.x * kParts * a.cols;
    const float inv = 1.0f / (float)a.cols;
    const P *w1 = post ? (const P *)a.post_w : nullptr, *w2 = (const P *)a.pre_w;
    for (uint64_t row = first; row < last; ++row) {
        const T *y = (const T *)a.y + row * a.ld_y, *z = (const T *)a.s + row * a.ld_s;
        const T *ds = (const T *)a.ds + row * a.ld_ds, *dx = (const T *)a.dx + row * a.ld_dx;
        const uint64_t gk = row / a.rows_per_gate;
        const P *g = a.gate ? (const P *)a.gate + gk * a.cols : nullptr;
        float sum[3] = {0.0f, 0.0f, 0.0f};
        if (post || pre) {
            long_row(a.cols, [&](uint32_t i, int have) {
                float v[4], u[4], d[4], w[4];
                load4(y, i, have, v), load4(z, i, have, u), load4(dx, i, have, d), param4(w2, i, have, w);
                for (int k = 0; k < have; ++k) {
                    sum[0] += v[k] * v[k];
                    if (pre) sum[1] += u[k] * u[k], sum[2] += d[k] * w[k] * u[k];
                }
            });
            group_sum<W, 3>(sum, slots3, turn3);
        }
        const float r1 = post ? 1.0f / sqrtf(sum[0] * inv + a.eps) : 1.0f;
        const float r2 = pre ? 1.0f / sqrtf(sum[1] * inv + a.eps) : 1.0f;
        const float c2 = r2 * r2 * (sum[2] * inv);
        // the gradient of s, and dx * s / rms(s)
        auto total = [&](uint32_t i, int have, float *G, float *unit2) {
            float u[4], d[4], w[4];
            load4(ds, i, have, G), load4(z, i, have, u), load4(dx, i, have, d), param4(w2, i, have, w);
            for (int k = 0; k < 4; ++k) {
                if (!a.has_ds) G[k] = 0.0f;
                if (pre) G[k] += r2 * (d[k] * w[k] - u[k] * c2);
                unit2[k] = d[k] * (u[k] * r2);
            }
        };
        float svy[1] = {0.0f}, c1 = 0.0f;
        if (post) {
            long_row(a.cols, [&](uint32_t i, int have) {
                float G[4], t[4], v[4], w[4], h[4];
                total(i, have, G, t), load4(y, i, have, v), param4(w1, i, have, w), param4(g, i, have, h);
                for (int k = 0; k < have; ++k) svy[0] += G[k] * h[k] * w[k] * v[k];
            });
            group_sum<W, 1>(svy, slots1, turn1);
            c1 = r1 * r1 * (svy[0] * inv);
        }
        const bool new_gate = row == first || row % a.rows_per_gate == 0;
        const GateOut<P> o = gate_out<P>(a, part, gk, first, last);
        const bool gate_ends = o.whole && (row + 1) % a.rows_per_gate == 0;
        // a gate row that ends here adds up in the tail row until then
        float *acc = o.whole ? part + (size_t)kPartGateTail * a.cols : o.part;
        auto add = [&](float *p, uint32_t i, int have, bool fresh, float *v) {
            float old[4];
            if (!fresh) {
                load4(p, i, have, old);
                for (int k = 0; k < 4; ++k) v[k] += old[k];
            }
        };
        long_row(a.cols, [&](uint32_t i, int have) {
            float G[4], t[4], v[4], w[4], h[4], dn[4], p[4];
            total(i, have, G, t), load4(y, i, have, v), param4(w1, i, have, w), param4(g, i, have, h);
            if (a.want & kWantPre) {
                float *to = part + (size_t)kPartPre * a.cols;
                add(to, i, have, row == first, t);
                store4(to, i, have, t);
            }
            for (int k = 0; k < 4; ++k) dn[k] = G[k] * h[k];
            if (a.want & kWantPost) {
                float *to = part + (size_t)kPartPost * a.cols;
                for (int k = 0; k < 4; ++k) p[k] = dn[k] * (v[k] * r1);
                add(to, i, have, row == first, p);
                store4(to, i, have, p);
            }
            if (a.want & kWantGate) {
                for (int k = 0; k < 4; ++k) p[k] = G[k] * (v[k] * r1 * w[k]);
                add(acc, i, have, new_gate, p);
                if (gate_ends) store4(o.whole, i, have, p);
                else store4(acc, i, have, p);
            }
            for (int k = 0; k < 4; ++k) {
                const float q = dn[k] * w[k];
                dn[k] = post ? r1 * (q - v[k] * c1) : q;
                G[k] = a.alpha * G[k];
            }
            store4((T *)a.dr + row * a.ld_dr, i, have, G);
            store4((T *)a.dy + row * a.ld_dy, i, have, dn);
        });
    }
}

// The parameter gradients from the workgroups' partial sums, added in the
// order of the rows: 64 columns a workgroup, kFinishWaves runs of workgroups
// side by side.  blockIdx.y: 0 post weight, 1 pre weight, from 2 on the gate
// rows whose rows fell to several workgroups.
constexpr int kFinishWaves = 16;

struct FinishArgs {
    const float *part;
    void *dpost, *dpre, *dgate;
    uint64_t rows, rows_per_gate, gate_rows;
    uint32_t cols, groups;
};

template <typename P> __global__ __launch_bounds__(64 * kFinishWaves) void norm_finish_kernel(const FinishArgs a)
{
    __shared__ float sums[kFinishWaves][64];
    uint32_t w0 = 0, w1 = a.groups - 1;  // workgroups to add, both included
    P *out;
    int head, which;
    if (blockIdx.y < 2) {
        which = head = blockIdx.y == 0 ? kPartPost : kPartPre;
        out = (P *)(blockIdx.y == 0 ? a.dpost : a.dpre);
        if (!out) return;
    } else {
        uint64_t k = blockIdx.y - 2;
        if (!a.dgate) return;
        if (a.gate_rows > a.groups) {
            // at most one such gate row begins in each workgroup: the one of its last row
            w0 = (uint32_t)k;
            k = (first_row(a.rows, w0 + 1, a.groups) - 1) / a.rows_per_gate;
            if (k * a.rows_per_gate < first_row(a.rows, w0, a.groups)) return;
        } else {
            w0 = group_of(a.rows, k * a.rows_per_gate, a.groups);
        }
        w1 = group_of(a.rows, (k + 1) * a.rows_per_gate - 1, a.groups);
        if (w0 == w1) return;  // written whole
        which = kPartGateHead;
        // a gate row that begins with its first workgroup's rows is in its tail row
        head = kPartGateTail;
        out = (P *)a.dgate + k * a.cols;
    }
    const uint32_t col = blockIdx.x * 64 + (threadIdx.x & 63u), wave = threadIdx.x >> 6;
    const uint32_t n = w1 - w0 + 1, from = w0 + (uint32_t)((uint64_t)n * wave / kFinishWaves),
                   to = w0 + (uint32_t)((uint64_t)n * (wave + 1) / kFinishWaves);
    float t = 0.0f;
    if (col < a.cols) {
#pragma unroll 16
        for (uint32_t w = from; w < to; ++w)
            t += a.part[((size_t)w * kParts + (w == w0 ? head : which)) * a.cols + col];
    }
    sums[wave][threadIdx.x & 63u] = t;
    __syncthreads();
    if (wave == 0 && col < a.cols) {
#pragma unroll
        for (int k = 1; k < kFinishWaves; ++k) t += sums[k][threadIdx.x];
        out[col] = (P)t;
    }
}

template <typename P> __global__ void norm_zero_kernel(P *p, uint64_t n)
{
    for (uint64_t i = (uint64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (uint64_t)gridDim.x * blockDim.x)
        p[i] = (P)0.0f;
}

}  // namespace dev

namespace {

using namespace dev;

// Rows below this leave compute units without a workgroup: then a row is
// spread over more threads.
constexpr size_t kFewRows = 256;

int check_norm(const ar_norm_desc *d)
{
    if (!d) return AR_ERR_ARG;
    if (!known_dtype(d->dtype) || !known_dtype(d->param_dtype)) return AR_ERR_UNSUPPORTED;
    if (d->cols < 1 || d->cols > (1u << 30) || d->rows > kOpsMaxSize / d->cols) return AR_ERR_ARG;
    if (d->flags & ~(AR_NORM_POST | AR_NORM_PRE)) return AR_ERR_ARG;
    if (!isfinite(d->alpha)) return AR_ERR_ARG;
    if (d->flags && (!isfinite(d->eps) || d->eps <= 0.0f)) return AR_ERR_ARG;
    if (d->gate_rows > kOpsMaxSize / d->cols || (d->gate_rows && d->rows % d->gate_rows != 0)) return AR_ERR_ARG;
    for (size_t ld : {d->ld_y, d->ld_residual, d->ld_s, d->ld_x, d->ld_ds, d->ld_dx, d->ld_dy})
        if (ld && (ld < d->cols || ld > kOpsMaxSize / (d->rows ? d->rows : 1))) return AR_ERR_ARG;
    return AR_OK;
}

// An output may be one of the inputs it is read with element by element, and
// meets nothing else.
int check_outputs(const Mat *outs, int n_out, const Mat *ins, int n_in, const Mat *params, int n_par)
{
    for (int i = 0; i < n_out; ++i) {
        if (!outs[i].p) continue;
        for (int j = 0; j < n_in; ++j)
            if (meet(outs[i], ins[j]) && !outs[i].same(ins[j])) return AR_ERR_ARG;
        for (int j = 0; j < n_par; ++j)
            if (meet(outs[i], params[j])) return AR_ERR_ARG;
        for (int j = 0; j < i; ++j)
            if (meet(outs[i], outs[j])) return AR_ERR_ARG;
    }
    return AR_OK;
}

uint64_t rows_per_gate(const ar_norm_desc &d) { return d.gate_rows ? d.rows / d.gate_rows : (d.rows ? d.rows : 1); }

// Threads of a row and vectors of each, by the vectors of a row.  Two vectors a
// thread rather than four: 16384 x 8192 bf16 forward, 256 threads of four 216
// us, 512 of two 190, 1024 of one 238 (its waves wait for each other longer).
// Few rows are spread over more threads.
struct RowShape {
    int threads, vecs;  // 0: the row does not fit
};
RowShape forward_shape(size_t nvec, bool few, int dtype)
{
    if (few && nvec > 64) {
        if (nvec <= 256) return {256, 1};
        if (nvec <= 1024) return {1024, 1};
    }
    if (nvec <= 64) return {64, 1};
    if (nvec <= 128) return {64, 2};
    if (nvec <= 512) return {256, 2};
    if (nvec <= 1024) return {512, 2};
    if (nvec <= 2048) return {512, 4};
    if (nvec <= 3072 && dtype == AR_FLOAT32) return {1024, 3};
    return {0, 0};
}
// The backward holds four rows, three parameters and their sums; above 1024
// vectors see Room.  What does not fit goes several times over memory (2048 x
// 5120 fp32: in registers 52 us, so 123; 2048 x 12288: with the sums in LDS 130
// us, so 287; 4096 x 12288 bf16: 140 and 495).
RowShape backward_shape(size_t nvec, int dtype)
{
    if (nvec <= 64) return {64, 1};
    if (nvec <= 256) return {256, 1};
    if (nvec <= 512) return {256, 2};
    if (nvec <= 1024) return {512, 2};
    if (nvec <= 1536) return {512, 3};
    if (nvec <= 2048 && dtype == AR_FLOAT32) return {512, 4};
    if (nvec <= 3072 && dtype == AR_FLOAT32) return {512, 6};
    return {0, 0};
}

// Workgroups of the forward: each with a run of rows, as many as the device
// holds at once, and with many rows more of shorter runs (16384 x 8192 bf16:
// 1024 workgroups 214 us, 8192 190).
uint32_t forward_groups(const ar_norm_desc &d, int threads)
{
    const size_t fit = 256 * (size_t)(2048 / threads), half = d.rows / 2 < 8192 ? d.rows / 2 : 8192;
    const size_t groups = half > fit ? half : fit;
    return (uint32_t)(d.rows < groups ? d.rows : groups);
}
// The backward pass writes a row of partial sums for each workgroup: as few as
// keep the device busy (8192 x 4096 bf16, of 256 threads: 512 89 us, 1024 94,
// 256 115; 8192 x 8192, of 512 threads: 256 179 us, 512 188; 65536 x 512, of one
// wave: 2048 85 us, 1024 126; 4096 no better).  Rows of one wave are short beside
// their workgroup's partial sums: at least eight of them to a workgroup (1834 x 248
// 16.6 us, one to a workgroup 25.8; 5445 x 176 22.6 and 27.5).  For wider rows
// that is slower (2000 x 4096: 33 us for 30).
uint32_t backward_groups(const ar_norm_desc &d)
{
    const RowShape sh = backward_shape((d.cols * elem_bytes(d.dtype) + 15) / 16, d.dtype);
    const size_t most = sh.threads == 64 ? 2048 : sh.threads == 256 ? 512 : 256;
    const size_t few = sh.threads == 64 && d.rows > 256 ? (d.rows / 8 > 256 ? d.rows / 8 : 256) : d.rows;
    return (uint32_t)(few < most ? few : most);
}

template <typename T, typename P> int launch_norm(const ar_norm_desc &d, const NormArgs &a, hipStream_t st)
{
    const size_t nvec = (d.cols + kVec<T> - 1) / kVec<T>;
    const bool tail = d.cols % kVec<T> != 0;
    const RowShape sh = forward_shape(nvec, d.rows <= kFewRows, d.dtype);
    if (!sh.threads) {
        hipLaunchKernelGGL((norm_long_kernel<T, P>), dim3(forward_groups(d, kLongThreads)), dim3(kLongThreads), 0, st, a);
        return launch_status();
    }
    const dim3 grid(forward_groups(d, sh.threads));
#define AR_NORM_CASE(BS, NV)                                                                                   \
    if (sh.threads == BS && sh.vecs == NV) {                                                                   \
        if (tail) hipLaunchKernelGGL((norm_kernel<T, P, NV, BS, true>), grid, dim3(BS), 0, st, a);             \
        else hipLaunchKernelGGL((norm_kernel<T, P, NV, BS, false>), grid, dim3(BS), 0, st, a);                 \
        return launch_status();                                                                                \
    }
    AR_NORM_CASE(64, 1)
    AR_NORM_CASE(64, 2)
    AR_NORM_CASE(256, 1)
    AR_NORM_CASE(256, 2)
    AR_NORM_CASE(512, 2)
    AR_NORM_CASE(512, 4)
    AR_NORM_CASE(1024, 1)
    if constexpr (sizeof(T) == 4) {
        AR_NORM_CASE(1024, 3)
    }
#undef AR_NORM_CASE
    return AR_ERR_UNSUPPORTED;
}

template <typename T, typename P, int NV, int BS, bool TAIL, Room ROOM>
int launch_bwd_shape(const NormBwdArgs &a, uint32_t groups, hipStream_t st)
{
    constexpr int LDS = ROOM == kSumsInLds ? kSumsBytes<T, NV, BS> : 0;
    if (LDS) {
        static OncePerDevice once;
        const int rc = allow_lds(once, (const void *)norm_bwd_kernel<T, P, NV, BS, TAIL, ROOM>, LDS);
        if (rc != AR_OK) return rc;
    }
    hipLaunchKernelGGL((norm_bwd_kernel<T, P, NV, BS, TAIL, ROOM>), dim3(groups), dim3(BS), LDS, st, a);
    return launch_status();
}

template <typename T, typename P>
int launch_norm_bwd(const ar_norm_desc &d, const NormBwdArgs &a, uint32_t groups, hipStream_t st)
{
    const size_t nvec = (d.cols + kVec<T> - 1) / kVec<T>;
    const bool tail = d.cols % kVec<T> != 0;
    const RowShape sh = backward_shape(nvec, d.dtype);
    if (!sh.threads) {
        hipLaunchKernelGGL((norm_bwd_long_kernel<T, P>), dim3(groups), dim3(kLongThreads), 0, st, a);
        return launch_status();
    }
#define AR_NORM_CASE(BS, NV, ROOM)                                                     \
    if (sh.threads == BS && sh.vecs == NV)                                             \
        return tail ? launch_bwd_shape<T, P, NV, BS, true, ROOM>(a, groups, st)        \
                    : launch_bwd_shape<T, P, NV, BS, false, ROOM>(a, groups, st);
    AR_NORM_CASE(64, 1, kNextAhead)
    AR_NORM_CASE(256, 1, kNextAhead)
    AR_NORM_CASE(256, 2, kNextAhead)
    AR_NORM_CASE(512, 2, kNextAhead)
    AR_NORM_CASE(512, 3, sizeof(T) == 4 ? kNoneAhead : kSumsInLds)
    if constexpr (sizeof(T) == 4) {
        AR_NORM_CASE(512, 4, kNoneAhead)
        AR_NORM_CASE(512, 6, kSumsInLds)
    }
#undef AR_NORM_CASE
    return AR_ERR_UNSUPPORTED;
}

template <typename P> int zero_param(void *p, uint64_t n, hipStream_t st)
{
    if (!p || !n) return AR_OK;
    const uint64_t groups = (n + 255) / 256;
    hipLaunchKernelGGL((norm_zero_kernel<P>), dim3((uint32_t)(groups < 2048 ? groups : 2048)), dim3(256), 0, st, (P *)p, n);
    return launch_status();
}

int norm(const ar_norm_desc *desc, const void *y, const void *residual, const void *post_w, const void *gate,
         const void *pre_w, void *s, void *x, void *stream)
{
    int rc = check_norm(desc);
    if (rc != AR_OK) return rc;
    const ar_norm_desc &d = *desc;
    const bool post = d.flags & AR_NORM_POST, pre = d.flags & AR_NORM_PRE;
    if (d.rows == 0) return AR_OK;
    const Mat ins[] = {mat(y, d.rows, d.cols, d.ld_y, d.dtype), mat(residual, d.rows, d.cols, d.ld_residual, d.dtype)};
    const Mat outs[] = {mat(s, d.rows, d.cols, d.ld_s, d.dtype), mat(pre ? x : nullptr, d.rows, d.cols, d.ld_x, d.dtype)};
    const Mat pars[] = {mat(post ? post_w : nullptr, 1, d.cols, 0, d.param_dtype),
                        mat(pre ? pre_w : nullptr, 1, d.cols, 0, d.param_dtype),
                        mat(d.gate_rows ? gate : nullptr, d.gate_rows, d.cols, 0, d.param_dtype)};
    if (!ins[0].ok() || !ins[1].ok() || !outs[0].ok() || (pre && !outs[1].ok())) return AR_ERR_ARG;
    if (d.gate_rows && !gate) return AR_ERR_ARG;
    for (const Mat &p : pars)
        if (!p.aligned()) return AR_ERR_ARG;
    rc = check_outputs(outs, 2, ins, 2, pars, 3);
    if (rc != AR_OK) return rc;
    NormArgs a{};
    a.y = y, a.residual = residual, a.post_w = post_w, a.gate = d.gate_rows ? gate : nullptr, a.pre_w = pre ? pre_w : nullptr;
    a.s = s, a.x = pre ? x : s;
    a.rows = d.rows, a.rows_per_gate = rows_per_gate(d);
    a.ld_y = ins[0].ld, a.ld_r = ins[1].ld, a.ld_s = outs[0].ld, a.ld_x = outs[1].ld;
    a.cols = (uint32_t)d.cols, a.flags = d.flags, a.alpha = d.alpha, a.eps = d.eps;
    hipStream_t st = (hipStream_t)stream;
    if (d.dtype == AR_FLOAT32)
        return d.param_dtype == AR_FLOAT32 ? launch_norm<float, float>(d, a, st) : launch_norm<float, bf16>(d, a, st);
    return d.param_dtype == AR_FLOAT32 ? launch_norm<bf16, float>(d, a, st) : launch_norm<bf16, bf16>(d, a, st);
}

int norm_backward(const ar_norm_desc *desc, const void *y, const void *s, const void *ds, const void *dx,
                  const void *post_w, const void *gate, const void *pre_w, void *dy, void *dr, void *dpost, void *dgate,
                  void *dpre, void *ws, size_t ws_bytes, void *stream)
{
    int rc = check_norm(desc);
    if (rc != AR_OK) return rc;
    const ar_norm_desc &d = *desc;
    const bool post = d.flags & AR_NORM_POST, pre = d.flags & AR_NORM_PRE;
    hipStream_t st = (hipStream_t)stream;
    if ((dpost && !post) || (dpre && !pre) || (dgate && !d.gate_rows)) return AR_ERR_ARG;
    const Mat ins[] = {mat(y, d.rows, d.cols, d.ld_y, d.dtype), mat(s, d.rows, d.cols, d.ld_s, d.dtype),
                       mat(ds, d.rows, d.cols, d.ld_ds, d.dtype), mat(pre ? dx : nullptr, d.rows, d.cols, d.ld_dx, d.dtype)};
    const Mat outs[] = {mat(dy, d.rows, d.cols, d.ld_dy, d.dtype), mat(dr, d.rows, d.cols, d.ld_residual, d.dtype),
                        mat(dpost, 1, d.cols, 0, d.param_dtype), mat(dpre, 1, d.cols, 0, d.param_dtype),
                        mat(dgate, d.gate_rows, d.cols, 0, d.param_dtype)};
    const Mat pars[] = {mat(post ? post_w : nullptr, 1, d.cols, 0, d.param_dtype),
                        mat(pre ? pre_w : nullptr, 1, d.cols, 0, d.param_dtype),
                        mat(d.gate_rows ? gate : nullptr, d.gate_rows, d.cols, 0, d.param_dtype)};
    for (const Mat &m : pars)
        if (!m.aligned()) return AR_ERR_ARG;
    for (const Mat &m : outs)
        if (!m.aligned()) return AR_ERR_ARG;
    if (d.rows == 0) {
        // sums over no rows
        for (const Mat &m : {outs[2], outs[3], outs[4]}) {
            rc = d.param_dtype == AR_FLOAT32 ? zero_param<float>((void *)m.p, m.rows * m.cols, st)
                                             : zero_param<bf16>((void *)m.p, m.rows * m.cols, st);
            if (rc != AR_OK) return rc;
        }
        return AR_OK;
    }
    if (!ins[0].ok() || !ins[1].ok() || !ins[2].aligned() || (pre && !ins[3].ok()) || !outs[0].ok() || !outs[1].ok())
        return AR_ERR_ARG;
    if (d.gate_rows && !gate) return AR_ERR_ARG;
    rc = check_outputs(outs, 5, ins, 4, pars, 3);
    if (rc != AR_OK) return rc;
    for (int i = 2; i < 5; ++i)  // sums over rows cannot take an input's place
        for (const Mat &m : ins)
            if (meet(outs[i], m)) return AR_ERR_ARG;
    NormBwdArgs a{};
    a.want = (dpost ? kWantPost : 0) | (dpre ? kWantPre : 0) | (dgate ? kWantGate : 0);
    const uint32_t groups = backward_groups(d);
    if (a.want) {
        if (!ws || ws_bytes < ar_residual_norm_backward_workspace(desc)) return AR_ERR_SCRATCH;
        if ((uintptr_t)ws % 256 != 0) return AR_ERR_ARG;
        const Mat wsm{ws, 1, ws_bytes, ws_bytes, 1};
        for (const Mat &m : ins)
            if (meet(wsm, m)) return AR_ERR_ARG;
        for (const Mat &m : outs)
            if (meet(wsm, m)) return AR_ERR_ARG;
        for (const Mat &m : pars)
            if (meet(wsm, m)) return AR_ERR_ARG;
    }
    a.y = y, a.s = s, a.ds = ds ? ds : s, a.dx = pre ? dx : s, a.has_ds = ds != nullptr;
    a.post_w = post_w, a.gate = d.gate_rows ? gate : nullptr, a.pre_w = pre ? pre_w : nullptr;
    a.dy = dy, a.dr = dr, a.dgate = dgate, a.part = (float *)ws;
    a.rows = d.rows, a.rows_per_gate = rows_per_gate(d);
    a.ld_y = ins[0].ld, a.ld_s = ins[1].ld, a.ld_ds = ds ? ins[2].ld : ins[1].ld, a.ld_dx = pre ? ins[3].ld : ins[1].ld, a.ld_dy = outs[0].ld, a.ld_dr = outs[1].ld;
    a.cols = (uint32_t)d.cols, a.flags = d.flags, a.alpha = d.alpha, a.eps = d.eps;
    if (d.dtype == AR_FLOAT32)
        rc = d.param_dtype == AR_FLOAT32 ? launch_norm_bwd<float, float>(d, a, groups, st)
                                         : launch_norm_bwd<float, bf16>(d, a, groups, st);
    else
        rc = d.param_dtype == AR_FLOAT32 ? launch_norm_bwd<bf16, float>(d, a, groups, st)
                                         : launch_norm_bwd<bf16, bf16>(d, a, groups, st);
    if (rc != AR_OK || !a.want) return rc;
    FinishArgs f{};
    f.part = (const float *)ws, f.dpost = dpost, f.dpre = dpre, f.dgate = dgate;
    f.rows = d.rows, f.rows_per_gate = a.rows_per_gate, f.gate_rows = d.gate_rows, f.cols = a.cols, f.groups = groups;
    const uint32_t gates = dgate ? (uint32_t)(d.gate_rows < groups ? d.gate_rows : groups) : 0;
    const dim3 grid((a.cols + 63) / 64, 2 + gates);
    if (d.param_dtype == AR_FLOAT32) hipLaunchKernelGGL((norm_finish_kernel<float>), grid, dim3(64 * kFinishWaves), 0, st, f);
    else hipLaunchKernelGGL((norm_finish_kernel<bf16>), grid, dim3(64 * kFinishWaves), 0, st, f);
    return launch_status();
}

}  // namespace
}  // namespace ar

extern "C" int ar_residual_norm(const ar_norm_desc *desc, const void *y, const void *residual, const void *post_weight,
                                const void *gate, const void *pre_weight, void *s, void *x, void *stream)
{
    return ar::ops_ret(ar::norm(desc, y, residual, post_weight, gate, pre_weight, s, x, stream));
}

extern "C" int ar_residual_norm_backward(const ar_norm_desc *desc, const void *y, const void *s, const void *ds,
                                         const void *dx, const void *post_weight, const void *gate,
                                         const void *pre_weight, void *dy, void *dresidual, void *dpost_weight,
                                         void *dgate, void *dpre_weight, void *workspace, size_t workspace_bytes,
                                         void *stream)
{
    return ar::ops_ret(ar::norm_backward(desc, y, s, ds, dx, post_weight, gate, pre_weight, dy, dresidual, dpost_weight,
                                         dgate, dpre_weight, workspace, workspace_bytes, stream));
}

extern "C" size_t ar_residual_norm_backward_workspace(const ar_norm_desc *desc)
{
    if (ar::check_norm(desc) != AR_OK) return 0;
    return ar::backward_groups(*desc) * (size_t)ar::dev::kParts * desc->cols * sizeof(float);
}
