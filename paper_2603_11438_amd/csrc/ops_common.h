// Shared by the operators around the collectives (C ABI in ar_ops.h): host
// checks of matrices, and device loads, conversions and reductions.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stddef.h>
#include <stdint.h>

#include "ar_internal.h"
#include "ar_ops.h"
#include "once_per_device.h"

namespace ar {

// ---- host -------------------------------------------------------------------

inline int ops_ret(int code)
{
    if (code != AR_OK) set_last_error(code);
    return code;
}

inline bool known_dtype(int dt) { return dt == AR_FLOAT32 || dt == AR_BFLOAT16; }
inline size_t elem_bytes(int dt) { return dt == AR_FLOAT32 ? 4 : 2; }
inline size_t round_up(size_t a, size_t b) { return (a + b - 1) / b * b; }

// Sizes above this are refused: products of three sizes then stay far inside
// 64 bits.
constexpr size_t kOpsMaxSize = (size_t)1 << 40;

// A matrix argument as the checks see it.
struct Mat {
    const void *p;
    size_t rows, cols, ld, elem;
    size_t bytes() const { return rows && cols ? ((rows - 1) * ld + cols) * elem : 0; }
    bool aligned() const { return ((uintptr_t)p % elem) == 0; }
    bool ok() const { return p && aligned(); }
    bool same(const Mat &o) const { return p == o.p && ld == o.ld; }
};

inline Mat mat(const void *p, size_t rows, size_t cols, size_t ld, int dtype)
{
    return Mat{p, rows, cols, ld ? ld : cols, elem_bytes(dtype)};
}

// Whether two matrices may share an element.  Exact for equal row strides,
// where column ranges of one buffer interleave without meeting; otherwise the
// address ranges decide.
inline bool meet(const Mat &a, const Mat &b)
{
    if (!a.p || !b.p || !a.bytes() || !b.bytes()) return false;
    const uintptr_t pa = (uintptr_t)a.p, pb = (uintptr_t)b.p;
    if (pa >= pb + b.bytes() || pb >= pa + a.bytes()) return false;
    const size_t la = a.ld * a.elem, lb = b.ld * b.elem;
    if (la == lb) {
        const size_t d = pa >= pb ? (pa - pb) % la : (la - (pb - pa) % la) % la;  // a's column offset after b's
        if (d >= b.cols * b.elem && d + a.cols * a.elem <= la) return false;
    }
    return true;
}

// A batch of equal matrices, `stride` elements from each to the next.
struct Batch {
    Mat first;
    size_t count, stride;
    size_t bytes() const { return count ? (count - 1) * stride * first.elem + first.bytes() : 0; }
    Mat at(size_t k) const
    {
        Mat m = first;
        m.p = (const char *)m.p + k * stride * m.elem;
        return m;
    }
};

// Whether matrices of two batches, of one count, may share an element: as `meet` for
// each pair whose address ranges meet.
inline bool meet(const Batch &a, const Batch &b)
{
    if (!a.first.p || !b.first.p || !a.bytes() || !b.bytes()) return false;
    const uintptr_t pa = (uintptr_t)a.first.p, pb = (uintptr_t)b.first.p;
    if (pa >= pb + b.bytes() || pb >= pa + a.bytes()) return false;
    if (a.stride == b.stride) {
        // a pair's places beside each other depend on the difference of its indexes alone
        for (size_t k = 0; k < a.count; ++k)
            if (meet(a.at(k), b.first) || meet(a.first, b.at(k))) return true;
        return false;
    }
    size_t pairs = 0;
    const size_t step = b.stride * b.first.elem, span = b.first.bytes();
    for (size_t i = 0; i < a.count; ++i) {
        const Mat m = a.at(i);
        const uintptr_t p = (uintptr_t)m.p;
        // the matrices of b that end behind m's begin and begin before its end
        const size_t from = p >= pb + span ? (p - pb - span) / step + 1 : 0;
        for (size_t k = from; k < b.count && pb + k * step < p + m.bytes(); ++k)
            if (++pairs > (1u << 20) || meet(m, b.at(k))) return true;  // past a million pairs: the ranges decide
    }
    return false;
}

// Lets a kernel's launches on the current device have `bytes` of dynamic LDS.
inline int allow_lds(OncePerDevice &once, const void *kernel, int bytes)
{
    int device = 0;
    const bool ok = hipGetDevice(&device) == hipSuccess && once(device, [&] {
        return hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes) == hipSuccess;
    });
    return ok ? AR_OK : AR_ERR_HIP;
}

inline int launch_status() { return hipGetLastError() == hipSuccess ? AR_OK : AR_ERR_HIP; }

// ---- device -----------------------------------------------------------------

namespace dev {

typedef __bf16 bf16;
template <typename T, int N> struct VecOf;
template <> struct VecOf<float, 4> { typedef float type __attribute__((ext_vector_type(4), aligned(4))); };
template <> struct VecOf<bf16, 8> { typedef bf16 type __attribute__((ext_vector_type(8), aligned(2))); };
template <> struct VecOf<bf16, 4> { typedef bf16 type __attribute__((ext_vector_type(4), aligned(2))); };

// Rows start on any element: loads of 16 bytes need no more alignment than
// their elements on gfx950.
template <typename T, int N> __device__ __forceinline__ void load_vec(const T *p, float *out)
{
    constexpr int W = sizeof(T) == 4 ? 4 : N < 8 ? 4 : 8;
#pragma unroll
    for (int k = 0; k < N / W; ++k) {
        const auto v = *(const typename VecOf<T, W>::type *)(p + k * W);
#pragma unroll
        for (int j = 0; j < W; ++j) out[k * W + j] = (float)v[j];
    }
}

template <typename T, int N> __device__ __forceinline__ void store_vec(T *p, const float *in)
{
    constexpr int W = sizeof(T) == 4 ? 4 : N < 8 ? 4 : 8;
#pragma unroll
    for (int k = 0; k < N / W; ++k) {
        typename VecOf<T, W>::type v;
#pragma unroll
        for (int j = 0; j < W; ++j) v[j] = (T)in[k * W + j];
        *(typename VecOf<T, W>::type *)(p + k * W) = v;
    }
}

// The first `have` of N elements; the others read as zero.
template <typename T, int N> __device__ __forceinline__ void load_part(const T *p, int have, float *out)
{
#pragma unroll
    for (int j = 0; j < N; ++j) out[j] = j < have ? (float)p[j] : 0.0f;
}
template <typename T, int N> __device__ __forceinline__ void store_part(T *p, int have, const float *in)
{
#pragma unroll
    for (int j = 0; j < N; ++j)
        if (j < have) p[j] = (T)in[j];
}

// Sum over a wave, the same value in every lane.  The data-parallel-primitive
// moves stay in the vector unit: rows of 16 lanes, then the rows.
template <int CTRL, int ROWS> __device__ __forceinline__ float add_moved(float v)
{
    return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ float wave_sum(float v)
{
    v = add_moved<0x111, 0xf>(v);  // row_shr 1, 2, 4, 8
    v = add_moved<0x112, 0xf>(v);
    v = add_moved<0x114, 0xf>(v);
    v = add_moved<0x118, 0xf>(v);
    v = add_moved<0x142, 0xa>(v);  // row_bcast 15 into rows 1 and 3
    v = add_moved<0x143, 0xc>(v);  // row_bcast 31 into rows 2 and 3
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}

// Sums of K values over a workgroup of W waves, the same in every thread.  One
// barrier: successive calls take the two halves of `slots` in turn (`turn`
// counts them), so a wave that is still reading one sum's slots is not
// overtaken by the next sum's writes.
template <int W, int K> __device__ __forceinline__ void group_sum(float *v, float (*slots)[W * K], uint32_t &turn)
{
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = wave_sum(v[k]);
    if constexpr (W > 1) {
        float *s = slots[turn & 1];
        ++turn;
        const uint32_t wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63u) == 0)
#pragma unroll
            for (int k = 0; k < K; ++k) s[wave * K + k] = v[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float t = s[k];
#pragma unroll
            for (int w = 1; w < W; ++w) t += s[w * K + k];
            v[k] = t;
        }
    }
}

}  // namespace dev
}  // namespace ar
