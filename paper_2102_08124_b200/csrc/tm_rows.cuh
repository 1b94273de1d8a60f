// Rows of a matrix as vectors, and reductions over the threads that share a row: what the operators of the training step
// (layer norm, largest logits, distillation) have in common.
#pragma once
#include <cmath>
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "tm_device.cuh"

namespace tmask {

// DT = kF32 or kBF16: storage type, element size, elements of a 16-byte vector
template <int DT> struct RowType;
template <> struct RowType<kF32> { using T = float; static constexpr int kBytes = 4, kVec = 4; };
template <> struct RowType<kBF16> { using T = __nv_bfloat16; static constexpr int kBytes = 2, kVec = 8; };

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void from_float(float* p, float v) { *p = v; }
__device__ __forceinline__ void from_float(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// two fp32 numbers rounded to bf16 (nearest even) in one word, the first in the low half
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return reinterpret_cast<const uint32_t&>(h);
}

// 32-bit words of storage <-> fp32 values
template <int DT, int WORDS> __device__ __forceinline__ void unpack_words(const uint32_t (&w)[WORDS], float* v) {
#pragma unroll
    for (int i = 0; i < WORDS; ++i) {
        if constexpr (DT == kF32) v[i] = __uint_as_float(w[i]);
        else { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
    }
}
template <int DT, int WORDS> __device__ __forceinline__ void pack_words(const float* v, uint32_t (&w)[WORDS]) {
#pragma unroll
    for (int i = 0; i < WORDS; ++i) {
        if constexpr (DT == kF32) w[i] = __float_as_uint(v[i]);
        else w[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
    }
}

// A row seen as 16-byte vectors that start on 16-byte boundaries: vector 0 begins `lead` elements before the row.  Only the
// first and the last vector can reach past the row; they are accessed one element at a time, so that nothing outside the
// row is touched whatever its alignment.
template <int DT> struct RowVectors {
    using T = typename RowType<DT>::T;
    static constexpr int V = RowType<DT>::kVec;
    const T* base;      // element of column 0
    long long n;        // columns
    int lead;           // elements between the 16-byte boundary at or before column 0 and column 0
    long long count;    // vectors
    __device__ __forceinline__ RowVectors(const void* row, long long cols) : base(static_cast<const T*>(row)), n(cols) {
        lead = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
        count = cols > 0 ? (cols + lead + V - 1) / V : 0;
    }
    __device__ __forceinline__ long long column(long long i) const { return i * V - lead; }      // of the vector's first element; may be negative
    __device__ __forceinline__ bool full(long long i) const { return column(i) >= 0 && column(i) + V <= n; }
    __device__ __forceinline__ void load(long long i, float* v, float fill) const {
        const long long c = column(i);
        if (full(i)) {
            const uint4 u = *reinterpret_cast<const uint4*>(base + c);
            const uint32_t w[4] = {u.x, u.y, u.z, u.w};
            unpack_words<DT, 4>(w, v);
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = (c + j >= 0 && c + j < n) ? to_float(base[c + j]) : fill;
        }
    }
    // stores the vector to another row of the same length; `aligned`: that row starts at the same distance from a boundary
    __device__ __forceinline__ void store(void* row, bool aligned, long long i, const float* v) const {
        T* out = static_cast<T*>(row);
        const long long c = column(i);
        if (aligned && full(i)) {
            uint32_t w[4];
            pack_words<DT, 4>(v, w);
            *reinterpret_cast<uint4*>(out + c) = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (c + j >= 0 && c + j < n) from_float(out + c + j, v[j]);
        }
    }
};

// 2^x, flushed to zero below the normal range: one instruction, relative error below 2^-22
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

template <int WIDTH> __device__ __forceinline__ float group_sum(float v) {
#pragma unroll
    for (int o = WIDTH / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o, WIDTH);
    return v;
}
template <int WIDTH> __device__ __forceinline__ float group_max(float v) {
#pragma unroll
    for (int o = WIDTH / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, o, WIDTH));
    return v;
}

// Sum over the TPR threads of a row (a power of two; the CTA holds one row where TPR > 32).  `buf` holds TPR / 32 floats, and
// two calls in a row use different ones: the barrier of the second keeps the first one's readers apart from its next writer.
template <int TPR> __device__ __forceinline__ float row_sum(float v, float* buf) {
    if constexpr (TPR <= 32) return group_sum<TPR>(v);
    else {
        v = group_sum<32>(v);
        if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = v;
        __syncthreads();
        const float t = (threadIdx.x & 31) < TPR / 32 ? buf[threadIdx.x & 31] : 0.0f;
        return group_sum<32>(t);
    }
}

}  // namespace tmask
