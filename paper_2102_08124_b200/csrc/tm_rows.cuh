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
// (and a word of -Inf)
template <int DT> struct RowType;
template <> struct RowType<kF32> { using T = float; static constexpr int kBytes = 4, kVec = 4; static constexpr uint32_t kLow = 0xFF800000u; };
template <> struct RowType<kBF16> { using T = __nv_bfloat16; static constexpr int kBytes = 2, kVec = 8; static constexpr uint32_t kLow = 0xFF80FF80u; };

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

template <int DT> __device__ __forceinline__ void unpack_vector(const uint4& u, float* v) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
    unpack_words<DT, 4>(w, v);
}

// the largest of a vector's elements; NaN only where all are
template <int DT> __device__ __forceinline__ float vector_max(const uint4& u) {
    if constexpr (DT == kF32) return fmaxf(fmaxf(__uint_as_float(u.x), __uint_as_float(u.y)), fmaxf(__uint_as_float(u.z), __uint_as_float(u.w)));
    else {
        const __nv_bfloat162 m = __hmax2(__hmax2(reinterpret_cast<const __nv_bfloat162&>(u.x), reinterpret_cast<const __nv_bfloat162&>(u.y)),
                                         __hmax2(reinterpret_cast<const __nv_bfloat162&>(u.z), reinterpret_cast<const __nv_bfloat162&>(u.w)));
        const uint32_t w = reinterpret_cast<const uint32_t&>(m);
        return fmaxf(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
    }
}

// the same, NaN if any is
__device__ __forceinline__ float max_nan(float a, float b) { float m; asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(a), "f"(b)); return m; }
template <int DT> __device__ __forceinline__ float vector_max_nan(const uint4& u) {
    if constexpr (DT == kF32) return max_nan(max_nan(__uint_as_float(u.x), __uint_as_float(u.y)), max_nan(__uint_as_float(u.z), __uint_as_float(u.w)));
    else {
        const __nv_bfloat162 m = __hmax2_nan(__hmax2_nan(reinterpret_cast<const __nv_bfloat162&>(u.x), reinterpret_cast<const __nv_bfloat162&>(u.y)),
                                             __hmax2_nan(reinterpret_cast<const __nv_bfloat162&>(u.z), reinterpret_cast<const __nv_bfloat162&>(u.w)));
        const uint32_t w = reinterpret_cast<const uint32_t&>(m);
        return max_nan(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
    }
}

// A row seen as 16-byte vectors that start on 16-byte boundaries: vector 0 begins `lead` elements before the row.  Only the
// first and the last vector can reach past the row; RowPart gives their elements one at a time, so that nothing outside the row is
// touched whatever its alignment.
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
};

// The part [from, to) of a row's vectors (to <= its count) that one thread block works on: `inside` full vectors from `vec` on, at
// element `column`, and up to V - 1 elements in front of them and behind (the row's partial first and last vector, where they
// belong to this part).  Everything counts in 32 bits.
template <int DT> struct RowPart {
    using T = typename RowType<DT>::T;
    static constexpr int V = RowType<DT>::kVec;
    long long column;          // of the first full vector
    int inside, head, tail;    // vectors; elements before and after them
    __device__ __forceinline__ RowPart(const RowVectors<DT>& row, long long from, long long to) {
        const long long a = max(0ll, row.column(from)), b = min(row.n, row.column(to));
        const long long first = row.lead ? max(from, 1ll) : from, last = row.column(to) > row.n ? to - 1 : to;
        if (a >= b) { column = 0; inside = head = tail = 0; return; }
        inside = (int)max(0ll, last - first);
        column = inside > 0 ? row.column(first) : b;
        head = (int)(column - a);
        tail = inside > 0 ? (int)(b - (column + (long long)inside * V)) : 0;
    }
    // element k of the head and tail together, k < head + tail: its column
    __device__ __forceinline__ long long edge(int k) const { return k < head ? column - head + k : column + (long long)inside * V + (k - head); }
};

// Softmax sums take 2^(x - m) of scaled logits x = z log2(e) / T as fma(z, log2(e) / T, -m), m the running maximum of the rounded x.  The
// difference then holds that rounding, half a unit of m's last place: below one binade up to 2^24, but past 2^31 more than fp32's
// range.  So m starts at kFloor and what lies below it (masks, beside ordinary logits) counts as zero; a row whose largest x is not inside
// +-kReach goes again with differences of the logits themselves.
constexpr float kFloor = -16777216.0f, kReach = 8388608.0f;

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
    if constexpr (WIDTH == 32) {                          // one instruction for a whole warp
        float m;
        asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(m) : "f"(v));
        return m;
    } else {
#pragma unroll
        for (int o = WIDTH / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, o, WIDTH));
        return v;
    }
}

// Sums over the TPR threads of a row (a power of two); a block holds GROUPS = blockDim / TPR rows side by side, each with a named barrier
// of its own where TPR > 32 and GROUPS > 1 (a block that names barriers at run time takes all 16 of them, of the 64 of an SM).  `buf` holds blockDim / 32 entries, and two calls in a row use different ones: the barrier of the second
// keeps the first one's readers apart from its next writer.
template <int TPR, int GROUPS = 1> __device__ __forceinline__ void row_barrier() {
    if constexpr (TPR <= 32) __syncwarp();
    else if constexpr (GROUPS == 1) __syncthreads();
    else asm volatile("bar.sync %0, %1;" ::"r"(1 + (int)threadIdx.x / TPR), "n"(TPR) : "memory");
}
template <int TPR, int GROUPS = 1> __device__ __forceinline__ float row_sum(float v, float* buf) {
    if constexpr (TPR <= 32) return group_sum<TPR>(v);
    else {
        constexpr int W = TPR / 32;
        v = group_sum<32>(v);
        if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = v;
        row_barrier<TPR, GROUPS>();
        const float t = buf[(threadIdx.x / TPR) * W + (threadIdx.x & (W - 1))];
        return group_sum<W>(t);
    }
}
template <int TPR, int GROUPS = 1> __device__ __forceinline__ float2 row_sum2(float2 v, float2* buf) {
    if constexpr (TPR <= 32) return make_float2(group_sum<TPR>(v.x), group_sum<TPR>(v.y));
    else {
        constexpr int W = TPR / 32;
        v = make_float2(group_sum<32>(v.x), group_sum<32>(v.y));
        if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = v;
        row_barrier<TPR, GROUPS>();
        const float2 t = buf[(threadIdx.x / TPR) * W + (threadIdx.x & (W - 1))];
        return make_float2(group_sum<W>(t.x), group_sum<W>(t.y));
    }
}

// Thread-block clusters: this block's rank, a barrier among all their threads, and reads of another block's shared memory
__device__ __forceinline__ uint32_t cluster_rank() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t cluster_map(const void* shared, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"((uint32_t)__cvta_generic_to_shared(shared)), "r"(rank));
    return r;
}
__device__ __forceinline__ float2 cluster_load2(const float2* shared, uint32_t rank) {
    float2 v;
    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(cluster_map(shared, rank)) : "memory");
    return v;
}
__device__ __forceinline__ float cluster_load_float(const float* shared, uint32_t rank) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(cluster_map(shared, rank)) : "memory");
    return v;
}
__device__ __forceinline__ unsigned long long cluster_load64(const unsigned long long* shared, uint32_t rank) {
    unsigned long long v;
    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(cluster_map(shared, rank)) : "memory");
    return v;
}
__device__ __forceinline__ double cluster_load_double(const double* shared, uint32_t rank) {
    double v;
    asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(v) : "r"(cluster_map(shared, rank)) : "memory");
    return v;
}

}  // namespace tmask
