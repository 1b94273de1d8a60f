// Rows in the registers of the threads that share them, and parameters of their columns: what the norms have in common.
#pragma once
#include <type_traits>

#include "tm_rows.cuh"

namespace tmask {

// VB bytes of a row: N elements from column c on, out of a stage or from the row itself
template <int DT, int VB> struct Access {
    using T = typename RowType<DT>::T;
    static constexpr int kElems = VB / RowType<DT>::kBytes;
    static __device__ __forceinline__ void load(const char* p, float* v) {
        if constexpr (VB == 16) unpack_vector<DT>(*reinterpret_cast<const uint4*>(p), v);
        else v[0] = to_float(*reinterpret_cast<const T*>(p));
    }
    static __device__ __forceinline__ void store(T* p, const float* v) {
        if constexpr (VB == 16) {
            uint32_t o[4];
            pack_words<DT, 4>(v, o);
            *reinterpret_cast<uint4*>(p) = make_uint4(o[0], o[1], o[2], o[3]);
        } else from_float(p, v[0]);
    }
};

// N consecutive parameters (weight, bias) from column c on; `vec`: they may be read 16 bytes at a time
template <int N> __device__ __forceinline__ void load_params(const void* p, bool f32, bool vec, long long c, float* v, float none) {
    if (!p) {
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = none;
    } else if (f32) {
        const float* q = static_cast<const float*>(p) + c;
        if (N % 4 == 0 && vec) {
#pragma unroll
            for (int j = 0; j < N; j += 4) {
                const float4 u = *reinterpret_cast<const float4*>(q + j);
                v[j] = u.x; v[j + 1] = u.y; v[j + 2] = u.z; v[j + 3] = u.w;
            }
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j) v[j] = q[j];
        }
    } else {
        const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(p) + c;
        if (N % 8 == 0 && vec) {
#pragma unroll
            for (int j = 0; j < N; j += 8) {
                const uint4 u = *reinterpret_cast<const uint4*>(q + j);
                const uint32_t w[4] = {u.x, u.y, u.z, u.w};
                unpack_words<kBF16, 4>(w, v + j);
            }
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j) v[j] = __bfloat162float(q[j]);
        }
    }
}

template <int DT> __device__ __forceinline__ const typename RowType<DT>::T* row_of(const void* p, long long ld, long long r) {
    return static_cast<const typename RowType<DT>::T*>(p) + r * ld;
}
template <int DT> __device__ __forceinline__ typename RowType<DT>::T* row_of(void* p, long long ld, long long r) {
    return static_cast<typename RowType<DT>::T*>(p) + r * ld;
}

// What TPR threads hold of a row: E elements each, in accesses of VB bytes; access i of thread t starts at column (i TPR + t) VB / size.
template <int DT, int VB, int TPR, int E> struct RowRegs {
    using A = Access<DT, VB>;
    using T = typename RowType<DT>::T;
    static constexpr int VE = A::kElems, NV = E / VE;
    static __device__ __forceinline__ int column(int i) { return (i * TPR + (int)threadIdx.x % TPR) * VE; }
    // (v, v) for elements 2k and 2k + 1, zero for those past the last column
    static __device__ __forceinline__ float2 inside(int k, int cols, float v) {
        return make_float2(column(2 * k / VE) < cols ? v : 0.0f, column((2 * k + 1) / VE) < cols ? v : 0.0f);
    }
    static __device__ __forceinline__ void load(const T* row, int cols, float2 (&v)[E / 2]) {
        float* f = reinterpret_cast<float*>(v);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = column(i);
#pragma unroll
            for (int j = 0; j < VE; ++j) f[i * VE + j] = 0.0f;
            if (c < cols) A::load(reinterpret_cast<const char*>(row + c), f + i * VE);
        }
    }
    // the same in two steps, for a row that is asked for ahead of its turn
    using Raw = std::conditional_t<VB == 16, uint4, T>;
    static __device__ __forceinline__ void ask(const T* row, int cols, Raw (&u)[NV]) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            u[i] = Raw{};
            if (column(i) < cols) u[i] = *reinterpret_cast<const Raw*>(row + column(i));
        }
    }
    static __device__ __forceinline__ void take(const Raw (&u)[NV], float2 (&v)[E / 2]) {
        float* f = reinterpret_cast<float*>(v);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if constexpr (VB == 16) unpack_vector<DT>(u[i], f + i * VE);
            else f[i] = to_float(u[i]);
        }
    }
    // brings row r of two matrices to L2, a line a thread: half the threads cover a row of E <= 16
    static __device__ __forceinline__ void fetch(const void* a, long long ld_a, const void* b, long long ld_b, long long r, long long rows, int cols) {
        const int t = threadIdx.x % TPR, c = (t & (TPR / 2 - 1)) * (128 / (int)sizeof(T));
        if (r < rows && c < cols) {
            const T* p = t < TPR / 2 ? row_of<DT>(a, ld_a, r) + c : row_of<DT>(b, ld_b, r) + c;
            asm volatile("prefetch.global.L2 [%0];" ::"l"(p));
        }
    }
    static __device__ __forceinline__ void store(T* row, int cols, const float2 (&v)[E / 2]) {
        const float* f = reinterpret_cast<const float*>(v);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = column(i);
            if (c < cols) A::store(row + c, f + i * VE);
        }
    }
    static __device__ __forceinline__ void params(const void* p, bool f32, bool vec, int cols, float2 (&v)[E / 2], float none) {
        float* f = reinterpret_cast<float*>(v);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = column(i);
#pragma unroll
            for (int j = 0; j < VE; ++j) f[i * VE + j] = 0.0f;
            if (c < cols) load_params<VE>(p, f32, vec, c, f + i * VE, none);
        }
    }
};

}  // namespace tmask
