// Layer normalisation with an optional residual sum, forward and backward.
//
//   forward    h = x (+ residual);  mu = mean_c h;  r = (mean_c (h - mu)^2 + eps)^(-1/2);  y = (h - mu) r w + b
//   backward   g = dy w;  xh = (h - mu) r;  dx = r (g - mean_c g - xh mean_c (g xh)) (+ dsum);
//              dw = sum_rows dy xh;  db = sum_rows dy
//
// Bound: HBM (8 respectively 14 operations an element against 4 to 16 bytes).  A row is read once and stays in the registers of
// the threads that share it -- 8 or 32 threads of a warp, or a whole CTA, by its width -- between the reductions and the
// output, so nothing is read twice and the centred squares are summed after the mean is known (no difference of large
// numbers).  The normalised value uses the sum before it is rounded for sum_out: one rounding, at the end.
// A thread owns the same columns of every row, so the backward pass keeps its share of dw and db in registers over all rows
// that its CTA takes; CTAs leave one partial row each, which a second kernel adds up in a fixed order (same input, same bits).
// Rows wider than the register forms read the row again from L2 for every step (wide_* kernels).
#include <algorithm>

#include "tm_launch.h"
#include "tm_rows.cuh"

namespace tmask {

namespace {

// VB consecutive bytes of a row as one access, kept as stored until used
template <int DT, int VB> struct Access {
    static constexpr int kElems = VB / RowType<DT>::kBytes;
    static constexpr int kWords = VB >= 4 ? VB / 4 : 1;
    uint32_t w[kWords];
    __device__ __forceinline__ void load(const void* p) {
        if constexpr (VB == 16) {
            const uint4 u = *static_cast<const uint4*>(p);
            w[0] = u.x; w[1] = u.y; w[2] = u.z; w[3] = u.w;
        } else if constexpr (VB == 4) w[0] = *static_cast<const uint32_t*>(p);
        else w[0] = *static_cast<const uint16_t*>(p);
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = 0u;
    }
    __device__ __forceinline__ float get(int j) const {
        if constexpr (DT == kF32) return __uint_as_float(w[j]);
        else return (j & 1) ? __uint_as_float(w[j >> 1] & 0xFFFF0000u) : __uint_as_float(w[j >> 1] << 16);
    }
    static __device__ __forceinline__ void store(void* p, const float* v) {
        if constexpr (VB == 2) *static_cast<__nv_bfloat16*>(p) = __float2bfloat16_rn(v[0]);
        else {
            uint32_t o[kWords];
            pack_words<DT, kWords>(v, o);
            if constexpr (VB == 16) *static_cast<uint4*>(p) = make_uint4(o[0], o[1], o[2], o[3]);
            else *static_cast<uint32_t*>(p) = o[0];
        }
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

// TPR threads share a row, E elements each in accesses of VB bytes; access i of thread t starts at column (i TPR + t) VB / size
template <int DT, int VB, int TPR, int E>
__global__ void __launch_bounds__(TPR <= 32 ? 128 : TPR) norm_forward_kernel(const NormArgs a) {
    using A = Access<DT, VB>;
    constexpr int VE = A::kElems, NV = E / VE, kThreads = TPR <= 32 ? 128 : TPR, kGroups = kThreads / TPR;
    __shared__ float buf[2][32];
    const int t = threadIdx.x % TPR, g = threadIdx.x / TPR;
    const float inv_n = 1.0f / (float)a.cols;
    for (long long r0 = (long long)blockIdx.x * kGroups; r0 < a.rows; r0 += (long long)gridDim.x * kGroups) {
        const long long r = r0 + g;
        const bool on = r < a.rows;                       // whole groups idle together, but take part in the shuffles
        float h[E];
        {
            A x[NV];
            const auto* xr = row_of<DT>(a.x, a.ld_x, on ? r : 0);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const long long c = (long long)(i * TPR + t) * VE;
                if (on && c < a.cols) x[i].load(xr + c); else x[i].clear();
            }
            if (a.residual) {
                A s[NV];
                const auto* sr = row_of<DT>(a.residual, a.ld_residual, on ? r : 0);
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const long long c = (long long)(i * TPR + t) * VE;
                    if (on && c < a.cols) s[i].load(sr + c); else s[i].clear();
                }
#pragma unroll
                for (int k = 0; k < E; ++k) h[k] = x[k / VE].get(k % VE) + s[k / VE].get(k % VE);
            } else {
#pragma unroll
                for (int k = 0; k < E; ++k) h[k] = x[k / VE].get(k % VE);
            }
        }
        float sum = 0.0f;
#pragma unroll
        for (int k = 0; k < E; ++k) sum += h[k];
        const float mean = row_sum<TPR>(sum, buf[0]) * inv_n;
        float sq = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if ((long long)(i * TPR + t) * VE < a.cols) {
#pragma unroll
                for (int j = 0; j < VE; ++j) { const float d = h[i * VE + j] - mean; sq = fmaf(d, d, sq); }
            }
        }
        const float rstd = rsqrtf(row_sum<TPR>(sq, buf[1]) * inv_n + a.eps);
        if (!on) continue;
        if (t == 0) {
            if (a.mean) a.mean[r] = mean;
            if (a.rstd) a.rstd[r] = rstd;
        }
        auto* yr = row_of<DT>(a.y, a.ld_y, r);
        auto* hr = a.sum ? row_of<DT>(a.sum, a.ld_sum, r) : nullptr;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const long long c = (long long)(i * TPR + t) * VE;
            if (c < a.cols) {
                float w[VE], b[VE], o[VE];
                load_params<VE>(a.weight, a.weight_f32, a.weight_vec, c, w, 1.0f);
                load_params<VE>(a.bias, a.weight_f32, a.bias_vec, c, b, 0.0f);
#pragma unroll
                for (int j = 0; j < VE; ++j) o[j] = fmaf((h[i * VE + j] - mean) * rstd, w[j], b[j]);
                A::store(yr + c, o);
                if (hr) A::store(hr + c, h + i * VE);
            }
        }
    }
}

// One CTA a row, the row read three times (twice from L2): rows wider than the register form
template <int DT> __global__ void __launch_bounds__(1024) wide_norm_forward_kernel(const NormArgs a) {
    __shared__ float buf[2][32];
    const float inv_n = 1.0f / (float)a.cols;
    for (long long r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const auto* xr = row_of<DT>(a.x, a.ld_x, r);
        const auto* sr = a.residual ? row_of<DT>(a.residual, a.ld_residual, r) : nullptr;
        auto* yr = row_of<DT>(a.y, a.ld_y, r);
        auto* hr = a.sum ? row_of<DT>(a.sum, a.ld_sum, r) : nullptr;
        auto value = [&](long long c) { float v = to_float(xr[c]); if (sr) v += to_float(sr[c]); return v; };
        float sum = 0.0f, sq = 0.0f;
        for (long long c = threadIdx.x; c < a.cols; c += 1024) sum += value(c);
        const float mean = row_sum<1024>(sum, buf[0]) * inv_n;
        for (long long c = threadIdx.x; c < a.cols; c += 1024) { const float d = value(c) - mean; sq = fmaf(d, d, sq); }
        const float rstd = rsqrtf(row_sum<1024>(sq, buf[1]) * inv_n + a.eps);
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[r] = mean;
            if (a.rstd) a.rstd[r] = rstd;
        }
        for (long long c = threadIdx.x; c < a.cols; c += 1024) {
            float w, b;
            load_params<1>(a.weight, a.weight_f32, false, c, &w, 1.0f);
            load_params<1>(a.bias, a.weight_f32, false, c, &b, 0.0f);
            const float h = value(c);
            from_float(yr + c, fmaf((h - mean) * rstd, w, b));
            if (hr) from_float(hr + c, h);
        }
    }
}

template <int DT, int VB, int TPR, int E>
__global__ void __launch_bounds__(TPR <= 32 ? 128 : TPR) norm_backward_kernel(const NormBackArgs a) {
    using A = Access<DT, VB>;
    constexpr int VE = A::kElems, NV = E / VE, kThreads = TPR <= 32 ? 128 : TPR, kGroups = kThreads / TPR;
    __shared__ float buf[4][32];
    extern __shared__ float fold[];                       // kGroups > 1: [2][cols]
    const int t = threadIdx.x % TPR, g = threadIdx.x / TPR;
    const float inv_n = 1.0f / (float)a.cols;
    float dw[E], db[E];
#pragma unroll
    for (int k = 0; k < E; ++k) dw[k] = db[k] = 0.0f;
    int turn = 0;
    for (long long r0 = (long long)blockIdx.x * kGroups; r0 < a.rows; r0 += (long long)gridDim.x * kGroups, turn ^= 2) {
        const long long r = r0 + g;
        const bool on = r < a.rows;
        const long long rr = on ? r : 0;
        A dy[NV], h[NV];
        const auto* dyr = row_of<DT>(a.dy, a.ld_dy, rr);
        const auto* hr = row_of<DT>(a.h, a.ld_h, rr);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const long long c = (long long)(i * TPR + t) * VE;
            if (on && c < a.cols) { dy[i].load(dyr + c); h[i].load(hr + c); } else { dy[i].clear(); h[i].clear(); }
        }
        const float mean = a.mean[rr], rstd = a.rstd[rr];
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const long long c = (long long)(i * TPR + t) * VE;
            if (on && c < a.cols) {
                float w[VE];
                load_params<VE>(a.weight, a.weight_f32, a.weight_vec, c, w, 1.0f);
#pragma unroll
                for (int j = 0; j < VE; ++j) {
                    const float d = dy[i].get(j), xh = (h[i].get(j) - mean) * rstd, u = d * w[j];
                    s1 += u;
                    s2 = fmaf(u, xh, s2);
                    dw[i * VE + j] = fmaf(d, xh, dw[i * VE + j]);
                    db[i * VE + j] += d;
                }
            }
        }
        s1 = row_sum<TPR>(s1, buf[turn]) * inv_n;
        s2 = row_sum<TPR>(s2, buf[turn + 1]) * inv_n;
        if (!on) continue;
        auto* dxr = row_of<DT>(a.dx, a.ld_dx, r);
        const auto* er = a.dsum ? row_of<DT>(a.dsum, a.ld_dsum, r) : nullptr;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const long long c = (long long)(i * TPR + t) * VE;
            if (c < a.cols) {
                float w[VE], o[VE];
                load_params<VE>(a.weight, a.weight_f32, a.weight_vec, c, w, 1.0f);
                A e;
                if (er) e.load(er + c); else e.clear();
#pragma unroll
                for (int j = 0; j < VE; ++j) {
                    const float xh = (h[i].get(j) - mean) * rstd;
                    o[j] = fmaf(rstd, dy[i].get(j) * w[j] - s1 - xh * s2, e.get(j));
                }
                A::store(dxr + c, o);
            }
        }
    }
    if (!a.partials) return;
    float* out = a.partials + (long long)blockIdx.x * 2 * a.cols;
    if constexpr (kGroups > 1) {
        // the groups add their columns one after the other
        for (int k = 0; k < kGroups; ++k) {
            if (g == k) {
#pragma unroll
                for (int i = 0; i < NV; ++i)
#pragma unroll
                    for (int j = 0; j < VE; ++j) {
                        const long long c = (long long)(i * TPR + t) * VE + j;
                        if (c < a.cols) {
                            fold[c] = dw[i * VE + j] + (k ? fold[c] : 0.0f);
                            fold[a.cols + c] = db[i * VE + j] + (k ? fold[a.cols + c] : 0.0f);
                        }
                    }
            }
            __syncthreads();
        }
        for (long long c = threadIdx.x; c < 2 * a.cols; c += kThreads) out[c] = fold[c];
    } else {
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < VE; ++j) {
                const long long c = (long long)(i * TPR + t) * VE + j;
                if (c < a.cols) { out[c] = dw[i * VE + j]; out[a.cols + c] = db[i * VE + j]; }
            }
    }
}

template <int DT> __global__ void __launch_bounds__(1024) wide_norm_backward_kernel(const NormBackArgs a) {
    __shared__ float buf[4][32];
    const float inv_n = 1.0f / (float)a.cols;
    int turn = 0;
    for (long long r = blockIdx.x; r < a.rows; r += gridDim.x, turn ^= 2) {
        const auto* dyr = row_of<DT>(a.dy, a.ld_dy, r);
        const auto* hr = row_of<DT>(a.h, a.ld_h, r);
        const auto* er = a.dsum ? row_of<DT>(a.dsum, a.ld_dsum, r) : nullptr;
        auto* dxr = row_of<DT>(a.dx, a.ld_dx, r);
        const float mean = a.mean[r], rstd = a.rstd[r];
        float s1 = 0.0f, s2 = 0.0f;
        for (long long c = threadIdx.x; c < a.cols; c += 1024) {
            float w;
            load_params<1>(a.weight, a.weight_f32, false, c, &w, 1.0f);
            const float u = to_float(dyr[c]) * w;
            s1 += u;
            s2 = fmaf(u, (to_float(hr[c]) - mean) * rstd, s2);
        }
        s1 = row_sum<1024>(s1, buf[turn]) * inv_n;
        s2 = row_sum<1024>(s2, buf[turn + 1]) * inv_n;
        for (long long c = threadIdx.x; c < a.cols; c += 1024) {
            float w;
            load_params<1>(a.weight, a.weight_f32, false, c, &w, 1.0f);
            const float xh = (to_float(hr[c]) - mean) * rstd;
            from_float(dxr + c, fmaf(rstd, to_float(dyr[c]) * w - s1 - xh * s2, er ? to_float(er[c]) : 0.0f));
        }
    }
}
// a thread a column, every gridDim.y-th row: partial row blockIdx.y.  Runs before dx is written: dx may lie on dy or h.
template <int DT> __global__ void __launch_bounds__(128) wide_norm_columns_kernel(const NormBackArgs a) {
    const long long c = (long long)blockIdx.x * 128 + threadIdx.x;
    if (c >= a.cols) return;
    float dw = 0.0f, db = 0.0f;
    for (long long r = blockIdx.y; r < a.rows; r += gridDim.y) {
        const float d = to_float(row_of<DT>(a.dy, a.ld_dy, r)[c]);
        dw = fmaf(d, (to_float(row_of<DT>(a.h, a.ld_h, r)[c]) - a.mean[r]) * a.rstd[r], dw);
        db += d;
    }
    float* out = a.partials + (long long)blockIdx.y * 2 * a.cols;
    out[c] = dw;
    out[a.cols + c] = db;
}

// Adds up `n` partial rows of 2 cols entries: 32 columns a CTA, 16 warps share the rows, always in the same order.
constexpr int kFoldWarps = 16;
__global__ void __launch_bounds__(32 * kFoldWarps) norm_fold_kernel(const float* partials, int n, long long cols, void* dweight, void* dbias, int weight_f32) {
    __shared__ float s[kFoldWarps][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long c = (long long)blockIdx.x * 32 + lane;
    cudaGridDependencySynchronize();
    float v = 0.0f;
    if (c < 2 * cols)
        for (int k = warp; k < n; k += kFoldWarps) v += partials[(long long)k * 2 * cols + c];
    s[warp][lane] = v;
    __syncthreads();
    if (warp || c >= 2 * cols) return;
#pragma unroll
    for (int k = 1; k < kFoldWarps; ++k) v += s[k][lane];
    void* out = c < cols ? dweight : dbias;
    const long long at = c < cols ? c : c - cols;
    if (!out) return;
    if (weight_f32) static_cast<float*>(out)[at] = v;
    else static_cast<__nv_bfloat16*>(out)[at] = __float2bfloat16_rn(v);
}

// CTAs that fill the device with this kernel, asked once per device and kernel
struct PerDeviceFill {
    std::atomic<int> per_sm[64];
    template <class K> int ctas(K kernel, int threads, size_t smem, int sms) {
        int dev = 0;
        if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return sms; }
        int n = per_sm[dev & 63].load(std::memory_order_relaxed);
        if (n == 0) {
            if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, threads, smem) != cudaSuccess || n < 1) { cudaGetLastError(); n = 1; }
            per_sm[dev & 63].store(n, std::memory_order_relaxed);
        }
        return n * sms;
    }
};

template <int DT, int VB, int TPR, int E> cudaError_t forward(const NormArgs& a, int sms, cudaStream_t stream) {
    constexpr int kThreads = TPR <= 32 ? 128 : TPR, kGroups = kThreads / TPR;
    static PerDeviceFill fill;
    const long long want = (a.rows + kGroups - 1) / kGroups;
    const int cap = fill.ctas(norm_forward_kernel<DT, VB, TPR, E>, kThreads, 0, sms);
    norm_forward_kernel<DT, VB, TPR, E><<<(unsigned)std::min<long long>(want, cap), kThreads, 0, stream>>>(a);
    return cudaGetLastError();
}

template <int DT, int VB, int TPR, int E> cudaError_t backward(const NormBackArgs& a, int slots, int sms, int* used, cudaStream_t stream) {
    constexpr int kThreads = TPR <= 32 ? 128 : TPR, kGroups = kThreads / TPR;
    static PerDeviceFill fill;
    const size_t smem = kGroups > 1 && a.partials ? 2 * sizeof(float) * (size_t)a.cols : 0;      // at most 8 KB: these rows have 1024 columns or fewer
    const long long want = (a.rows + kGroups - 1) / kGroups;
    const int cap = std::min(fill.ctas(norm_backward_kernel<DT, VB, TPR, E>, kThreads, kGroups > 1 ? (size_t)TPR * E * 8 : 0, sms), slots);
    *used = (int)std::min<long long>(want, cap);
    norm_backward_kernel<DT, VB, TPR, E><<<(unsigned)*used, kThreads, smem, stream>>>(a);
    return cudaGetLastError();
}

// the form for a row of `cols` elements: threads that share it, elements of each
template <int DT, int VB> cudaError_t forward_by_width(const NormArgs& a, int sms, cudaStream_t stream) {
    if (a.cols <= 64) return forward<DT, VB, 8, 8>(a, sms, stream);
    if (a.cols <= 256) return forward<DT, VB, 32, 8>(a, sms, stream);
    if (a.cols <= 1024) return forward<DT, VB, 32, 32>(a, sms, stream);
    if (a.cols <= 2048) return forward<DT, VB, 128, 16>(a, sms, stream);
    if (a.cols <= 4096) return forward<DT, VB, 256, 16>(a, sms, stream);
    if (a.cols <= 8192) return forward<DT, VB, 512, 16>(a, sms, stream);
    return forward<DT, VB, 1024, 16>(a, sms, stream);
}
template <int DT, int VB> cudaError_t backward_by_width(const NormBackArgs& a, int slots, int sms, int* used, cudaStream_t stream) {
    if (a.cols <= 64) return backward<DT, VB, 8, 8>(a, slots, sms, used, stream);
    if (a.cols <= 256) return backward<DT, VB, 32, 8>(a, slots, sms, used, stream);
    if (a.cols <= 1024) return backward<DT, VB, 32, 32>(a, slots, sms, used, stream);
    if (a.cols <= 2048) return backward<DT, VB, 128, 16>(a, slots, sms, used, stream);
    if (a.cols <= 4096) return backward<DT, VB, 256, 16>(a, slots, sms, used, stream);
    return backward<DT, VB, 512, 16>(a, slots, sms, used, stream);
}

bool aligned(const void* p, long long ld, int elem, int bytes) {
    return !p || ((uintptr_t)p % bytes == 0 && (ld * elem) % bytes == 0);
}

}  // namespace

constexpr long long kForwardWidth = 16384, kBackwardWidth = 8192;

int norm_partial_rows(long long rows, long long cols) {
    const long long cap = cols <= 2048 ? 1184 : (cols <= 65536 ? 296 : 64);
    return (int)std::max<long long>(1, std::min(rows, cap));
}

cudaError_t launch_norm_forward(NormArgs a, int dtype, int sms, cudaStream_t stream) {
    if (a.rows == 0 || a.cols == 0) return cudaSuccess;
    const int e = dtype == kF32 ? 4 : 2;
    a.weight_vec = (uintptr_t)a.weight % 16 == 0;
    a.bias_vec = (uintptr_t)a.bias % 16 == 0;
    if (a.cols > kForwardWidth) {
        const unsigned grid = (unsigned)std::min<long long>(a.rows, 2ll * sms);
        if (dtype == kF32) wide_norm_forward_kernel<kF32><<<grid, 1024, 0, stream>>>(a);
        else wide_norm_forward_kernel<kBF16><<<grid, 1024, 0, stream>>>(a);
        return cudaGetLastError();
    }
    auto all = [&](int bytes) {
        return (a.cols * e) % bytes == 0 && aligned(a.x, a.ld_x, e, bytes) && aligned(a.residual, a.ld_residual, e, bytes) &&
               aligned(a.sum, a.ld_sum, e, bytes) && aligned(a.y, a.ld_y, e, bytes);
    };
    if (dtype == kF32) return all(16) ? forward_by_width<kF32, 16>(a, sms, stream) : forward_by_width<kF32, 4>(a, sms, stream);
    if (all(16)) return forward_by_width<kBF16, 16>(a, sms, stream);
    return all(4) ? forward_by_width<kBF16, 4>(a, sms, stream) : forward_by_width<kBF16, 2>(a, sms, stream);
}

cudaError_t launch_norm_backward(NormBackArgs a, int dtype, void* dweight, void* dbias, int sms, cudaStream_t stream) {
    if (a.cols == 0) return cudaSuccess;
    if (!dweight && !dbias) a.partials = nullptr;
    const int e = dtype == kF32 ? 4 : 2;
    a.weight_vec = (uintptr_t)a.weight % 16 == 0;
    const int slots = norm_partial_rows(a.rows, a.cols);
    int used = 0;
    cudaError_t err = cudaSuccess;
    if (a.rows > 0 && a.cols > kBackwardWidth) {
        if (a.partials) {
            used = slots;
            const dim3 grid((unsigned)((a.cols + 127) / 128), (unsigned)used);
            if (dtype == kF32) wide_norm_columns_kernel<kF32><<<grid, 128, 0, stream>>>(a);
            else wide_norm_columns_kernel<kBF16><<<grid, 128, 0, stream>>>(a);
            if ((err = cudaGetLastError()) != cudaSuccess) return err;
        }
        const unsigned grid = (unsigned)std::min<long long>(a.rows, 2ll * sms);
        if (dtype == kF32) wide_norm_backward_kernel<kF32><<<grid, 1024, 0, stream>>>(a);
        else wide_norm_backward_kernel<kBF16><<<grid, 1024, 0, stream>>>(a);
        err = cudaGetLastError();
    } else if (a.rows > 0) {
        auto all = [&](int bytes) {
            return (a.cols * e) % bytes == 0 && aligned(a.dy, a.ld_dy, e, bytes) && aligned(a.h, a.ld_h, e, bytes) &&
                   aligned(a.dsum, a.ld_dsum, e, bytes) && aligned(a.dx, a.ld_dx, e, bytes);
        };
        if (dtype == kF32) err = all(16) ? backward_by_width<kF32, 16>(a, slots, sms, &used, stream) : backward_by_width<kF32, 4>(a, slots, sms, &used, stream);
        else if (all(16)) err = backward_by_width<kBF16, 16>(a, slots, sms, &used, stream);
        else err = all(4) ? backward_by_width<kBF16, 4>(a, slots, sms, &used, stream) : backward_by_width<kBF16, 2>(a, slots, sms, &used, stream);
    }
    if (err != cudaSuccess || (!dweight && !dbias)) return err;
    // rows == 0: nothing was launched and the sums over no rows are zeros (used == 0)
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((2 * a.cols + 31) / 32));
    cfg.blockDim = dim3(32 * kFoldWarps);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, norm_fold_kernel, (const float*)a.partials, used, a.cols, dweight, dbias, a.weight_f32);
}

}  // namespace tmask
