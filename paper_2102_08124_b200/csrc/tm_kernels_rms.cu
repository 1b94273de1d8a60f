// The residual branch: dropout from a counter-based generator, and the root-mean-square norm of the residual sum.
//
//   dropout    d(x)_c = x_c / (1 - p) where column c of the row stays, else 0;  y = d(x) (+ residual)
//   forward    h = d(x) (+ residual);  r = (mean_c h^2 + eps)^(-1/2);  y = h r w
//              8 bits: a scale s = max(max |y| / 448, 2^-126) for every group of columns, and y / s rounded to e4m3
//   backward   g = dy w;  xh = h r;  dh = r (g - xh mean_c (g xh)) (+ dsum);  dx = d(dh);  dw = sum_rows dy xh
//
// Which columns stay is worked out again from the seed wherever it is needed, the backward pass included.
#include <algorithm>

#include <cuda_fp8.h>

#include "tm_philox.cuh"
#include "tm_row_regs.cuh"

namespace tmask {

// Partial rows of the weight's gradient
int rms_partial_rows(long long rows, long long cols) {
    const long long cap = cols <= 4096 ? 888 : (cols <= 65536 ? 296 : 64);
    return (int)std::max<long long>(1, std::min(rows, cap));
}

namespace {

constexpr float kMostE4m3 = 448.0f, kLeastScale = 1.17549435e-38f;      // 2^-126

// Eight columns from c on (c a multiple of 8), zeros past the last
template <int DT, bool VEC> __device__ __forceinline__ void load_block(const typename RowType<DT>::T* row, long long c, long long cols, float (&v)[8]) {
    constexpr int V = RowType<DT>::kVec;
#pragma unroll
    for (int i = 0; i < 8; i += V) {
        if (VEC && c + i + V <= cols) unpack_vector<DT>(*reinterpret_cast<const uint4*>(row + c + i), v + i);
        else {
#pragma unroll
            for (int j = i; j < i + V; ++j) v[j] = c + j < cols ? to_float(row[c + j]) : 0.0f;
        }
    }
}
template <int DT, bool VEC> __device__ __forceinline__ void store_block(typename RowType<DT>::T* row, long long c, long long cols, const float (&v)[8]) {
    constexpr int V = RowType<DT>::kVec;
#pragma unroll
    for (int i = 0; i < 8; i += V) {
        if (VEC && c + i + V <= cols) {
            uint32_t o[4];
            pack_words<DT, 4>(v + i, o);
            *reinterpret_cast<uint4*>(row + c + i) = make_uint4(o[0], o[1], o[2], o[3]);
        } else {
#pragma unroll
            for (int j = i; j < i + V; ++j) if (c + j < cols) from_float(row + c + j, v[j]);
        }
    }
}
// their weights, ones where there are none
__device__ __forceinline__ void load_weights(const void* w, bool f32, bool vec, long long c, long long cols, float (&v)[8]) {
    if (c + 8 <= cols) load_params<8>(w, f32, vec, c, v, 1.0f);
    else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            v[j] = 1.0f;
            if (c + j < cols) load_params<1>(w, f32, false, c + j, v + j, 1.0f);
        }
    }
}
__device__ __forceinline__ void drop_block(const PhiloxKey& key, const DropSpec& d, long long r, long long c, float (&v)[8]) {
    const uint32_t kept = kept_bits(key((uint32_t)(c >> 3), (uint32_t)r), d.limit);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (kept >> j) & 1u ? v[j] * d.scale : 0.0f;      // a dropped Inf or NaN is gone
}

// four values in e4m3, the first in the low byte; beyond +-448 that value, NaN stays NaN
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
    uint16_t lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
    return (uint32_t)lo | (uint32_t)hi << 16;
}
__device__ __forceinline__ void store_e4m3(uint8_t* row, long long c, long long cols, const float (&v)[8], float inverse, bool vec) {
    float q[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) q[j] = v[j] * inverse;
    const uint32_t u[2] = {pack_e4m3(q[0], q[1], q[2], q[3]), pack_e4m3(q[4], q[5], q[6], q[7])};
    if (vec && c + 8 <= cols) *reinterpret_cast<uint2*>(row + c) = make_uint2(u[0], u[1]);
    else {
#pragma unroll
        for (int j = 0; j < 8; ++j) if (c + j < cols) row[c + j] = (uint8_t)(u[j / 4] >> (8 * (j % 4)));
    }
}
// A group's scale from its largest magnitude; NaN does not count (it stays in the values), and no scale is zero
__device__ __forceinline__ float scale_of(float most) { return fmaxf(most * (1.0f / kMostE4m3), kLeastScale); }

template <int DT, bool VEC> __global__ void __launch_bounds__(256) dropout_kernel(const DropoutArgs a) {
    const PhiloxKey key(a.drop.seed, a.drop.offset, a.drop.offset_dev);
    const long long blocks = (a.cols + 7) / 8, all = a.rows * blocks;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < all; i += (long long)gridDim.x * 256) {
        const long long r = i / blocks, c = (i - r * blocks) * 8;
        float v[8];
        load_block<DT, VEC>(row_of<DT>(a.x, a.ld_x, r), c, a.cols, v);
        if (a.drop.limit) drop_block(key, a.drop, r, c, v);
        if (a.residual) {
            float s[8];
            load_block<DT, VEC>(row_of<DT>(a.residual, a.ld_residual, r), c, a.cols, s);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += s[j];
        }
        store_block<DT, VEC>(row_of<DT>(a.y, a.ld_y, r), c, a.cols, v);
    }
}

// A block a row, the row read twice
constexpr int kWide = 512;
template <int DT, bool VEC, bool E8> __global__ void __launch_bounds__(kWide) wide_rms_forward_kernel(const RmsArgs a, bool vec8) {
    __shared__ float2 buf[2][32];
    const PhiloxKey key(a.drop.seed, a.drop.offset, a.drop.offset_dev);
    const float inv_n = 1.0f / (float)a.cols;
    const int lane = threadIdx.x & 31;
    const long long blocks = (a.cols + 7) / 8;
    int turn = 0;
    for (long long r = blockIdx.x; r < a.rows; r += gridDim.x, turn ^= 1) {
        auto sum = [&](long long c, float (&v)[8]) {
            load_block<DT, VEC>(row_of<DT>(a.x, a.ld_x, r), c, a.cols, v);
            if (a.drop.limit) drop_block(key, a.drop, r, c, v);
            if (a.residual) {
                float s[8];
                load_block<DT, VEC>(row_of<DT>(a.residual, a.ld_residual, r), c, a.cols, s);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] += s[j];
            }
        };
        float sq = 0.0f, most = 0.0f;
        for (long long b = threadIdx.x; b < blocks; b += kWide) {
            float h[8], w[8];
            sum(b * 8, h);
            if (E8) load_weights(a.weight, a.weight_f32, a.weight_vec, b * 8, a.cols, w);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                sq = fmaf(h[j], h[j], sq);
                if (E8) most = fmaxf(most, fabsf(h[j] * w[j]));
            }
        }
        float2 both = row_sum2<kWide>(make_float2(sq, 0.0f), buf[turn]);
        const float rstd = 1.0f / sqrtf(both.x * inv_n + a.eps);
        float scale = 1.0f;
        if (E8 && a.group == 0) {
            most = group_max<32>(most);
            __syncthreads();
            if (lane == 0) buf[turn][threadIdx.x >> 5].y = most;
            __syncthreads();
            most = 0.0f;
            for (int k = 0; k < kWide / 32; ++k) most = fmaxf(most, buf[turn][k].y);
            scale = scale_of(most * rstd);
            if (threadIdx.x == 0) a.scales[r] = scale;
        }
        if (threadIdx.x == 0 && a.rstd) a.rstd[r] = rstd;
        const int members = a.group / 8;
        const long long groups = a.group ? (a.cols + a.group - 1) / a.group : 1;
        for (long long b0 = 0; b0 < blocks; b0 += kWide) {
            const long long c = (b0 + threadIdx.x) * 8;
            float h[8], w[8], y[8];
            if (c < a.cols) {
                sum(c, h);
                load_weights(a.weight, a.weight_f32, a.weight_vec, c, a.cols, w);
            }
            float top = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                y[j] = c < a.cols ? h[j] * rstd * w[j] : 0.0f;
                if (E8) top = fmaxf(top, fabsf(y[j]));
            }
            if (E8 && a.group) {
                for (int o = members / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
                scale = scale_of(top);
                if (c < a.cols && threadIdx.x % members == 0) a.scales[r * groups + c / a.group] = scale;
            }
            if (c >= a.cols) continue;
            if (a.sum) store_block<DT, VEC>(row_of<DT>(a.sum, a.ld_sum, r), c, a.cols, h);
            if (E8) store_e4m3(static_cast<uint8_t*>(a.y) + r * a.ld_y, c, a.cols, y, 1.0f / scale, vec8);
            else store_block<DT, VEC>(row_of<DT>(a.y, a.ld_y, r), c, a.cols, y);
        }
        __syncthreads();
    }
}

template <int DT, bool VEC> __global__ void __launch_bounds__(kWide) wide_rms_backward_kernel(const RmsBackArgs a) {
    __shared__ float buf[2][32];
    const PhiloxKey key(a.drop.seed, a.drop.offset, a.drop.offset_dev);
    const float inv_n = 1.0f / (float)a.cols;
    const long long blocks = (a.cols + 7) / 8;
    int turn = 0;
    for (long long r = blockIdx.x; r < a.rows; r += gridDim.x, turn ^= 1) {
        const float rstd = a.rstd[r];
        float dot = 0.0f;
        for (long long b = threadIdx.x; b < blocks; b += kWide) {
            float d[8], h[8], w[8];
            load_block<DT, VEC>(row_of<DT>(a.dy, a.ld_dy, r), b * 8, a.cols, d);
            load_block<DT, VEC>(row_of<DT>(a.h, a.ld_h, r), b * 8, a.cols, h);
            load_weights(a.weight, a.weight_f32, a.weight_vec, b * 8, a.cols, w);
#pragma unroll
            for (int j = 0; j < 8; ++j) dot = fmaf(d[j] * w[j], h[j] * rstd, dot);
        }
        const float mean = row_sum<kWide>(dot, buf[turn]) * inv_n;
        for (long long b = threadIdx.x; b < blocks; b += kWide) {
            const long long c = b * 8;
            float d[8], h[8], w[8], e[8];
            load_block<DT, VEC>(row_of<DT>(a.dy, a.ld_dy, r), c, a.cols, d);
            load_block<DT, VEC>(row_of<DT>(a.h, a.ld_h, r), c, a.cols, h);
            load_weights(a.weight, a.weight_f32, a.weight_vec, c, a.cols, w);
#pragma unroll
            for (int j = 0; j < 8; ++j) e[j] = 0.0f;
            if (a.dsum) load_block<DT, VEC>(row_of<DT>(a.dsum, a.ld_dsum, r), c, a.cols, e);
#pragma unroll
            for (int j = 0; j < 8; ++j) d[j] = fmaf(rstd, d[j] * w[j] - h[j] * rstd * mean, e[j]);
            if (a.dh) store_block<DT, VEC>(row_of<DT>(a.dh, a.ld_dh, r), c, a.cols, d);
            if (a.dx) {
                if (a.drop.limit) drop_block(key, a.drop, r, c, d);
                store_block<DT, VEC>(row_of<DT>(a.dx, a.ld_dx, r), c, a.cols, d);
            }
        }
    }
}
// a thread a column, every gridDim.y-th row: partial row blockIdx.y.  Runs before dh and dx are written: they may lie on dy or h.
template <int DT> __global__ void __launch_bounds__(128) wide_rms_columns_kernel(const RmsBackArgs a) {
    const long long c = (long long)blockIdx.x * 128 + threadIdx.x;
    if (c >= a.cols) return;
    float dw = 0.0f;
    for (long long r = blockIdx.y; r < a.rows; r += gridDim.y)
        dw = fmaf(to_float(row_of<DT>(a.dy, a.ld_dy, r)[c]), to_float(row_of<DT>(a.h, a.ld_h, r)[c]) * a.rstd[r], dw);
    a.partials[(long long)blockIdx.y * a.cols + c] = dw;
}

// Adds up `n` partial rows: 32 columns a block, 16 warps share the rows, always in the same order
constexpr int kFoldWarps = 16;
__global__ void __launch_bounds__(32 * kFoldWarps) rms_fold_kernel(const float* partials, int n, long long cols, void* dweight, int weight_f32) {
    __shared__ float s[kFoldWarps][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long c = (long long)blockIdx.x * 32 + lane;
    float v = 0.0f;
    if (c < cols)
#pragma unroll 8
        for (int k = warp; k < n; k += kFoldWarps) v += partials[(long long)k * cols + c];
    s[warp][lane] = v;
    __syncthreads();
    if (warp || c >= cols) return;
#pragma unroll
    for (int k = 1; k < kFoldWarps; ++k) v += s[k][lane];
    if (weight_f32) static_cast<float*>(dweight)[c] = v;
    else static_cast<__nv_bfloat16*>(dweight)[c] = __float2bfloat16_rn(v);
}

// Rows that start on 16-byte boundaries, all of them
bool aligned(const void* p, long long ld, int elem) { return !p || ((uintptr_t)p % 16 == 0 && (ld * elem) % 16 == 0); }

}  // namespace

cudaError_t launch_dropout(const DropoutArgs& a, int dtype, int sms, cudaStream_t stream) {
    if (a.rows == 0 || a.cols == 0) return cudaSuccess;
    const int e = dtype == kF32 ? 4 : 2;
    const bool vec = aligned(a.x, a.ld_x, e) && aligned(a.residual, a.ld_residual, e) && aligned(a.y, a.ld_y, e);
    const long long all = a.rows * ((a.cols + 7) / 8);
    const unsigned grid = (unsigned)std::min<long long>((all + 255) / 256, 8ll * sms);
    if (dtype == kF32) { if (vec) dropout_kernel<kF32, true><<<grid, 256, 0, stream>>>(a); else dropout_kernel<kF32, false><<<grid, 256, 0, stream>>>(a); }
    else { if (vec) dropout_kernel<kBF16, true><<<grid, 256, 0, stream>>>(a); else dropout_kernel<kBF16, false><<<grid, 256, 0, stream>>>(a); }
    return cudaGetLastError();
}

cudaError_t launch_rms_forward(RmsArgs a, int dtype, int sms, cudaStream_t stream) {
    if (a.rows == 0 || a.cols == 0) return cudaSuccess;
    const int e = dtype == kF32 ? 4 : 2;
    a.weight_vec = (uintptr_t)a.weight % 16 == 0;
    const bool e8 = a.scales != nullptr;
    const bool vec = aligned(a.x, a.ld_x, e) && aligned(a.residual, a.ld_residual, e) && aligned(a.sum, a.ld_sum, e) && (e8 || aligned(a.y, a.ld_y, e));
    const bool vec8 = (uintptr_t)a.y % 8 == 0 && a.ld_y % 8 == 0;
    const unsigned grid = (unsigned)std::min<long long>(a.rows, 4ll * sms);
    auto go = [&](auto kernel) { kernel<<<grid, kWide, 0, stream>>>(a, vec8); return cudaGetLastError(); };
    if (dtype == kF32) {
        if (e8) return vec ? go(wide_rms_forward_kernel<kF32, true, true>) : go(wide_rms_forward_kernel<kF32, false, true>);
        return vec ? go(wide_rms_forward_kernel<kF32, true, false>) : go(wide_rms_forward_kernel<kF32, false, false>);
    }
    if (e8) return vec ? go(wide_rms_forward_kernel<kBF16, true, true>) : go(wide_rms_forward_kernel<kBF16, false, true>);
    return vec ? go(wide_rms_forward_kernel<kBF16, true, false>) : go(wide_rms_forward_kernel<kBF16, false, false>);
}

cudaError_t launch_rms_backward(RmsBackArgs a, int dtype, void* dweight, int sms, cudaStream_t stream) {
    if (a.cols == 0) return cudaSuccess;
    if (!dweight) a.partials = nullptr;
    const int e = dtype == kF32 ? 4 : 2;
    a.weight_vec = (uintptr_t)a.weight % 16 == 0;
    int used = 0;
    if (a.rows > 0) {
        const bool vec = aligned(a.dy, a.ld_dy, e) && aligned(a.h, a.ld_h, e) && aligned(a.dsum, a.ld_dsum, e) && aligned(a.dh, a.ld_dh, e) && aligned(a.dx, a.ld_dx, e);
        cudaError_t err;
        if (a.partials) {
            used = rms_partial_rows(a.rows, a.cols);
            const dim3 grid((unsigned)((a.cols + 127) / 128), (unsigned)used);
            if (dtype == kF32) wide_rms_columns_kernel<kF32><<<grid, 128, 0, stream>>>(a);
            else wide_rms_columns_kernel<kBF16><<<grid, 128, 0, stream>>>(a);
            if ((err = cudaGetLastError()) != cudaSuccess) return err;
        }
        const unsigned grid = (unsigned)std::min<long long>(a.rows, 4ll * sms);
        auto go = [&](auto kernel) { kernel<<<grid, kWide, 0, stream>>>(a); return cudaGetLastError(); };
        if (dtype == kF32) err = vec ? go(wide_rms_backward_kernel<kF32, true>) : go(wide_rms_backward_kernel<kF32, false>);
        else err = vec ? go(wide_rms_backward_kernel<kBF16, true>) : go(wide_rms_backward_kernel<kBF16, false>);
        if (err != cudaSuccess) return err;
    }
    if (!dweight) return cudaSuccess;
    // rows == 0: nothing was launched and the sum over no rows is zeros (used == 0)
    rms_fold_kernel<<<(unsigned)((a.cols + 31) / 32), 32 * kFoldWarps, 0, stream>>>(a.partials, used, a.cols, dweight, a.weight_f32);
    return cudaGetLastError();
}

}  // namespace tmask
