// The k largest logits of every row, largest first, and the log of the row's softmax sum at a temperature.
//
// Order: a logit is the 64-bit whole number (its value's pattern made monotone, then the index from above), so that equal
// values go by the lower index and no two entries are equal.  -0 counts as +0; NaN is above everything.
#include <algorithm>

#include "tm_launch.h"
#include "tm_rows.cuh"

namespace tmask {

namespace {

constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ uint32_t order_of(float v) {
    if (v != v) return 0xFFFFFFFFu;
    const uint32_t u = __float_as_uint(v + 0.0f);         // -0 + 0 = +0
    return u ^ ((u >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key) {
    return key == 0xFFFFFFFFu ? __uint_as_float(0x7FC00000u) : __uint_as_float(key ^ ((key >> 31) ? 0x80000000u : 0xFFFFFFFFu));
}
__device__ __forceinline__ unsigned long long entry_of(float v, long long column) {
    return ((unsigned long long)order_of(v) << 32) | (0xFFFFFFFFu - (uint32_t)column);
}

// exp((v - top) / T): the difference first, so that rows of the type's lowest or largest numbers keep their proportions; 1 where
// both are the same infinity
__device__ __forceinline__ float power(float v, float top, float c2) { return v == top ? 1.0f : exp2_fast((v - top) * c2); }
// log of s exponentials relative to the largest logit; s is NaN if a logit was, and counts the infinite ones if any was
__device__ __forceinline__ float log_sum(float top, float s, float temperature) {
    if (s != s || fabsf(top) == INFINITY) return s != s ? s : top;
    return (float)((double)top / temperature + (double)logf(s));
}

// Any vocabulary: one CTA a row, the row read again (from L2) for each of up to eight 8-bit digits of a radix selection.
constexpr int kWideThreads = 512;
template <int DT> __global__ void __launch_bounds__(kWideThreads) wide_top_kernel(const TopArgs a) {
    constexpr int V = RowType<DT>::kVec;
    __shared__ float bm[kWideThreads / 32], bs[kWideThreads / 32];
    __shared__ unsigned int hist[256];
    __shared__ unsigned long long found[kTopMax], prefix_s;
    __shared__ unsigned int left_s, done_s, n_found;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const float c2 = kLog2e / a.temperature;
    const int k = (int)min((long long)a.k, a.vocab);
    for (long long r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const RowVectors<DT> row(static_cast<const typename RowType<DT>::T*>(a.logits) + r * a.ld, a.vocab);
        float m = -INFINITY, s = 0.0f;
        bool odd = false;
        for (long long i = tid; i < row.count; i += kWideThreads) {
            float v[V];
            row.load(i, v, -INFINITY);
            float top = m;
#pragma unroll
            for (int j = 0; j < V; ++j) { top = fmaxf(top, v[j]); odd |= !(v[j] < INFINITY); }
            s *= power(m, top, c2);
#pragma unroll
            for (int j = 0; j < V; ++j) s += v[j] == -INFINITY ? 0.0f : power(v[j], top, c2);
            m = top;
        }
        if (odd && a.status) atomicOr(a.status, kDevNonFinite);
        const float wm = group_max<32>(m);
        const float ws = group_sum<32>(s * power(m, wm, c2));
        if (lane == 0) { bm[warp] = wm; bs[warp] = ws; }
        if (tid == 0) { prefix_s = 0; left_s = (unsigned)k; done_s = k == 0; n_found = 0; }
        __syncthreads();
        if (warp == 0) {
            const float om = lane < kWideThreads / 32 ? bm[lane] : -INFINITY, os = lane < kWideThreads / 32 ? bs[lane] : 0.0f;
            const float tm_ = group_max<32>(om);
            const float ts = group_sum<32>(os * power(om, tm_, c2));
            if (lane == 0 && a.lse) a.lse[r] = log_sum(tm_, ts, a.temperature);
        }
        for (int digit = 7; digit >= 0 && !done_s; --digit) {
            for (int b = tid; b < 256; b += kWideThreads) hist[b] = 0;
            __syncthreads();
            const unsigned long long prefix = prefix_s, care = digit == 7 ? 0ull : ~0ull << (8 * (digit + 1));
            for (long long i = tid; i < row.count; i += kWideThreads) {
                float v[V];
                row.load(i, v, 0.0f);
                const long long c = row.column(i);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    if (c + j < 0 || c + j >= a.vocab) continue;
                    const unsigned long long e = entry_of(v[j], c + j);
                    if ((e & care) == prefix) atomicAdd(&hist[(e >> (8 * digit)) & 255], 1u);
                }
            }
            __syncthreads();
            if (tid == 0) {
                unsigned int left = left_s, b = 255;
                while (hist[b] < left) left -= hist[b--];
                prefix_s = prefix | ((unsigned long long)b << (8 * digit));
                left_s = left;
                done_s = hist[b] == left;                 // the whole bin belongs to the list: lower digits may be anything
            }
            __syncthreads();
        }
        __syncthreads();
        if (k > 0) {
            const unsigned long long bound = prefix_s;
            for (long long i = tid; i < row.count; i += kWideThreads) {
                float v[V];
                row.load(i, v, 0.0f);
                const long long c = row.column(i);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    if (c + j < 0 || c + j >= a.vocab) continue;
                    const unsigned long long e = entry_of(v[j], c + j);
                    if (e >= bound) { const unsigned int at = atomicAdd(&n_found, 1u); if (at < kTopMax) found[at] = e; }
                }
            }
        }
        __syncthreads();
        for (int i = tid; i < a.k; i += kWideThreads) {
            if (i < k) {
                const unsigned long long e = found[i];
                int rank = 0;
                for (int j = 0; j < k; ++j) rank += found[j] > e;
                a.values[r * a.k + rank] = value_of((uint32_t)(e >> 32));
                a.ids[r * a.k + rank] = (int)(0xFFFFFFFFu - (uint32_t)e);
            } else { a.values[r * a.k + i] = -INFINITY; a.ids[r * a.k + i] = -1; }
        }
        __syncthreads();
    }
}

}  // namespace

cudaError_t launch_top(const TopArgs& a, int dtype, int sms, cudaStream_t stream) {
    if (a.rows == 0) return cudaSuccess;
    const unsigned grid = (unsigned)std::min<long long>(a.rows, 4ll * sms);
    if (dtype == kF32) wide_top_kernel<kF32><<<grid, kWideThreads, 0, stream>>>(a);
    else wide_top_kernel<kBF16><<<grid, kWideThreads, 0, stream>>>(a);
    return cudaGetLastError();
}

}  // namespace tmask
