// Distillation from a teacher's list of largest logits: loss, gradient, or both.
//
//   q = softmax(z / T) over the row;  p = softmax(v / T) over the list's entries, or, where the teacher's log-sum-exp L is
//   given, p_k = exp(v_k / T - L) and p_rest = max(0, 1 - sum_k p_k) for everything the list leaves out (q_rest: the student's)
//   loss      = f [ sum_k p_k (log p_k - log q_k) + p_rest (log p_rest - log q_rest) ],   f = scale * row weight
//   dloss/dz  = f / T (q_j - p_j) for a listed logit,  f / T (q_j - p_rest q_j / q_rest) for another one
//
// q_rest is the sum over the unlisted logits themselves, never one minus the listed mass: the difference would lose all its
// digits where the student puts nearly everything on the list.  Terms with p = 0 are left out, and so is the rest's term where
// the student has no mass there.
#include <algorithm>

#include "tm_launch.h"
#include "tm_rows.cuh"

namespace tmask {

namespace {

constexpr double kLog2eD = 1.4426950408889634074, kLn2D = 0.69314718055994530942;

// A row's list as the kernels use it: entries in their order, unusable ones (padding, out of range, repeated) with id -1.
struct List {
    int id[kTopMax];
    float p[kTopMax];      // the teacher's probability of the entry
    float z[kTopMax];      // the student's logit
};

__device__ __forceinline__ float warp_sum(float v) { return group_sum<32>(v); }
__device__ __forceinline__ double warp_sum_double(double v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}

// Any vocabulary: one CTA a row.  Which logits are listed is asked of a bit filter over id mod 32768 first and of the list
// itself only where the filter says so.
constexpr int kWideThreads = 512, kFilterBits = 32768;
template <int DT, bool LOSS, bool GRAD> __global__ void __launch_bounds__(kWideThreads) wide_distill_kernel(const DistillArgs a) {
    constexpr int V = RowType<DT>::kVec, kWarps = kWideThreads / 32;
    __shared__ List list;
    __shared__ uint32_t filter[kFilterBits / 32];
    __shared__ float bm[kWarps], bs[kWarps];
    __shared__ double bd[kWarps];
    __shared__ float share[8];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const float inv_t = 1.0f / a.temperature, c2 = (float)(kLog2eD / a.temperature);
    using T = typename RowType<DT>::T;
    for (long long r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const RowVectors<DT> row(static_cast<const T*>(a.logits) + r * a.ld, a.vocab);
        T* out = GRAD ? static_cast<T*>(a.dlogits) + r * a.ld_d : nullptr;
        const bool same = GRAD && ((reinterpret_cast<uintptr_t>(out) ^ reinterpret_cast<uintptr_t>(row.base)) & 15) == 0;
        const float weight = a.row_weight ? a.row_weight[r] : 1.0f;
        for (int i = tid; i < kFilterBits / 32; i += kWideThreads) filter[i] = 0;
        __syncthreads();
        // the list: entries in range, the first of equal ids, their logits
        bool bad = false;
        if (weight != 0.0f)
            for (int k = tid; k < a.k; k += kWideThreads) {
                const int id = a.ids[r * a.k + k];
                bool ok = id >= 0;
                if (ok && id >= a.vocab) { ok = false; bad = true; }
                for (int j = 0; ok && j < k; ++j)
                    if (a.ids[r * a.k + j] == id) { ok = false; bad = true; }
                list.id[k] = ok ? id : -1;
                list.z[k] = ok ? to_float(row.base[id]) : 0.0f;
                if (ok) atomicOr(&filter[(id & (kFilterBits - 1)) >> 5], 1u << (id & 31));
            }
        if (bad && a.status) atomicOr(a.status, kDevBadId);
        __syncthreads();
        // the teacher's side, by one warp
        if (warp == 0) {
            float vm = -INFINITY;
            int n = 0;
            if (weight != 0.0f)
                for (int k = lane; k < a.k; k += 32)
                    if (list.id[k] >= 0) { vm = fmaxf(vm, a.values[r * a.k + k] * inv_t); ++n; }
            vm = group_max<32>(vm);
            n = (int)__reduce_add_sync(0xFFFFFFFFu, (unsigned)n);
            float shift = a.teacher_lse ? a.teacher_lse[r] : 0.0f, s = 0.0f;
            if (!a.teacher_lse) {
                if (n > 0)
                    for (int k = lane; k < a.k; k += 32)
                        if (list.id[k] >= 0) s += expf(a.values[r * a.k + k] * inv_t - vm);
                s = warp_sum(s);
                shift = vm + logf(s);
            }
            double mass = 0.0, ent = 0.0;
            for (int k = lane; n > 0 && k < a.k; k += 32)
                if (list.id[k] >= 0) {
                    const float lp = a.values[r * a.k + k] * inv_t - shift, p = expf(lp);
                    list.p[k] = p;
                    mass += p;
                    if (p != 0.0f) ent += (double)p * lp;
                }
            mass = warp_sum_double(mass);
            ent = warp_sum_double(ent);
            if (lane == 0) {
                const float rest = a.teacher_lse ? fmaxf(0.0f, (float)(1.0 - mass)) : 0.0f;
                share[0] = __int_as_float(n);
                share[1] = rest;
                bd[0] = ent; bd[1] = mass;
            }
        }
        __syncthreads();
        const bool on = weight != 0.0f && __float_as_int(share[0]) > 0;
        const float rest = share[1];
        const double entropy = bd[0], mass = bd[1];
        __syncthreads();
        if (!on) {
            if (tid == 0) {
                if (LOSS) a.loss[r] = 0.0f;
                if (LOSS && a.stats) a.stats[2 * r] = a.stats[2 * r + 1] = 0.0f;
            }
            if constexpr (GRAD) {
                const float zero[V] = {};
                for (long long i = tid; i < row.count; i += kWideThreads) row.store(out, same, i, zero);
            }
            continue;
        }
        auto listed = [&](long long c) {
            if (!((filter[(c & (kFilterBits - 1)) >> 5] >> (c & 31)) & 1u)) return -1;
            for (int k = 0; k < a.k; ++k)
                if (list.id[k] == c) return k;
            return -1;
        };
        // q_j = 2^((z_j - ref) c2 - shift2): the difference first, so that a row of the type's lowest numbers keeps its proportions
        float ref, shift2, log_rest2;                     // log_rest2: log2 of q_rest
        if constexpr (LOSS) {
            float m = -INFINITY, s = 0.0f;                // unlisted logits
            for (long long i = tid; i < row.count; i += kWideThreads) {
                float v[V];
                row.load(i, v, -INFINITY);
                const long long c = row.column(i);
                float top = m;
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    if (c + j >= 0 && c + j < a.vocab && listed(c + j) >= 0) v[j] = -INFINITY;
                    top = fmaxf(top, v[j]);
                }
                const float ref = top == -INFINITY ? 0.0f : top;
                s *= exp2_fast((m - ref) * c2);
#pragma unroll
                for (int j = 0; j < V; ++j) s += exp2_fast((v[j] - ref) * c2);
                m = top;
            }
            float lm = -INFINITY;
            double dot = 0.0;
            for (int k = tid; k < a.k; k += kWideThreads)
                if (list.id[k] >= 0) {
                    lm = fmaxf(lm, list.z[k]);
                    if (list.p[k] != 0.0f) dot += (double)list.p[k] * list.z[k];
                }
            const float wm = group_max<32>(fmaxf(m, lm));
            if (lane == 0) bm[warp] = wm;
            __syncthreads();
            float M = -INFINITY;
            for (int w = 0; w < kWarps; ++w) M = fmaxf(M, bm[w]);
            s = warp_sum(m == -INFINITY ? s : s * exp2_fast((m - M) * c2));
            float sl = 0.0f;
            for (int k = tid; k < a.k; k += kWideThreads)
                if (list.id[k] >= 0) sl += exp2_fast((list.z[k] - M) * c2);
            sl = warp_sum(sl);
            dot = warp_sum_double(dot);
            __syncthreads();
            if (lane == 0) { bm[warp] = s; bs[warp] = sl; bd[warp] = dot; }
            __syncthreads();
            s = sl = 0.0f; dot = 0.0;
            for (int w = 0; w < kWarps; ++w) { s += bm[w]; sl += bs[w]; dot += bd[w]; }
            const float all2 = log2f(s + sl);
            ref = M;
            shift2 = all2;
            log_rest2 = log2f(s) - all2;
            if (tid == 0) {
                const double lse = (double)M / a.temperature + all2 * kLn2D, log_rest = (double)log_rest2 * kLn2D;
                double loss = entropy - dot / a.temperature + mass * lse;
                if (rest > 0.0f && s > 0.0f) loss += (double)rest * (logf(rest) - log_rest);
                if (s != s) loss = s;
                a.loss[r] = (float)(loss * weight * a.scale);
                if (a.stats) { a.stats[2 * r] = (float)lse; a.stats[2 * r + 1] = a.teacher_lse ? (float)log_rest : 0.0f; }
            }
        } else {
            ref = a.stats[2 * r];
            shift2 = 0.0f;
            log_rest2 = (float)(a.stats[2 * r + 1] * kLog2eD);
        }
        if constexpr (GRAD) {
            const float up = weight * a.scale * inv_t * (a.grad_loss ? a.grad_loss[r] : 1.0f);
            const float off = rest > 0.0f && log_rest2 > -INFINITY ? 1.0f - rest * exp2f(-log_rest2) : 1.0f;
            for (long long i = tid; i < row.count; i += kWideThreads) {
                float v[V];
                row.load(i, v, 0.0f);
                const long long c = row.column(i);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float q = LOSS ? exp2_fast(fmaf(v[j] - ref, c2, -shift2)) : exp2_fast(fmaf(v[j], inv_t, -ref) * (float)kLog2eD);
                    const int k = c + j >= 0 && c + j < a.vocab ? listed(c + j) : -1;
                    v[j] = up * (k >= 0 ? q - list.p[k] : q * off);
                }
                row.store(out, same, i, v);
            }
        }
        __syncthreads();
    }
}

template <bool LOSS, bool GRAD> cudaError_t launch(const DistillArgs& a, int dtype, int sms, cudaStream_t stream) {
    const unsigned grid = (unsigned)std::min<long long>(a.rows, 4ll * sms);
    if (dtype == kF32) wide_distill_kernel<kF32, LOSS, GRAD><<<grid, kWideThreads, 0, stream>>>(a);
    else wide_distill_kernel<kBF16, LOSS, GRAD><<<grid, kWideThreads, 0, stream>>>(a);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_distill(const DistillArgs& a, int dtype, bool loss, bool grad, int sms, cudaStream_t stream) {
    if (a.rows == 0) return cudaSuccess;
    if (loss && grad) return launch<true, true>(a, dtype, sms, stream);
    return loss ? launch<true, false>(a, dtype, sms, stream) : launch<false, true>(a, dtype, sms, stream);
}

}  // namespace tmask
