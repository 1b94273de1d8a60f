// Verification of drafted tokens against the target's probabilities.
//
//   p, q      softmax of a row of the target's logits and of the drafter's, z / T each
//   draft x   stays while u q(x) < p(x);  at the first that does not, the token is drawn from max(p - q, 0), behind the last from p
//   the draw  is a race of exponentials: the token with the largest r_k / E_k, E_k = -log(1 - u_k), wins with probability r_k / sum r, so no
//             sum over r and no search in running sums is needed, and the answer hangs on a comparison of two numbers, not on the rounding of a sum
//             of a hundred thousand terms
//
// A row's numbers e^(z/T) are 2^((z - m) c), c = log2(e) / T, m the running maximum (differences first: an offset that all logits share is no
// loss, and masks of the type's lowest value are zeros beside anything else).  Threads sum in fp32, the threads' sums are joined in fp64.
#include <algorithm>
#include <cfloat>

#include "tm_philox.cuh"
#include "tm_rows.cuh"

namespace tmask {
namespace {

constexpr uint32_t kTestBlocks = 0x80000000u;      // the generator's blocks of the acceptance tests; the draw's are tokens / 4, far below
constexpr float kMargin = 1e-3f;                   // of a logarithm to base 2 in the screening of the race: above its rounding down to 2^-1074

struct RowStat { float m; double s; bool bad; };   // largest logit, sum of 2^((z - m) c), NaN or +Inf among them or nothing but -Inf

template <int DT> __device__ __forceinline__ void take_logits(const float* v, int n, float c, float& m, float& s, bool& bad) {
    float top = v[0];
    for (int j = 1; j < n; ++j) top = max_nan(top, v[j]);
    bad |= !(top < INFINITY);
    if (top > m) { s *= exp2_fast((m - top) * c); m = top; }
#pragma unroll
    for (int j = 0; j < n; ++j) s += exp2_fast((v[j] - m) * c);
}

// A row's statistics, by a block of THREADS threads; the same for all of them
template <int DT, int THREADS> __device__ RowStat row_stat(const void* row, long long vocab, float c, double* buf_s, float* buf_m) {
    constexpr int V = RowType<DT>::kVec;
    const RowVectors<DT> vectors(row, vocab);
    const RowPart<DT> part(vectors, 0, vectors.count);
    float m = -FLT_MAX, s = 0.0f;
    bool bad = false;
    const uint4* p = reinterpret_cast<const uint4*>(vectors.base + part.column);
    for (int i = threadIdx.x; i < part.inside; i += THREADS) {
        float v[V];
        unpack_vector<DT>(p[i], v);
        take_logits<DT>(v, V, c, m, s, bad);
    }
    if ((int)threadIdx.x < part.head + part.tail) {
        const float v = to_float(vectors.base[part.edge(threadIdx.x)]);
        take_logits<DT>(&v, 1, c, m, s, bad);
    }
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const float wm = group_max<32>(m);
    bad = __any_sync(0xFFFFFFFFu, bad);
    if (lane == 0) buf_m[warp] = bad ? INFINITY : wm;
    __syncthreads();
    const float all = group_max<32>(buf_m[lane & (THREADS / 32 - 1)]);
    double t = (double)(s * exp2_fast((m - all) * c));
    for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xFFFFFFFFu, t, o);
    if (lane == 0) buf_s[warp] = t;
    __syncthreads();
    t = 0.0;
    for (int k = 0; k < THREADS / 32; ++k) t += buf_s[k];
    __syncthreads();
    return RowStat{all, t, !(all < INFINITY) || !(t > 0.0)};
}

constexpr int kThreads = 1024;
template <int DT> __global__ void __launch_bounds__(kThreads) verify_kernel(const VerifyArgs a) {
    using T = typename RowType<DT>::T;
    __shared__ double buf_s[32];
    __shared__ float buf_m[32];
    __shared__ double best_key[32];
    __shared__ int best_at[32];
    const PhiloxKey key(a.seed, a.offset, a.offset_dev);
    const int b = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const double cp64 = 1.4426950408889634 / (double)a.temperature, cq64 = 1.4426950408889634 / (double)a.draft_temperature, ln2 = 0.6931471805599453;
    const float cp = (float)cp64, cq = (float)cq64;
    int* tokens = a.tokens + (long long)b * (a.drafted + 1);
    float* logp = a.logp ? a.logp + (long long)b * (a.drafted + 1) : nullptr;
    int n = 0, flags = 0, refused = -1;                       // refused: the token whose draft was not taken
    RowStat p = {}, q = {};
    const T *rp = nullptr, *rq = nullptr;
    for (;; ++n) {
        rp = static_cast<const T*>(a.logits) + ((long long)b * (a.drafted + 1) + n) * a.ld;
        const int id = n < a.drafted ? a.ids[(long long)b * a.drafted + n] : -1;
        if (id >= a.vocab) flags |= kDevBadId;
        const bool draft = id >= 0 && id < a.vocab;
        p = row_stat<DT, kThreads>(rp, a.vocab, cp, buf_s, buf_m);
        if (p.bad || !draft) break;
        double pq = 1.0;
        if (a.draft_logits) {
            rq = static_cast<const T*>(a.draft_logits) + ((long long)b * a.drafted + n) * a.ld_draft;
            q = row_stat<DT, kThreads>(rq, a.vocab, cq, buf_s, buf_m);
            if (q.bad) { p.bad = true; break; }
            pq = exp2(((double)to_float(rq[id]) - (double)q.m) * cq64) / q.s;
        }
        const double lp = ((double)to_float(rp[id]) - (double)p.m) * cp64 - log2(p.s);
        const uint4 w = key(kTestBlocks + n / 4, b);
        const uint32_t word = n % 4 == 0 ? w.x : n % 4 == 1 ? w.y : n % 4 == 2 ? w.z : w.w;
        if (!(((double)word + 0.5) * 0x1p-32 * pq < exp2(lp))) { refused = id; break; }
        if (threadIdx.x == 0) {
            tokens[n] = id;
            if (logp) logp[n] = (float)(lp * ln2);
        }
    }
    int token = -1;
    if (!p.bad) {
        // the race; where p - q leaves nothing, p itself
        for (int pass = refused >= 0 ? 0 : 1; pass < 2 && token < 0; ++pass) {
            const bool minus = pass == 0;
            const double shift = minus && a.draft_logits ? log2(p.s) - log2(q.s) : 0.0;      // q in units of 2^(m c) of p
            double mine = 0.0;
            int at = -1;
            float best = -INFINITY;                             // log2 of the warp's best key, less the margin
            const long long blocks = (a.vocab + 3) / 4;
            for (long long i0 = 0; i0 < blocks; i0 += kThreads) {
                const long long k0 = (i0 + threadIdx.x) * 4;
                float z[4];
                uint4 w = make_uint4(0, 0, 0, 0);
                bool any = false;
                float x[4], lu[4];
                if (k0 < a.vocab) w = key((uint32_t)(k0 / 4), b);
                const uint32_t word[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    z[j] = k0 + j < a.vocab ? to_float(rp[k0 + j]) : -INFINITY;
                    x[j] = (z[j] - p.m) * cp;
                    lu[j] = __log2f(fmaf((float)word[j], 0x1p-32f, 0x1p-33f));
                    any |= x[j] - lu[j] > best;
                }
                if (!__any_sync(0xFFFFFFFFu, any)) continue;
                float top = -INFINITY;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (!(x[j] - lu[j] > best)) continue;
                    double r = exp2(((double)z[j] - (double)p.m) * cp64);
                    if (minus) {
                        if (a.draft_logits) r -= exp2(((double)to_float(rq[k0 + j]) - (double)q.m) * cq64 + shift);
                        else if (k0 + j == refused) r = 0.0;
                    }
                    if (!(r > 0.0)) continue;
                    const double k = r / -log1p(-((double)word[j] + 0.5) * 0x1p-32);
                    if (k > mine) { mine = k; at = (int)(k0 + j); }
                    top = fmaxf(top, (float)log2(k) - kMargin);
                }
                best = fmaxf(best, group_max<32>(top));
            }
            for (int o = 16; o > 0; o >>= 1) {
                const double ok = __shfl_xor_sync(0xFFFFFFFFu, mine, o);
                const int oa = __shfl_xor_sync(0xFFFFFFFFu, at, o);
                if (ok > mine || (ok == mine && (unsigned)oa < (unsigned)at)) { mine = ok; at = oa; }
            }
            if (lane == 0) { best_key[warp] = mine; best_at[warp] = at; }
            __syncthreads();
            mine = 0.0;
            for (int k = 0; k < kThreads / 32; ++k)
                if (best_key[k] > mine || (best_key[k] == mine && (unsigned)best_at[k] < (unsigned)token)) { mine = best_key[k]; token = best_at[k]; }
            __syncthreads();
        }
    } else flags |= kDevNonFinite;
    if (threadIdx.x == 0) {
        a.accepted[b] = n;
        tokens[n] = token;
        if (logp) logp[n] = token < 0 ? __int_as_float(0x7FC00000) : (float)((((double)to_float(rp[token]) - (double)p.m) * cp64 - log2(p.s)) * ln2);
        for (int k = n + 1; k <= a.drafted; ++k) {
            tokens[k] = -1;
            if (logp) logp[k] = 0.0f;
        }
        if (flags && a.status) atomicOr(a.status, flags);
    }
}

}  // namespace

cudaError_t launch_verify(const VerifyArgs& a, int dtype, int, cudaStream_t stream) {
    if (a.batch == 0) return cudaSuccess;
    if (dtype == kF32) verify_kernel<kF32><<<(unsigned)a.batch, kThreads, 0, stream>>>(a);
    else verify_kernel<kBF16><<<(unsigned)a.batch, kThreads, 0, stream>>>(a);
    return cudaGetLastError();
}

}  // namespace tmask
