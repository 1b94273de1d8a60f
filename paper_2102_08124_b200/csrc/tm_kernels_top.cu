// The k largest logits of every row, largest first, and the log of the row's softmax sum at a temperature.
//
// Order: a logit is the 64-bit whole number (its value's pattern made monotone, then the index from above), so that equal values go
// by the lower index and no two entries are equal.  -0 counts as +0; NaN is above everything.
//
// Bound: HBM (a logit is read once; about four instructions each, one of them an exponential).  A thread block goes through its row --
// or its slice of one, where a cluster shares a row -- with a running maximum and sum for the softmax and a bound below which no
// logit can be among the k largest: at first the k-th largest of the threads' maxima over the first block of vectors, later the
// k-th largest entry so far.  A vector whose maximum is below the bound costs one comparison.  Entries that pass go to a buffer in
// shared memory; when it holds more than a few hundred, a radix selection over it leaves k and raises the bound (a row of random
// logits does that once or twice).  A row that overruns the buffer between two looks at it, rising values for instance, goes again
// with a look after every vector, between which the buffer cannot overrun.
#include <algorithm>

#include "tm_launch.h"
#include "tm_rows.cuh"

namespace tmask {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kMaxCluster = 8, kBlockVectors = 4, kLook = 640;     // kLook: entries above which the buffer is cut back to k

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

struct TopPlan {
    int cluster;
    long long slice_vectors;
    double kappa;                  // (log2(e) / T) / c2, the rounding of c2
};

// entries of the buffer: kLook, what one vector of every thread can add and the row's edges, at least; and the lists of a cluster
template <int DT, int NT> constexpr int kCapacity = std::max(kLook + NT * RowType<DT>::kVec + 32, kTopMax * (kMaxCluster + 1));

// The k-th largest of buf[0, n), n > k > 0, by 8-bit digits from the top; all threads, which get the same answer.
template <int NT> struct Selection {
    unsigned int hist[256];
    unsigned long long prefix;
    unsigned int left, done;
    __device__ __forceinline__ unsigned long long operator()(const unsigned long long* buf, int n, int k) {
        const int tid = threadIdx.x, lane = tid & 31;
        if (tid == 0) { prefix = 0; left = (unsigned)k; done = 0; }
        for (int digit = 7; digit >= 0; --digit) {
            for (int b = tid; b < 256; b += NT) hist[b] = 0;
            __syncthreads();
            const unsigned long long known = prefix, care = digit == 7 ? 0ull : ~0ull << (8 * (digit + 1));
            for (int i = tid; i < n; i += NT) {
                const unsigned long long e = buf[i];
                if ((e & care) == known) atomicAdd(&hist[(e >> (8 * digit)) & 255], 1u);
            }
            __syncthreads();
            if (tid < 32) {
                // lane l has bins 255 - 8 l downwards: how many entries lie in the lanes before it
                unsigned int own = 0;
                for (int b = 0; b < 8; ++b) own += hist[255 - 8 * lane - b];
                unsigned int before = own;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) { const unsigned int t = __shfl_up_sync(0xFFFFFFFFu, before, o); if (lane >= o) before += t; }
                before -= own;
                const unsigned int want = left;
                __syncwarp();
                if (before < want && want <= before + own) {
                    unsigned int need = want - before;
                    int b = 255 - 8 * lane;
                    while (hist[b] < need) need -= hist[b--];
                    prefix = known | ((unsigned long long)b << (8 * digit));
                    left = need;
                    done = hist[b] == need;               // the whole bin is among the largest: lower digits may be anything
                }
            }
            __syncthreads();
            if (done) break;
        }
        return prefix;
    }
};

template <int DT, int NT> __global__ void __launch_bounds__(NT, NT == 256 ? 4 : 8) top_kernel(const TopArgs a, const TopPlan plan) {
    using T = typename RowType<DT>::T;
    constexpr int V = RowType<DT>::kVec, NW = NT / 32, U = kBlockVectors, kRoom = kCapacity<DT, NT>;
    extern __shared__ __align__(16) unsigned long long buf[];             // kRoom entries
    __shared__ unsigned long long found[kTopMax];
    __shared__ Selection<NT> select;
    __shared__ float2 part[2][NW];
    __shared__ int count_s, kept_s, have_s[2];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int C = plan.cluster;
    const uint32_t rank = C > 1 ? cluster_rank() : 0u;
    const float c2 = kLog2e / a.temperature;
    int turn = 0;

    for (long long r = blockIdx.x / C; r < a.rows; r += gridDim.x / C) {
        const RowVectors<DT> row(static_cast<const T*>(a.logits) + r * a.ld, a.vocab);
        const long long from = min(row.count, (long long)rank * plan.slice_vectors), to = min(row.count, from + plan.slice_vectors);
        const RowPart<DT> slice(row, from, to);
        const uint4* const vec = reinterpret_cast<const uint4*>(row.base + slice.column);
        const int inside = slice.inside, edges = slice.head + slice.tail;
        const int have = (int)min((long long)a.k, (long long)inside * V + edges);         // entries that this slice can give
        const int blocks = (inside + NT * U - 1) / (NT * U), whole = inside / (NT * U);
        auto fetch = [&](uint4 (&w)[U], int b) {
            const uint4* src = vec + b * (NT * U) + tid;
            if (b < whole) {
#pragma unroll
                for (int u = 0; u < U; ++u) w[u] = src[u * NT];
            } else {
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    w[u] = make_uint4(RowType<DT>::kLow, RowType<DT>::kLow, RowType<DT>::kLow, RowType<DT>::kLow);
                    if (b * (NT * U) + u * NT + tid < inside) w[u] = src[u * NT];
                }
            }
        };
        // entries at or above `bound` are collected; `bound_f` is its value (or -Inf, which everything passes)
        unsigned long long bound = 0;
        float bound_f = -INFINITY, m = -3.4028234663852886e38f, s = 0.0f;
        bool full = false, over = false;                  // this thread put an entry past kLook, or past the end
        auto set_bound = [&](unsigned long long b) {
            bound = b;
            const uint32_t key = (uint32_t)(b >> 32);
            bound_f = key <= 0x007FFFFFu ? -INFINITY : value_of(key);                 // -Inf itself is 0x007FFFFF
        };
        auto offer = [&](float v, long long column) {
            const unsigned long long e = entry_of(v, column);
            if (e >= bound) {
                const int at = atomicAdd(&count_s, 1);
                if (at < kRoom) buf[at] = e;
                full |= at >= kLook;
                over |= at >= kRoom;
            }
        };
        // cuts the buffer back to the k largest, whose last one is the new bound; all threads, at a point that all have reached
        auto cut = [&]() {
            const int n = count_s;
            const unsigned long long kth = select(buf, n, have);
            if (tid == 0) kept_s = 0;
            __syncthreads();
            for (int i = tid; i < n; i += NT) if (buf[i] >= kth) found[atomicAdd(&kept_s, 1)] = buf[i];
            __syncthreads();
            for (int i = tid; i < have; i += NT) buf[i] = found[i];
            if (tid == 0) count_s = have;
            if (kth > bound) set_bound(kth);
            full = false;
            __syncthreads();
        };
        auto offer_vector = [&](const uint4& q, float top, int i) {
            if (!(top < bound_f) && i < inside) {
                float v[V];
                unpack_vector<DT>(q, v);
#pragma unroll
                for (int j = 0; j < V; ++j)
                    if (!(v[j] < bound_f)) offer(v[j], slice.column + (long long)i * V + j);
            }
        };
        if (tid == 0) count_s = 0;
        __syncthreads();
        bool broken = false;                              // the buffer has overrun: the sums go on, the list comes from a second walk
        auto step = [&](const uint4 (&w)[U], int b) {
            float top[U];
#pragma unroll
            for (int u = 0; u < U; ++u) top[u] = vector_max_nan<DT>(w[u]);
            if (a.lse) {
                const float old = m;
                m = fmaxf(m, fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * c2);
                const float2 cc = make_float2(c2, c2), mm = make_float2(-m, -m);
                float2 add = make_float2(s * exp2_fast(old - m), 0.0f);
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    float v[V];
                    unpack_vector<DT>(w[u], v);
#pragma unroll
                    for (int j = 0; j < V; j += 2) {
                        const float2 x = __ffma2_rn(make_float2(v[j], v[j + 1]), cc, mm);
                        add = __fadd2_rn(add, make_float2(exp2_fast(x.x), exp2_fast(x.y)));
                    }
                }
                s = add.x + add.y;
            }
            if (b == 0 && min(inside, NT) >= a.k) {
                // at least k threads have a vector: the k-th largest of their maxima, or somewhat less, bounds the k-th largest logit
                const uint32_t key = tid < inside ? order_of(max_nan(max_nan(top[0], top[1]), max_nan(top[2], top[3]))) : 0u;
                uint32_t lo = 0u, hi = 0xFFFFFFFFu;
                for (int q = 0; q < 32 && lo < hi; ++q) {
                    const uint32_t mid = lo + (hi - lo) / 2 + 1;
                    const int n = __syncthreads_count(key >= mid);
                    if (n >= a.k) { lo = mid; if (n <= a.k + a.k / 4) break; } else hi = mid - 1;
                }
                set_bound((unsigned long long)lo << 32);
            }
            if (broken) return;
#pragma unroll
            for (int u = 0; u < U; ++u) offer_vector(w[u], top[u], b * (NT * U) + u * NT + tid);
            if (__syncthreads_or(full)) {
                broken = __syncthreads_or(over);
                if (!broken) cut();
            }
        };
        {
            uint4 even[U], odd[U];
            if (blocks > 0) fetch(even, 0);
            for (int b = 0; b < blocks;) {
                if (b + 1 < blocks) fetch(odd, b + 1);
                step(even, b);
                if (++b == blocks) break;
                if (b + 1 < blocks) fetch(even, b + 1);
                step(odd, b);
                ++b;
            }
        }
        if (broken) {
            if (tid == 0) count_s = 0;
            full = over = false;
            set_bound(0);
            __syncthreads();
            for (int i0 = 0; i0 < inside; i0 += NT) {
                const int i = i0 + tid;
                const uint4 q = i < inside ? vec[i] : make_uint4(0u, 0u, 0u, 0u);
                offer_vector(q, vector_max_nan<DT>(q), i);
                if (__syncthreads_or(full)) cut();
            }
        }
        if (tid < edges) {
            const long long c = slice.edge(tid);
            const float v = to_float(row.base[c]), old = m;
            m = fmaxf(m, v * c2);
            s = s * exp2_fast(old - m) + exp2_fast(fmaf(v, c2, -m));
            offer(v, c);
        }
        __syncthreads();
        if (count_s > have) cut();
        // this slice's list, sorted by counting the larger ones, and the warps' sums
        for (int i = tid; i < have; i += NT) found[i] = buf[i];
        __syncthreads();
        for (int i = tid; i < have; i += NT) {
            const unsigned long long e = found[i];
            int at = 0;
            for (int j = 0; j < have; ++j) at += found[j] > e;
            buf[at] = e;
        }
        auto post = [&]() {
            const float wm = group_max<32>(m), ws = group_sum<32>(s * exp2_fast(m - wm));
            if (lane == 0) part[turn][warp] = make_float2(wm, ws);
            if (tid == 0) have_s[turn] = have;
            __syncwarp();
            if (C > 1) cluster_sync(); else __syncthreads();
        };
        post();
        auto part_of = [&](int i) { return C > 1 ? cluster_load2(&part[turn][i % NW], i / NW) : part[turn][i]; };
        int total = have;
        unsigned long long best = have > 0 ? buf[0] : 0ull;
        if (C > 1) {
            // every block brings the other blocks' lists over and looks its own entries' places up in them
            total = 0;
            unsigned long long* const others = buf + kTopMax;
            int counts[kMaxCluster];
#pragma unroll
            for (int c = 0; c < kMaxCluster; ++c) {
                counts[c] = 0;
                if (c < C) {
                    asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(counts[c]) : "r"(cluster_map(&have_s[turn], c)) : "memory");
                    total += counts[c];
                    for (int i = tid; i < counts[c]; i += NT) others[c * kTopMax + i] = cluster_load64(buf + i, c);
                }
            }
            __syncthreads();
            total = min(total, a.k);
#pragma unroll
            for (int c = 0; c < kMaxCluster; ++c) if (counts[c] > 0) best = max(best, others[c * kTopMax]);
            for (int i = tid; i < have; i += NT) {
                const unsigned long long e = buf[i];
                int at = i;
#pragma unroll
                for (int c = 0; c < kMaxCluster; ++c) {
                    if (c == (int)rank) continue;
                    int lo = 0, hi = counts[c];           // entries of block c above e
                    while (lo < hi) { const int mid = (lo + hi) / 2; if (others[c * kTopMax + mid] > e) lo = mid + 1; else hi = mid; }
                    at += lo;
                }
                if (at < a.k) {
                    a.values[r * a.k + at] = value_of((uint32_t)(e >> 32));
                    a.ids[r * a.k + at] = (int)(0xFFFFFFFFu - (uint32_t)e);
                }
            }
        } else {
            for (int i = tid; i < have; i += NT) {
                a.values[r * a.k + i] = value_of((uint32_t)(buf[i] >> 32));
                a.ids[r * a.k + i] = (int)(0xFFFFFFFFu - (uint32_t)buf[i]);
            }
        }
        if (rank == 0) for (int i = total + tid; i < a.k; i += NT) { a.values[r * a.k + i] = -INFINITY; a.ids[r * a.k + i] = -1; }
        const float M = total > 0 ? value_of((uint32_t)(best >> 32)) : -INFINITY;
        const bool finite = fabsf(M) < INFINITY;
        if (rank == 0 && tid == 0) {
            if (a.status && total > 0 && !(M < INFINITY)) atomicOr(a.status, kDevNonFinite);
            if (a.lse && !finite) a.lse[r] = M;
        }
        if (a.lse && finite) {
            float R = -3.4028234663852886e38f;
            for (int i = lane; i < C * NW; i += 32) R = fmaxf(R, part_of(i).x);
            R = group_max<32>(R);
            const bool slow = !(fabsf(R) < 1e30f);
            if (slow) {
                // logits so large or small that their scaled form leaves the range: again, with the difference first
                s = 0.0f;
                auto add = [&](float v) { s += exp2_fast((v - M) * c2); };
                for (int i = tid; i < inside; i += NT) {
                    float v[V];
                    unpack_vector<DT>(vec[i], v);
                    for (int j = 0; j < V; ++j) add(v[j]);
                }
                if (tid < edges) add(to_float(row.base[slice.edge(tid)]));
                m = R = 0.0f;
                turn ^= 1;
                post();
            }
            if (rank == 0 && warp == 0) {
                float sum = 0.0f;
                for (int i = lane; i < C * NW; i += 32) { const float2 p = part_of(i); sum += p.y * exp2_fast(p.x - R); }
                sum = group_sum<32>(sum);
                if (lane == 0) a.lse[r] = (float)((slow ? (double)M / a.temperature : R * plan.kappa * 0.69314718055994530942) + (double)logf(sum));
            }
        }
        turn ^= 1;
        if (C > 1) cluster_sync(); else __syncthreads();  // the buffer, and what others read of it, is free again
    }
}

template <int DT, int NT> cudaError_t launch_rows(const TopArgs& a, const TopPlan& plan, cudaStream_t stream) {
    auto kernel = top_kernel<DT, NT>;
    cudaLaunchConfig_t cfg = {};
    cfg.blockDim = dim3(NT);
    cfg.gridDim = dim3((unsigned)plan.cluster);
    cfg.dynamicSmemBytes = kCapacity<DT, NT> * sizeof(unsigned long long);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)plan.cluster; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cudaError_t e;
    // clusters that the device holds at once: asked again only when this thread's last answer was for another shape
    static thread_local struct { int dev, cluster, clusters; } last = {-1, 0, 0};
    int dev = 0;
    if ((e = cudaGetDevice(&dev)) != cudaSuccess) return e;
    if (last.dev != dev || last.cluster != plan.cluster) {
        int clusters = 0;
        if ((e = cudaOccupancyMaxActiveClusters(&clusters, kernel, &cfg)) != cudaSuccess) return e;
        last = {dev, plan.cluster, clusters < 1 ? 1 : clusters};
    }
    cfg.gridDim = dim3((unsigned)(std::min<long long>(a.rows, last.clusters) * plan.cluster));
    return cudaLaunchKernelEx(&cfg, kernel, a, plan);
}

}  // namespace

cudaError_t launch_top(const TopArgs& a, int dtype, int sms, cudaStream_t stream) {
    if (a.rows == 0) return cudaSuccess;
    const int e = dtype == kF32 ? 4 : 2, V = 16 / e;
    const long long vectors = std::max<long long>(1, (a.vocab + 2 * V - 2) / V);      // of a row, wherever it starts
    TopPlan plan;
    const double c2 = 1.4426950408889634074 / a.temperature;
    plan.kappa = c2 / (double)(kLog2e / a.temperature);
    plan.cluster = 1;
    while (plan.cluster < kMaxCluster && a.rows * plan.cluster * 2 <= sms && vectors / plan.cluster > 256) plan.cluster *= 2;
    plan.slice_vectors = (vectors + plan.cluster - 1) / plan.cluster;
    const bool small = vectors <= 1024 && a.rows > 2ll * sms;
    if (dtype == kF32) return small ? launch_rows<kF32, 128>(a, plan, stream) : launch_rows<kF32, 256>(a, plan, stream);
    return small ? launch_rows<kBF16, 128>(a, plan, stream) : launch_rows<kBF16, 256>(a, plan, stream);
}

}  // namespace tmask
