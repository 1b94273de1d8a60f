// The k largest logits of every row, largest first, and the log of the row's softmax sum at a temperature.
//
// Order: a logit is the 64-bit whole number (its value's pattern made monotone, then the index from above), so that equal values go
// by the lower index and no two entries are equal.  -0 counts as +0; NaN is above everything.
//
// Bound: HBM (about six instructions a logit, one of them an exponential).  A thread block goes through its row -- or its slice of
// one, where a cluster shares a row -- twice.  Pass 1 takes the softmax's running maximum and sum and every thread's largest logit.
// The k-th largest of those is a bound that at least k logits reach, and few more do (of 131072 random ones and k = 64 some 75).  A
// slice of fewer vectors than k, or a list longer than the block, has none; the buffer then holds the whole slice.
// Pass 2 collects the logits that reach it: a comparison for a vector.  What shared memory had room for in pass 1 comes from there,
// the rest from L2, so that HBM is read once.  The entries are then put in order by counting, for each, the larger ones.
// Where far more reach the bound than the buffer holds (few threads have seen all the large ones), the vectors are gone through
// again one of each thread at a time, a radix selection cutting the buffer back to k, and raising the bound, whenever it fills up.
#include <algorithm>

#include "tm_launch.h"
#include "tm_rows.cuh"

namespace tmask {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kMaxCluster = 8, kBlockVectors = 4;
constexpr int kLook = 640;     // entries above which the buffer is cut back to k

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
    int cluster, stash;            // stash: blocks of NT * U vectors that stay in shared memory between the passes
    long long slice_vectors;
    double kappa;                  // (log2(e) / T) / c2, the rounding of c2
};

// entries of the buffer: kLook, what one vector of every thread can add and the row's edges, at least; and the lists of a cluster
template <int DT, int NT> constexpr int kCapacity = 2 * ((1 + std::max(kLook + NT * RowType<DT>::kVec + 32, kTopMax * (kMaxCluster + 1))) / 2);

// A block's list under way, in shared memory
struct Work {
    unsigned int hist[256];
    unsigned long long found[kTopMax], prefix;
    unsigned int left, done;
    int count, kept;               // entries of the buffer
};

// Cuts buf[0, w.count) back to its `have` largest (0 < have < w.count) and returns a number that exactly they reach: a radix
// selection by 8-bit digits from the top.  All threads; out of line, for its size.
template <int NT> __device__ __noinline__ unsigned long long cut_back(unsigned long long* buf, Work& w, int have) {
    const int tid = threadIdx.x, lane = tid & 31, n = w.count;
    if (tid == 0) { w.prefix = 0; w.left = (unsigned)have; w.done = 0; w.kept = 0; }
    for (int digit = 7; digit >= 0; --digit) {
        for (int b = tid; b < 256; b += NT) w.hist[b] = 0;
        __syncthreads();
        const unsigned long long known = w.prefix, care = digit == 7 ? 0ull : ~0ull << (8 * (digit + 1));
        for (int i = tid; i < n; i += NT) {
            const unsigned long long e = buf[i];
            if ((e & care) == known) atomicAdd(&w.hist[(e >> (8 * digit)) & 255], 1u);
        }
        __syncthreads();
        if (tid < 32) {
            // lane l has bins 255 - 8 l downwards: how many entries lie in the lanes before it
            unsigned int own = 0;
            for (int b = 0; b < 8; ++b) own += w.hist[255 - 8 * lane - b];
            unsigned int before = own;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) { const unsigned int t = __shfl_up_sync(0xFFFFFFFFu, before, o); if (lane >= o) before += t; }
            before -= own;
            const unsigned int want = w.left;
            __syncwarp();
            if (before < want && want <= before + own) {
                unsigned int need = want - before;
                int b = 255 - 8 * lane;
                while (w.hist[b] < need) need -= w.hist[b--];
                w.prefix = known | ((unsigned long long)b << (8 * digit));
                w.left = need;
                w.done = w.hist[b] == need;               // the whole bin is among the largest: lower digits may be anything
            }
        }
        __syncthreads();
        if (w.done) break;
    }
    const unsigned long long kth = w.prefix;
    for (int i = tid; i < n; i += NT) if (buf[i] >= kth) w.found[atomicAdd(&w.kept, 1)] = buf[i];
    __syncthreads();
    for (int i = tid; i < have; i += NT) buf[i] = w.found[i];
    if (tid == 0) w.count = have;
    __syncthreads();
    return kth;
}

// value below which no entry reaches `bound` (-Inf: none)
__device__ __forceinline__ float bound_value(unsigned long long bound) {
    const uint32_t key = (uint32_t)(bound >> 32);
    return key <= 0x007FFFFFu ? -INFINITY : value_of(key);                            // -Inf itself is 0x007FFFFF
}

// A number that at least k of the threads' keys reach, and hardly more: the k-th largest by its upper 16 bits.  All threads.
template <int NT> __device__ __noinline__ uint32_t bound_of_keys(uint32_t key, int k, Work& w) {
    const int tid = threadIdx.x, lane = tid & 31;
    if (tid == 0) { w.prefix = 0; w.left = (unsigned)k; }
    for (int digit = 3; digit >= 2; --digit) {
        for (int b = tid; b < 256; b += NT) w.hist[b] = 0;
        __syncthreads();
        const uint32_t known = (uint32_t)w.prefix;
        if (digit == 3 || (key >> 24) == known >> 24) atomicAdd(&w.hist[(key >> (8 * digit)) & 255], 1u);
        __syncthreads();
        if (tid < 32) {
            unsigned int own = 0;
            for (int b = 0; b < 8; ++b) own += w.hist[255 - 8 * lane - b];
            unsigned int before = own;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) { const unsigned int t = __shfl_up_sync(0xFFFFFFFFu, before, o); if (lane >= o) before += t; }
            before -= own;
            const unsigned int want = w.left;
            __syncwarp();
            if (before < want && want <= before + own) {
                unsigned int need = want - before;
                int b = 255 - 8 * lane;
                while (w.hist[b] < need) need -= w.hist[b--];
                w.prefix = known | ((uint32_t)b << (8 * digit));
                w.left = need;
            }
        }
        __syncthreads();
    }
    return (uint32_t)w.prefix;
}

// The entries of a vector at or above the bound, into the buffer as far as it has room.  Out of line: few vectors get here.
template <int DT> __device__ __noinline__ void offer_vector(uint4 q, float least, unsigned long long bound, long long column, unsigned long long* buf, int room, int* count) {
    constexpr int V = RowType<DT>::kVec;
    float v[V];
    unpack_vector<DT>(q, v);
#pragma unroll
    for (int j = 0; j < V; ++j) {
        if (v[j] < least) continue;
        const unsigned long long e = entry_of(v[j], column + j);
        if (e >= bound) {
            const int at = atomicAdd(count, 1);
            if (at < room) buf[at] = e;
        }
    }
}

// Collects the entries at or above the bound one vector of each thread at a time, with a look at the buffer after each.  All threads,
// none of which may still have to read the count when the first one enters.
template <int DT, int NT> __device__ __noinline__ void collect_slowly(unsigned long long* buf, Work& w, const uint4* vec, int inside, unsigned long long bound, long long column,
                                                                      int have) {
    constexpr int V = RowType<DT>::kVec;
    if (threadIdx.x == 0) w.count = 0;
    __syncthreads();
    for (int i0 = 0; i0 < inside; i0 += NT) {
        const int i = i0 + (int)threadIdx.x;
        bool full = false;
        if (i < inside) {
            const uint4 q = vec[i];
            const float least = bound_value(bound);
            if (!(vector_max_nan<DT>(q) < least)) {
                float v[V];
                unpack_vector<DT>(q, v);
                for (int j = 0; j < V; ++j)
                    if (!(v[j] < least)) {
                        const unsigned long long e = entry_of(v[j], column + (long long)i * V + j);
                        if (e >= bound) {
                            const int at = atomicAdd(&w.count, 1);
                            buf[at] = e;
                            full |= at >= kLook;
                        }
                    }
            }
        }
        if (__syncthreads_or(full)) bound = max(bound, cut_back<NT>(buf, w, have));
    }
}

template <int NT> constexpr int kBlocks = 1024 / NT;       // blocks an SM: the registers they may use

template <int DT, int NT> __global__ void __launch_bounds__(NT, kBlocks<NT>) top_kernel(const TopArgs a, const TopPlan plan) {
    using T = typename RowType<DT>::T;
    constexpr int V = RowType<DT>::kVec, NW = NT / 32, U = kBlockVectors, kRoom = kCapacity<DT, NT>;
    extern __shared__ __align__(16) unsigned long long buf[];             // kRoom entries, then the stash
    uint4* const stash = reinterpret_cast<uint4*>(buf + kRoom);
    __shared__ Work work;
    __shared__ float2 part[2][NW];
    __shared__ int have_s[2];
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
        auto fetch = [&](uint4 (&w)[U], const uint4* src, int b) {
            src += b * (NT * U) + tid;
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
        // use(block, its number) for all of this thread's blocks, the first `kept` of them from the stash
        auto walk = [&](int kept, auto&& use) {
#pragma unroll 1
            for (int b = 0; b < blocks; ++b) {
                uint4 w[U];
                fetch(w, b < kept ? stash : vec, b);
                use(w, b);
            }
        };
        float m = kFloor, s = 0.0f, largest = -INFINITY;
        walk(0, [&](const uint4 (&w)[U], int b) {
            if (b < plan.stash) {
#pragma unroll
                for (int u = 0; u < U; ++u) stash[b * (NT * U) + u * NT + tid] = w[u];
            }
            float top = vector_max_nan<DT>(w[0]);
#pragma unroll
            for (int u = 1; u < U; ++u) top = max_nan(top, vector_max_nan<DT>(w[u]));
            largest = max_nan(largest, top);
            if (a.lse) {
                const float old = m;
                m = fmaxf(m, top * c2);
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
        });
        // entries at or above the bound are collected
        unsigned long long bound = 0;
        if (tid == 0) work.count = 0;
        if (min(inside, NT) >= a.k) bound = (unsigned long long)bound_of_keys<NT>(tid < inside ? order_of(largest) : 0u, a.k, work) << 32;
        else __syncthreads();
        const float least = bound_value(bound);
        auto offer = [&](float v, long long column) {
            const unsigned long long e = entry_of(v, column);
            if (e >= bound) {
                const int at = atomicAdd(&work.count, 1);
                if (at < kRoom) buf[at] = e;
            }
        };
        walk(plan.stash, [&](const uint4 (&w)[U], int b) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = b * (NT * U) + u * NT + tid;
                if (!(vector_max_nan<DT>(w[u]) < least) && i < inside) offer_vector<DT>(w[u], least, bound, slice.column + (long long)i * V, buf, kRoom, &work.count);
            }
        });
        __syncthreads();
        const bool over = work.count > kRoom - 32;
        __syncthreads();                                  // everybody has read the count that the next function sets back
        if (over) collect_slowly<DT, NT>(buf, work, vec, inside, bound, slice.column, have);
        if (tid < edges) {
            const long long c = slice.edge(tid);
            const float v = to_float(row.base[c]), old = m;
            m = fmaxf(m, v * c2);
            s = s * exp2_fast(old - m) + exp2_fast(fmaf(v, c2, -m));
            offer(v, c);
        }
        __syncthreads();
        if (work.count > max(have, kTopMax)) cut_back<NT>(buf, work, have);
        // this slice's list, sorted by counting the larger ones, and the warps' sums
        const int n = work.count;
        for (int i = tid; i < n; i += NT) work.found[i] = buf[i];
        __syncthreads();
        for (int i = tid; i < n; i += NT) {
            const unsigned long long e = work.found[i];
            int at = 0;
            for (int j = 0; j < n; ++j) at += work.found[j] > e;
            if (at < have) buf[at] = e;
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
            float R = kFloor;
            for (int i = lane; i < C * NW; i += 32) R = fmaxf(R, part_of(i).x);
            R = group_max<32>(R);
            const bool slow = !(fabsf(R) < kReach);
            if (slow) {
                // the largest logit lies out of reach of scaled differences: again, with the difference first
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

template <int DT, int NT> cudaError_t launch_rows(const TopArgs& a, TopPlan plan, cudaStream_t stream) {
    // of an SM's 228 KB each block's share, less its buffer and static arrays
    constexpr int kShare = 226 * 1024 / kBlocks<NT> - kCapacity<DT, NT> * 8 - 5 * 1024;
    plan.stash = (int)std::min<long long>(plan.slice_vectors / (NT * kBlockVectors), std::max(0, kShare) / (NT * kBlockVectors * 16));

    auto kernel = top_kernel<DT, NT>;
    static PerDeviceOnce once;
    cudaLaunchConfig_t cfg = {};
    cfg.blockDim = dim3(NT);
    cfg.gridDim = dim3((unsigned)plan.cluster);
    cfg.dynamicSmemBytes = kCapacity<DT, NT> * sizeof(unsigned long long) + (size_t)plan.stash * NT * kBlockVectors * sizeof(uint4);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)plan.cluster; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cudaError_t e = once.run([&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 200 * 1024); });
    if (e != cudaSuccess) return e;
    // clusters that the device holds at once: asked again only when this thread's last answer was for another shape
    static thread_local struct { int dev, cluster, clusters; size_t smem; } last = {-1, 0, 0, 0};
    int dev = 0;
    if ((e = cudaGetDevice(&dev)) != cudaSuccess) return e;
    if (last.dev != dev || last.cluster != plan.cluster || last.smem != cfg.dynamicSmemBytes) {
        int clusters = 0;
        if ((e = cudaOccupancyMaxActiveClusters(&clusters, kernel, &cfg)) != cudaSuccess) return e;
        last = {dev, plan.cluster, clusters < 1 ? 1 : clusters, cfg.dynamicSmemBytes};
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
    // Short rows by small blocks, of which more are under way (4096 x 1000 bf16: 25 us with 128 threads, 44 with 256); the longest by
    // large ones, whose rows then fit L2 (4096 x 131072 bf16: 335 us with 256, 333 with 512; 64 x 100000: 17.7 and 14.8)
    // A list longer than the block has no bound (too few threads' maxima) and takes in the whole row: as fast where that fits the buffer
    // (4096 x 1000 fp32, k 200: 73 us with 128 threads, 89 with 256; x 1700 bf16: 109 and 120), else not (x 4000 fp32, k 129: 151 and
    // 81; x 8000 bf16, k 200: 294 and 146)
    static_assert(kCapacity<kF32, 128> == kCapacity<kBF16, 128>, "one limit for both types");
    const bool longer = a.k > 128 && a.vocab > kCapacity<kF32, 128> - 32;
    const int nt = vectors > 8192 ? 512 : vectors > 1024 || a.rows <= 2ll * sms || longer ? 256 : 128;
    if (dtype == kF32) return nt == 512 ? launch_rows<kF32, 512>(a, plan, stream) : nt == 128 ? launch_rows<kF32, 128>(a, plan, stream) : launch_rows<kF32, 256>(a, plan, stream);
    return nt == 512 ? launch_rows<kBF16, 512>(a, plan, stream) : nt == 128 ? launch_rows<kBF16, 128>(a, plan, stream) : launch_rows<kBF16, 256>(a, plan, stream);
}

}  // namespace tmask
