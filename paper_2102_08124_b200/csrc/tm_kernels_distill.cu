// Distillation from a teacher's list of largest logits: loss, gradient, or both.
//
//   q = softmax(z / T) over the row;  p = softmax(v / T) over the list's entries, or, where the teacher's log-sum-exp L is
//   given, p_k = exp(v_k / T - L) and p_rest = max(0, 1 - sum_k p_k) for everything the list leaves out (q_rest: the student's)
//   loss      = f [ sum_k p_k (log p_k - log q_k) + p_rest (log p_rest - log q_rest) ],   f = scale * row weight
//   dloss/dz  = f / T (q_j - p_j) for a listed logit,  f / T (q_j - p_rest q_j / q_rest) for another one
//
// q_rest is the sum over the unlisted logits themselves, never one minus the listed mass: the difference would lose all its
// digits where the student puts nearly everything on the list.  The unlisted logits' sum has a reference of its own, the largest of them,
// so that log q_rest is right however far they lie below the listed ones, and an unlisted gradient is written as
// f / T (q_rest - p_rest) (q_j / q_rest), whose last factor is a softmax over the unlisted logits alone.
// Terms with p = 0 are left out, and so is the rest's term where the student has no mass there: unlisted logits of -Inf, or more than
// 2^20 binades below the listed ones, which only masks are.
#include <algorithm>
#include <type_traits>

#include "tm_launch.h"
#include "tm_rows.cuh"

namespace tmask {

namespace {

constexpr double kLog2eD = 1.4426950408889634074, kLn2D = 0.69314718055994530942;

__device__ __forceinline__ double warp_sum_double(double v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}

constexpr int kHash = 512, kEntries = kTopMax / 32;      // slots of the table that finds repeated ids; entries of a lane

__device__ __forceinline__ float lowest() { return -3.4028234663852886e38f; }

// 2^(x - R) of a logit: `slow` rows (R out of the reach of scaled differences) have R in logits and take the difference first.
__device__ __forceinline__ float power_of(float z, float R, bool slow, float c2) { return exp2_fast(slow ? (z - R) * c2 : fmaf(z, c2, -R)); }

constexpr float kMasked = 1048576.0f;                    // less than kReach above kFloor: binades below the listed logits from which unlisted ones count as masked

// What a row's gradient needs beside its list, in units of f / T: 2^(x - R) inv - p for a listed logit, 2^(x - R_rest) rest for another one.
struct Scale { float R, inv, R_rest, rest; bool slow; };
// The sums of a row: over the unlisted and the listed logits, each relative to the largest of them.
struct Sums { float R_rest, s_rest, R_list, s_list; };
// s_rest becomes 0 where the unlisted logits count as masked.  Returns the sum over the whole row, relative to the R that it sets.
__device__ __forceinline__ float scale_of_sums(Sums& s, float p_rest, bool slow, float c2, Scale& k) {
    const float unit = slow ? c2 : 1.0f;                  // binades of a difference of references
    k.slow = slow;
    k.R = fmaxf(s.R_rest, s.R_list);
    const float gap = (k.R - s.R_rest) * unit, s_all = s.s_rest * exp2_fast(-gap) + s.s_list * exp2_fast((s.R_list - k.R) * unit);
    if (!(gap < kMasked) && s.s_rest == s.s_rest) s.s_rest = 0.0f;
    k.inv = 1.0f / s_all;
    k.R_rest = k.R;
    k.rest = k.inv;
    if (p_rest > 0.0f && s.s_rest > 0.0f) {
        k.R_rest = s.R_rest;
        k.rest = exp2_fast(-gap) * k.inv - p_rest / s.s_rest;                  // (q_rest - p_rest) / s_rest
    }
    return s_all;
}
// The same from the statistics.  unit: what a log-sum-exp in units of T is in scaled logits x = z c2, that is c2 T (log2(e) but for c2's rounding).
__device__ __forceinline__ Scale scale_of_stats(float lse, float log_rest, float p_rest, double unit) {
    // q = 2^(x - R) 2^(R - lse unit): the second factor, of R's rounding, joins the others
    const double want = (double)lse * unit;
    Scale k;
    k.slow = false;
    k.R = (float)want;
    k.inv = exp2f((float)((double)k.R - want));
    k.R_rest = k.R;
    k.rest = k.inv;
    if (p_rest > 0.0f && log_rest > -kMasked * (float)kLn2D) {
        // the same for q_j / q_rest, whose logarithm is x less the sum of the two statistics
        const double want_rest = ((double)lse + log_rest) * unit;
        k.R_rest = (float)want_rest;
        k.rest = (expf(log_rest) - p_rest) * exp2f((float)((double)k.R_rest - want_rest));
    }
    return k;
}

// A log-sum-exp in fp32 is off by up to 2^-24 of itself, and so are then all q = exp(z / T - lse), relatively; the same goes for log q_rest and
// q_j / q_rest.  Beyond this size of either (2^-14) a row's sums are taken again from its logits.
constexpr float kFarLse = 1024.0f;

// The sums of a whole row in logits, by all threads of a block; listed logits are told by their ids in the table (kHash words of -1, left
// so).  For the few rows whose statistics are not enough: it goes through them an element a thread (were all rows of 2048 x 32001 such, the
// gradient would take 433 us in fp32 and 368 in bf16, instead of 94 and 54).
template <int DT, int THREADS> __device__ __noinline__ Sums sums_of_row(const typename RowType<DT>::T* base, int n, const int* ids, int slots, int* hash, float c2, Sums* part) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const auto slot_of = [](int id) { return (int)(((uint32_t)id * 2654435769u) >> 23); };
    for (int i = tid; i < slots; i += THREADS) {
        const int id = ids[i];
        if (id >= 0 && id < n) {
            int h = slot_of(id);
            for (int probe = 0; probe < kHash; ++probe, h = (h + 1) & (kHash - 1)) {
                const int old = atomicCAS(&hash[h], -1, id);
                if (old == -1 || old == id) break;
            }
        }
    }
    __syncthreads();
    float2 sum[2] = {make_float2(lowest(), 0.0f), make_float2(lowest(), 0.0f)};            // unlisted, listed: the largest logit, the sum relative to it
    const auto add = [&](float2& a, float v) {
        if (v > a.x) a = make_float2(v, fmaf(a.y, exp2_fast((a.x - v) * c2), 1.0f));
        else a.y += exp2_fast((v - a.x) * c2);
    };
    for (int c = tid; c < n; c += THREADS) {
        int h = slot_of(c);
        while (hash[h] != -1 && hash[h] != c) h = (h + 1) & (kHash - 1);                  // at most kTopMax of the kHash words are taken
        if (hash[h] == c) add(sum[1], to_float(base[c]));
        else add(sum[0], to_float(base[c]));
    }
    Sums s;
    s.R_rest = group_max<32>(sum[0].x);
    s.R_list = group_max<32>(sum[1].x);
    s.s_rest = group_sum<32>(sum[0].y * exp2_fast((sum[0].x - s.R_rest) * c2));
    s.s_list = group_sum<32>(sum[1].y * exp2_fast((sum[1].x - s.R_list) * c2));
    if (lane == 0) part[warp] = s;
    __syncthreads();
    for (int i = tid; i < kHash; i += THREADS) hash[i] = -1;
    for (int i = 0; i < THREADS / 32; ++i) { s.R_rest = fmaxf(s.R_rest, part[i].R_rest); s.R_list = fmaxf(s.R_list, part[i].R_list); }
    s.s_rest = s.s_list = 0.0f;
    for (int i = 0; i < THREADS / 32; ++i) {
        s.s_rest += part[i].s_rest * exp2_fast((part[i].R_rest - s.R_rest) * c2);
        s.s_list += part[i].s_list * exp2_fast((part[i].R_list - s.R_list) * c2);
    }
    if (!(fmaxf(s.R_rest, s.R_list) < INFINITY)) s.s_rest = s.s_list = __uint_as_float(0x7FC00000u);
    __syncthreads();
    return s;
}

// A row's list, entry e * 32 + lane in the lanes of one warp: unusable entries (padding, out of range, repeated) get id -1.
struct List {
    int id[kEntries];
    float p[kEntries];     // the teacher's probability (its logit until probabilities() ran)
    float entropy;         // sum p (log p + log norm)
    float norm;            // what the exponentials were divided by (1 where the teacher's log-sum-exp is given)
    float rest;            // p_rest
    bool some;             // any entry

    // between rows and barriers a list waits in shared memory: ids and values, kTopMax each
    __device__ __forceinline__ void load(const int* ids, const float* values, int slots) {
        const int lane = threadIdx.x & 31;
#pragma unroll
        for (int e = 0; e < kEntries; ++e) {
            id[e] = -1; p[e] = 0.0f;
            if (e * 32 < slots) { id[e] = ids[e * 32 + lane]; p[e] = values[e * 32 + lane]; }
        }
    }
    // true if an entry was out of range or repeated.  `hash`: kHash words of -1 (left so), this warp's own.
    __device__ __forceinline__ bool weed(const DistillArgs& a, int slots, int* hash) {
        const int lane = threadIdx.x & 31;
        bool bad = false, again = false;
        int at[kEntries];
#pragma unroll
        for (int e = 0; e < kEntries; ++e)
            if (id[e] >= a.vocab) { id[e] = -1; bad = true; }
        // the table tells whether ids repeat at all; only then the first of each is looked for
#pragma unroll
        for (int e = 0; e < kEntries; ++e) {
            at[e] = -1;
            if (e * 32 < slots && id[e] >= 0) {
                int h = (int)(((uint32_t)id[e] * 2654435769u) >> 23);
                for (int probe = 0; probe < kHash; ++probe) {
                    const int old = atomicCAS(&hash[h], -1, id[e]);
                    if (old == -1) { at[e] = h; break; }
                    if (old == id[e]) { again = true; break; }
                    h = (h + 1) & (kHash - 1);
                }
            }
        }
        __syncwarp();
#pragma unroll
        for (int e = 0; e < kEntries; ++e)
            if (at[e] >= 0) hash[at[e]] = -1;
        __syncwarp();
        if (__any_sync(0xFFFFFFFFu, again)) {
            int gone = 0;                                 // bit e: an earlier entry has this id
#pragma unroll
            for (int j = 0; j < kEntries; ++j) {
                if (j * 32 >= slots) break;
                for (int l = 0; l < 32; ++l) {
                    const int other = __shfl_sync(0xFFFFFFFFu, id[j], l);
#pragma unroll
                    for (int e = 0; e < kEntries; ++e)
                        if (id[e] == other && j * 32 + l < e * 32 + lane) gone |= 1 << e;
                }
            }
#pragma unroll
            for (int e = 0; e < kEntries; ++e)
                if (gone >> e & 1) id[e] = -1;
        }
        return bad | again;
    }
    // log p = (v - top) / T - log norm, or v / T - lse with one rounding of the difference (1 / T = it + it_low)
    __device__ __forceinline__ void probabilities(const DistillArgs& a, float weight, float lse_t, float it, float it_low) {
        float top = -INFINITY;
        some = false;
        float mass = 0.0f;
        entropy = rest = 0.0f;
        norm = 1.0f;
#pragma unroll
        for (int e = 0; e < kEntries; ++e)
            if (id[e] >= 0) { some = true; top = fmaxf(top, p[e]); }
        some = __any_sync(0xFFFFFFFFu, some) && weight != 0.0f;
        if (!some) return;
        float log_p[kEntries];
        const bool own = !a.teacher_lse;
        if (own) top = group_max<32>(top);
#pragma unroll
        for (int e = 0; e < kEntries; ++e) {
            log_p[e] = 0.0f;
            if (id[e] >= 0) {
                log_p[e] = own ? (p[e] - top) * it : fmaf(p[e], it, -lse_t) + (p[e] > -INFINITY ? p[e] * it_low : 0.0f);
                p[e] = expf(log_p[e]);
            } else p[e] = 0.0f;
            mass += p[e];
        }
        mass = group_sum<32>(mass);
        float scale = 1.0f;
        if (own) {
            norm = mass;
            scale = 1.0f / norm;
        } else rest = fmaxf(0.0f, 1.0f - mass);
#pragma unroll
        for (int e = 0; e < kEntries; ++e) {
            p[e] *= scale;
            if (p[e] != 0.0f) entropy = fmaf(p[e], log_p[e], entropy);
        }
        entropy = group_sum<32>(entropy);
    }
};

// One warp: row r's list as given into shared memory (entries past it as padding).
__device__ __forceinline__ void fetch_list(const DistillArgs& a, long long r, int slots, int* ids, float* values) {
    for (int k = threadIdx.x & 31; k < slots; k += 32) {
        const bool in = k < a.k;
        ids[k] = in ? a.ids[r * a.k + k] : -1;
        values[k] = in ? a.values[r * a.k + k] : 0.0f;
    }
    __syncwarp();
}

// What a block's listed logits add to the loss: sum p and sum p (z - z0), z0 the largest of them.  entropy, norm: the list's.
struct ListSums { double dot; float mass, z0, entropy, norm; };

// A row's loss, by one warp: sum p log p - sum p log q + p_rest (log p_rest - log q_rest), put together in 64 bits because the sums
// nearly cancel: an offset that all logits share drops out of (z0 - R) before anything is rounded.  Lane c < C brings block c's ListSums
// (entropy and norm: those of any block).  The four logs are taken side by side in four lanes.  The exponentials' sums are relative to
// R base_unit in units of the temperature, or to R itself where `slow`; R_rest: the rest's reference.  Lane 0 returns the loss, and the statistics.
__device__ __forceinline__ float row_loss(float rest, const ListSums& l, int C, bool slow, double inv_t, double base_unit, float R, float R_rest, float s_all, float s_rest,
                                          float& lse, float& log_rest) {
    const int lane = threadIdx.x & 31;
    const double unit = slow ? inv_t : base_unit;
    const double above = slow ? ((double)l.z0 - R) * inv_t : l.z0 * inv_t - R * base_unit;       // z0 / T - base
    float mass = l.mass;
    double cross = l.dot * inv_t + (mass > 0.0f ? mass * above : 0.0);                           // sum p (z / T - base)
    if (C > 1) {
        mass = group_sum<32>(lane < C ? mass : 0.0f);
        cross = warp_sum_double(lane < C ? cross : 0.0);
    }
    const double log_all = log((double)(lane == 0 ? s_all : lane == 1 ? s_rest : lane == 2 ? rest : l.norm));      // lane 0's
    const double log_s = __shfl_sync(0xFFFFFFFFu, log_all, 1), log_r = __shfl_sync(0xFFFFFFFFu, log_all, 2), log_n = __shfl_sync(0xFFFFFFFFu, log_all, 3);
    const double log_rest_d = log_s - log_all - ((double)R - R_rest) * unit;
    double loss = (double)l.entropy - mass * log_n - cross + mass * log_all;
    if (rest > 0.0f && s_rest > 0.0f) loss += rest * (log_r - log_rest_d);
    if (s_rest != s_rest) loss = s_rest;
    lse = (float)(R * unit + log_all);
    log_rest = (float)log_rest_d;
    return (float)loss;
}

// ---- a row by a cluster of thread blocks -----------------------------------------------------------------------------
//
// Bound: HBM, with the exponentials close behind (a logit costs one in the loss and one in the gradient; the units that make them
// give 16 a clock and SM).  C blocks share a row, a slice each: NT workers and one warp for the list.
//   pass 1  the workers' running maximum and sum over their vectors of the slice; meanwhile the list's warp works out the teacher's
//           probabilities and the listed logits' part.  Listed logits stay out of the workers' sum by a byte of flags for every
//           vector in shared memory, which is zero nearly always.
//   totals  the warps' partial results, by shared memory (of the whole cluster)
//   pass 2  the gradient, from the copy of the slice that pass 1 left in shared memory: a row is read once.  Meanwhile the list's
//           warp puts the loss together; after the pass it writes the listed logits' gradients.
// Several blocks share an SM, so one's loads cover another's exponentials and waits.
// Exponents live in base 2, scaled: x_j = z_j c2 with c2 = log2(e) / T, as differences x_j - R with one rounding (fma), R the largest
// x.  A row whose R is out of their reach (all logits masked, say) goes again with differences of the logits first.

constexpr int kMaxCluster = 8;
constexpr size_t kRowSmem = 216 * 1024;            // of a block's 227 KB, beside the static arrays

struct RowPlan {
    int cluster, slots;            // slots: list entries, a multiple of 32
    int slice_vectors, flags;      // flags: bytes, a multiple of 16 (0 without a loss)
    int stash;                     // blocks of NT * U vectors that stay in shared memory between the passes
    float inv_t, inv_t_low, c2;    // 1 / T and what its rounding left out; log2(e) / T
    double inv_t_d, kappa, unit;   // 1 / T; (log2(e) / T) / c2, the rounding of c2; c2 T
};

constexpr int kBlockVectors = 4;                   // vectors of a thread's block
// Blocks an SM, that is the registers a thread may use.  256 threads: the loss of 2048 x 32001 fp32 takes 65 us with three blocks and 67 with
// four, the gradient alone in bf16 58.7 and 54.4.  128 threads, six blocks and eight (ptxas then spills 410 bytes of the loss, and 48 to 52
// of the two other forms): the loss of 4000 x 4000 fp32 32.8 and 34.7 us, 4096 x 8000 bf16 42.0 and 43.0, but 4096 x 1000 bf16, whose time
// is the list's, 33.4 and 32.5; loss and gradient 46.1 and 39.8, 55.9 and 51.5; the gradient alone of 4096 x 8000 bf16 37.9 and 35.8.
template <bool LOSS, bool GRAD, int NT> constexpr int kBlocks = NT == 512 ? 2 : NT == 256 ? (LOSS ? 3 : 4) : LOSS && !GRAD ? 6 : 8;

template <int DT, bool LOSS, bool GRAD, int NT>
__global__ void __launch_bounds__(NT + 32, kBlocks<LOSS, GRAD, NT>) distill_kernel(const DistillArgs a, const RowPlan plan) {
    using T = typename RowType<DT>::T;
    constexpr int V = RowType<DT>::kVec, NW = NT / 32, U = kBlockVectors;
    extern __shared__ __align__(16) uint8_t dynamic[];
    uint8_t* const flags = dynamic;
    uint4* const stash = reinterpret_cast<uint4*>(dynamic + plan.flags);
    __shared__ int hash[kHash];
    __shared__ int list_id[kTopMax];                                      // the row's list as given, then without what was weeded out
    __shared__ float list_v[kTopMax];
    __shared__ int list_at[kTopMax];                                      // ids of this slice's listed logits, or -1
    __shared__ float list_p[kTopMax], list_z[kTopMax];
    __shared__ float2 part[2][NW], list_part[2];
    __shared__ ListSums list_sums[2];
    __shared__ Sums far_part[NW + 1];
    __shared__ float rest_s;
    __shared__ int on_s;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const bool lister = warp == NW;
    const int C = plan.cluster, slots = plan.slots;
    const uint32_t rank = C > 1 ? cluster_rank() : 0u;
    const float inv_t = plan.inv_t, c2 = plan.c2;
    const long long step = gridDim.x / C;
    for (int i = tid; i < kHash; i += NT + 32) hash[i] = -1;
    for (int i = tid; i < plan.flags / 16; i += NT + 32) reinterpret_cast<uint4*>(flags)[i] = make_uint4(0u, 0u, 0u, 0u);
    int turn = 0;
    float next_weight = 1.0f;                                             // read a row ahead, as is the list
    uint4 w[U];
    const long long start = blockIdx.x / C;
    if (start < a.rows) {
        if (a.row_weight) next_weight = a.row_weight[start];
        if (lister) fetch_list(a, start, slots, list_id, list_v);
    }
    __syncthreads();

    for (long long r = start; r < a.rows; r += step) {
        const RowVectors<DT> row(static_cast<const T*>(a.logits) + r * a.ld, a.vocab);
        const long long from = min(row.count, (long long)rank * plan.slice_vectors), to = min(row.count, from + plan.slice_vectors);
        const RowPart<DT> slice(row, from, to);
        const uint4* const vec = reinterpret_cast<const uint4*>(row.base + slice.column);
        const int inside = slice.inside, edges = slice.head + slice.tail;
        T* const out = GRAD ? static_cast<T*>(a.dlogits) + r * a.ld_d : nullptr;
        const float weight = next_weight;
        if (a.row_weight && r + step < a.rows) next_weight = a.row_weight[r + step];
        // A thread's vectors come in blocks of U, NT apart; all blocks but the last are whole.  The first one is on its way while the list is read.
        const int whole = inside / (NT * U), blocks = (inside + NT * U - 1) / (NT * U);
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
        // use(block, its number) for all of this thread's blocks, the first `kept` of them from the stash; block 0 is in `w`
        auto walk = [&](int kept, auto&& use) {
#pragma unroll 1
            for (int b = 0; b < blocks; ++b) {
                if (b > 0) fetch(w, b < kept ? stash : vec, b);
                use(w, b);
            }
        };
        if (lister) {
            List list;
            list.load(list_id, list_v, slots);
            if (list.weed(a, slots, hash) && rank == 0 && weight != 0.0f && a.status) atomicOr(a.status, kDevBadId);
            bool some = false;
            const long long c0 = max(0ll, row.column(from)), c1 = row.column(to);
#pragma unroll
            for (int e = 0; e < kEntries; ++e) {
                if (e * 32 >= slots) break;
                some |= list.id[e] >= 0;
                const bool here = list.id[e] >= c0 && list.id[e] < c1 && list.id[e] >= 0;
                list_at[e * 32 + lane] = here ? list.id[e] : -1;
                if (LOSS) list_id[e * 32 + lane] = list.id[e];
                const long long place = (long long)list.id[e] - slice.column;             // among the full vectors
                if (LOSS && here && place >= 0 && place < (long long)inside * V)
                    atomicOr(reinterpret_cast<uint32_t*>(flags) + (uint32_t)place / (4 * V), 1u << ((uint32_t)place / V % 4 * 8 + (uint32_t)place % V));
            }
            some = __any_sync(0xFFFFFFFFu, some) && weight != 0.0f;
            if (lane == 0) on_s = some;
            if (!LOSS) {
                list.probabilities(a, weight, a.teacher_lse ? a.teacher_lse[r] : 0.0f, inv_t, plan.inv_t_low);
                if (lane == 0) rest_s = list.rest;
#pragma unroll
                for (int e = 0; e < kEntries; ++e)
                    if (e * 32 < slots) {
                        const int i = e * 32 + lane;
                        list_p[i] = list.p[e];
                        list_z[i] = list_at[i] >= 0 ? to_float(row.base[list_at[i]]) : 0.0f;   // before anything is written: dlogits may be the logits
                    }
            }
        } else {
            if (weight != 0.0f && blocks > 0) fetch(w, vec, 0);
        }
        __syncthreads();
        const bool on = on_s;
        auto unflag = [&](int e) {                        // the lister clears what it set
            const long long place = (long long)list_at[e] - slice.column;
            if (list_at[e] >= 0 && place >= 0 && place < (long long)inside * V) reinterpret_cast<uint32_t*>(flags)[(uint32_t)place / (4 * V)] = 0u;
        };
        // the gradient's full vectors and edge elements: what(vector or element) as stored
        const bool same = GRAD && ((reinterpret_cast<uintptr_t>(out) ^ reinterpret_cast<uintptr_t>(row.base)) & 15) == 0;
        auto put = [&](int i, const uint32_t (&q)[4]) {
            if (same) __stcs(reinterpret_cast<uint4*>(out + slice.column) + i, make_uint4(q[0], q[1], q[2], q[3]));
            else {
                float v[V];
                unpack_words<DT, 4>(q, v);
#pragma unroll
                for (int j = 0; j < V; ++j) from_float(out + slice.column + (long long)i * V + j, v[j]);
            }
        };
        if (!on) {
            if (LOSS && rank == 0 && tid == 0) {
                a.loss[r] = 0.0f;
                if (!GRAD && a.stats) a.stats[2 * r] = a.stats[2 * r + 1] = 0.0f;
            }
            if constexpr (GRAD) {
                const uint32_t zero[4] = {0u, 0u, 0u, 0u};
                if (!lister) {
                    for (int i = tid; i < inside; i += NT) put(i, zero);
                    if (tid < edges) from_float(out + slice.edge(tid), 0.0f);
                }
            }
            if (lister && r + step < a.rows) fetch_list(a, r + step, slots, list_id, list_v);
            if (LOSS && lister) for (int e = lane; e < slots; e += 32) unflag(e);
            __syncthreads();
            continue;
        }
        Scale k;
        float rest;
        if constexpr (LOSS) {
            Sums sums;
            float m = kFloor, s = 0.0f;
            // the largest m of the workers' (m, s) and of the lists', each with the sums relative to it
            auto totals = [&]() {
                const float wm = group_max<32>(m);
                const float ws = group_sum<32>(s * exp2_fast(m - wm));
                if (lane == 0) {
                    if (lister) list_part[turn] = make_float2(wm, ws);
                    else part[turn][warp] = make_float2(wm, ws);
                }
                __syncwarp();
                if (C > 1) cluster_sync(); else __syncthreads();
                float top = lowest();
                for (int i = lane; i < C * NW; i += 32) top = fmaxf(top, (C > 1 ? cluster_load2(&part[turn][i % NW], i / NW) : part[turn][i]).x);
                sums.R_rest = group_max<32>(top);
                float sum = 0.0f;
                for (int i = lane; i < C * NW; i += 32) {
                    const float2 v = C > 1 ? cluster_load2(&part[turn][i % NW], i / NW) : part[turn][i];
                    sum += v.y * exp2_fast(v.x - sums.R_rest);
                }
                sums.s_rest = group_sum<32>(sum);
                if (C > 1) {
                    const float2 of_list = lane < C ? cluster_load2(&list_part[turn], lane) : make_float2(lowest(), 0.0f);
                    sums.R_list = group_max<32>(of_list.x);
                    sums.s_list = group_sum<32>(of_list.y * exp2_fast(of_list.x - sums.R_list));
                } else { sums.R_list = list_part[turn].x; sums.s_list = list_part[turn].y; }
                turn ^= 1;
            };
            // listed elements of a vector become -Inf
            auto mask = [&](uint4& q, uint32_t f) {
                uint32_t v[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
                for (int j = 0; j < V; ++j)
                    if (f >> j & 1u) {
                        if constexpr (DT == kF32) v[j] = 0xFF800000u;
                        else v[j / 2] = j & 1 ? (v[j / 2] & 0xFFFFu) | 0xFF800000u : (v[j / 2] & 0xFFFF0000u) | 0xFF80u;
                    }
                q = make_uint4(v[0], v[1], v[2], v[3]);
            };
            // this thread's vectors, listed elements masked, a block at a time (absent vectors are -Inf)
            auto each = [&](auto&& use, bool keep) {
                walk(0, [&](uint4 (&now)[U], int b) {
                    const int i0 = b * (NT * U) + tid;
                    const uint8_t* fl = flags + i0;
                    uint32_t f[U];
                    if (b < whole) {
#pragma unroll
                        for (int u = 0; u < U; ++u) f[u] = fl[u * NT];
                    } else {
#pragma unroll
                        for (int u = 0; u < U; ++u) f[u] = i0 + u * NT < inside ? fl[u * NT] : 0u;
                    }
                    if (keep && b < plan.stash) {
#pragma unroll
                        for (int u = 0; u < U; ++u) stash[i0 + u * NT] = now[u];
                    }
                    if ((f[0] | f[1] | f[2] | f[3]) != 0u) {
#pragma unroll
                        for (int u = 0; u < U; ++u) if (f[u] != 0u) mask(now[u], f[u]);
                    }
                    use(now);
                });
                if (tid < edges) {                        // at most one element a thread, as a vector of its own
                    const long long c = slice.edge(tid);
                    bool listed = false;
                    for (int e = 0; e < slots; ++e) listed |= list_at[e] == c;
                    uint4 now[U];
#pragma unroll
                    for (int u = 0; u < U; ++u) now[u] = make_uint4(RowType<DT>::kLow, RowType<DT>::kLow, RowType<DT>::kLow, RowType<DT>::kLow);
                    if (!listed) {
                        if constexpr (DT == kF32) now[0].x = __float_as_uint(row.base[c]);
                        else now[0].x = (RowType<DT>::kLow & 0xFFFF0000u) | (uint32_t)__bfloat16_as_ushort(row.base[c]);
                    }
                    use(now);
                }
            };
            if (lister) {
                List list;
                list.load(list_id, list_v, slots);
                list.probabilities(a, weight, a.teacher_lse ? a.teacher_lse[r] : 0.0f, inv_t, plan.inv_t_low);
                float z[kEntries], z0 = -INFINITY;
#pragma unroll
                for (int e = 0; e < kEntries; ++e) {
                    if (e * 32 >= slots) break;
                    const int id = list_at[e * 32 + lane];
                    z[e] = id >= 0 ? to_float(row.base[id]) : -INFINITY;
                    list_p[e * 32 + lane] = list.p[e];
                    list_z[e * 32 + lane] = z[e];
                    z0 = fmaxf(z0, z[e]);
                }
                m = fmaxf(m, z0 * c2);
                z0 = group_max<32>(z0);
                if (!(z0 > -INFINITY)) z0 = 0.0f;
                float mass = 0.0f;
                double dot = 0.0;
#pragma unroll
                for (int e = 0; e < kEntries; ++e) {
                    if (e * 32 >= slots) break;
                    s += exp2_fast(fmaf(z[e], c2, -m));
                    if (list_at[e * 32 + lane] >= 0 && list.p[e] != 0.0f) {
                        mass += list.p[e];
                        dot += (double)list.p[e] * ((double)z[e] - z0);
                    }
                }
                mass = group_sum<32>(mass);
                dot = warp_sum_double(dot);
                if (lane == 0) { rest_s = list.rest; list_sums[turn] = {dot, mass, z0, list.entropy, list.norm}; }
            } else {
                float2 add = make_float2(0.0f, 0.0f);
                const float2 cc = make_float2(c2, c2);
                each([&](const uint4 (&now)[U]) {
                    float top = vector_max<DT>(now[0]);
#pragma unroll
                    for (int u = 1; u < U; ++u) top = fmaxf(top, vector_max<DT>(now[u]));
                    const float old = m;
                    m = fmaxf(m, top * c2);
                    const float move = exp2_fast(old - m);
                    add = __fmul2_rn(add, make_float2(move, move));
                    const float2 mm = make_float2(-m, -m);
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        float v[V];
                        unpack_vector<DT>(now[u], v);
#pragma unroll
                        for (int j = 0; j < V; j += 2) {
                            const float2 x = __ffma2_rn(make_float2(v[j], v[j + 1]), cc, mm);
                            add = __fadd2_rn(add, make_float2(exp2_fast(x.x), exp2_fast(x.y)));
                        }
                    }
                }, GRAD);
                s = add.x + add.y;
            }
            totals();
            const bool slow = !(fabsf(fmaxf(sums.R_rest, sums.R_list)) < kReach);
            if (slow) {
                // the largest logit lies out of reach of scaled differences: the largest ones as they are, then the sums
                m = lowest(); s = 0.0f;
                if (lister) { for (int e = lane; e < slots; e += 32) m = fmaxf(m, list_z[e]); }
                else { if (blocks > 0) fetch(w, vec, 0); each([&](const uint4 (&now)[U]) { for (int u = 0; u < U; ++u) m = fmaxf(m, vector_max<DT>(now[u])); }, false); }
                totals();
                const float M_rest = sums.R_rest, M_list = sums.R_list;
                m = 0.0f; s = 0.0f;
                if (lister) { for (int e = lane; e < slots; e += 32) s += exp2_fast((list_z[e] - M_list) * c2); }
                else {
                    if (blocks > 0) fetch(w, vec, 0);
                    each([&](const uint4 (&now)[U]) {
                        for (int u = 0; u < U; ++u) {
                            float v[V];
                            unpack_vector<DT>(now[u], v);
                            for (int j = 0; j < V; ++j) s += exp2_fast((v[j] - M_rest) * c2);
                        }
                    }, false);
                }
                totals();
                sums.R_rest = M_rest; sums.R_list = M_list;
            }
            rest = rest_s;
            const float s_all = scale_of_sums(sums, rest, slow, c2, k);
            if (lister) {
                for (int e = lane; e < slots; e += 32) unflag(e);
                __syncwarp();
                if (r + step < a.rows) fetch_list(a, r + step, slots, list_id, list_v);
            }
            if (lister && rank == 0) {
                float lse, log_rest;
                const ListSums* const from = &list_sums[turn ^ 1];        // as turn was in pass 1: one round of totals, or three
                ListSums l = *from;
                if (C > 1) {
                    const uint32_t c = lane < C ? lane : 0;
                    l.mass = cluster_load_float(&from->mass, c);
                    l.dot = cluster_load_double(&from->dot, c);
                    l.z0 = cluster_load_float(&from->z0, c);
                }
                const float loss = row_loss(rest, l, C, k.slow, plan.inv_t_d, plan.kappa * kLn2D, k.R, sums.R_rest, s_all, sums.s_rest, lse, log_rest);
                if (lane == 0) {
                    a.loss[r] = loss * weight * a.scale;
                    if (!GRAD && a.stats) { a.stats[2 * r] = lse; a.stats[2 * r + 1] = a.teacher_lse ? log_rest : 0.0f; }
                }
            }
        } else {
            rest = rest_s;
            const float lse = a.stats[2 * r], log_rest = a.stats[2 * r + 1];
            const bool far_rest = rest > 0.0f && log_rest < -kFarLse && log_rest > -kMasked * (float)kLn2D;
            if (fabsf(lse) < kFarLse && !far_rest) k = scale_of_stats(lse, log_rest, rest, plan.unit);
            else {
                Sums sums = sums_of_row<DT, NT + 32>(row.base, (int)a.vocab, list_id, slots, hash, c2, far_part);
                scale_of_sums(sums, rest, true, c2, k);
                if (C > 1) cluster_sync();                // dlogits may be the logits, of which every block has read the whole row
            }
            if (lister && r + step < a.rows) fetch_list(a, r + step, slots, list_id, list_v);
        }
        if constexpr (GRAD) {
            const float up = weight * a.scale * (!LOSS && a.grad_loss ? a.grad_loss[r] : 1.0f) * inv_t, scale = up * k.rest;
            if (!lister) {
                const int kept = LOSS ? plan.stash : 0;
                if (LOSS && blocks > 0) fetch(w, kept > 0 ? stash : vec, 0);
                const float2 cc = make_float2(c2, c2), rr = make_float2(-k.R_rest, -k.R_rest), ss = make_float2(scale, scale);
                auto pass = [&](auto&& power2) {
                    walk(kept, [&](uint4 (&now)[U], int b) {
                        const int i0 = b * (NT * U) + tid;
#pragma unroll
                        for (int u = 0; u < U; ++u) {
                            float v[V];
                            uint32_t q[4];
                            unpack_vector<DT>(now[u], v);
#pragma unroll
                            for (int j = 0; j < V; j += 2) {
                                const float2 g = __fmul2_rn(power2(make_float2(v[j], v[j + 1])), ss);
                                v[j] = g.x; v[j + 1] = g.y;
                            }
                            pack_words<DT, 4>(v, q);
                            if (b < whole || i0 + u * NT < inside) put(i0 + u * NT, q);
                        }
                    });
                };
                if (!k.slow) pass([&](float2 z) { const float2 x = __ffma2_rn(z, cc, rr); return make_float2(exp2_fast(x.x), exp2_fast(x.y)); });
                else pass([&](float2 z) { return make_float2(power_of(z.x, k.R_rest, true, c2), power_of(z.y, k.R_rest, true, c2)); });
                if (tid < edges) from_float(out + slice.edge(tid), scale * power_of(to_float(row.base[slice.edge(tid)]), k.R_rest, k.slow, c2));
            }
            __syncthreads();
            if (lister)
                for (int e = lane; e < slots; e += 32)
                    if (list_at[e] >= 0) from_float(out + list_at[e], up * fmaf(power_of(list_z[e], k.R, k.slow, c2), k.inv, -list_p[e]));
        }
    }
    if (LOSS && C > 1) cluster_sync();                    // nobody's shared memory goes while others may still read it
}

template <int DT, bool LOSS, bool GRAD, int NT> cudaError_t launch_rows(const DistillArgs& a, const RowPlan& plan, cudaStream_t stream) {
    auto kernel = distill_kernel<DT, LOSS, GRAD, NT>;
    static PerDeviceOnce once;
    cudaError_t e = once.run([&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kRowSmem); });
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.blockDim = dim3(NT + 32);
    cfg.gridDim = dim3((unsigned)plan.cluster);
    cfg.dynamicSmemBytes = (size_t)plan.flags + (size_t)plan.stash * NT * kBlockVectors * 16;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)plan.cluster; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
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

template <int DT, bool LOSS, bool GRAD, int NT> cudaError_t launch_as(const DistillArgs& a, RowPlan plan, cudaStream_t stream) {
    // a block's share of an SM's 228 KB for the stash, less its flags and static arrays
    constexpr int kBlockBytes = NT * kBlockVectors * 16, kShare = 226 * 1024 / kBlocks<LOSS, GRAD, NT> - 9 * 1024;
    plan.stash = LOSS && GRAD ? std::max(0, std::min(plan.slice_vectors / (NT * kBlockVectors), (kShare - plan.flags) / kBlockBytes)) : 0;
    return launch_rows<DT, LOSS, GRAD, NT>(a, plan, stream);
}

template <bool LOSS, bool GRAD> cudaError_t launch(const DistillArgs& a, int dtype, int sms, cudaStream_t stream) {
    const int e = dtype == kF32 ? 4 : 2, V = 16 / e;
    const long long vectors = std::max<long long>(1, (a.vocab + 2 * V - 2) / V);      // of a row, wherever it starts
    RowPlan plan;
    plan.slots = (a.k + 31) / 32 * 32;
    plan.inv_t_d = 1.0 / (double)a.temperature;
    plan.inv_t = (float)plan.inv_t_d;
    plan.inv_t_low = (float)(plan.inv_t_d - (double)plan.inv_t);
    plan.c2 = (float)(kLog2eD / a.temperature);
    plan.kappa = kLog2eD / a.temperature / (double)plan.c2;
    plan.unit = (double)plan.c2 * a.temperature;
    // Several blocks to a row where the rows alone do not fill the device (a row of 131072 bf16 logits: 14 us on one block, 11.4 us on
    // eight), and where a row is longer than 256 KB
    plan.cluster = 1;
    while (plan.cluster < kMaxCluster && (vectors + plan.cluster - 1) / plan.cluster > 16500) plan.cluster *= 2;
    while (plan.cluster < kMaxCluster && a.rows * plan.cluster * 2 <= sms && vectors / plan.cluster > 256) plan.cluster *= 2;
    plan.slice_vectors = (int)((vectors + plan.cluster - 1) / plan.cluster);
    plan.flags = LOSS ? (plan.slice_vectors + 15) / 16 * 16 : 0;
    // Short rows by small blocks, of which more are under way (4096 x 4000 fp32, loss and gradient: 50 us with 128 threads, 75 with 256);
    // longer ones by larger blocks, with more loads in flight than rows (300 x 32001 fp32: 32 and 24 us); the longest, where the
    // gradient reads them again, by fewer and larger blocks, whose rows then fit L2 (4096 x 131072 bf16: 505 us with 256, 453 with 512)
    auto as = [&](auto type) {
        constexpr int DT = decltype(type)::value;
        if (vectors <= 2048 && a.rows > 2ll * sms) return launch_as<DT, LOSS, GRAD, 128>(a, plan, stream);
        if constexpr (LOSS && GRAD) { if (vectors > 8192) return launch_as<DT, LOSS, GRAD, 512>(a, plan, stream); }
        return launch_as<DT, LOSS, GRAD, 256>(a, plan, stream);
    };
    return dtype == kF32 ? as(std::integral_constant<int, kF32>()) : as(std::integral_constant<int, kBF16>());
}

}  // namespace

cudaError_t launch_distill(const DistillArgs& a, int dtype, bool loss, bool grad, int sms, cudaStream_t stream) {
    if (a.rows == 0) return cudaSuccess;
    if (loss && grad) return launch<true, true>(a, dtype, sms, stream);
    return loss ? launch<true, false>(a, dtype, sms, stream) : launch<false, true>(a, dtype, sms, stream);
}

}  // namespace tmask
