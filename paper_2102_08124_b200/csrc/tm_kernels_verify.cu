// Verification of drafted tokens against the target's probabilities.
//
//   p, q      softmax of a row of the target's logits and of the drafter's, z / T each
//   draft x   stays while u q(x) < p(x);  at the first that does not, the token is drawn from max(p - q, 0), behind the last from p
//   the draw  is a race of exponentials: the token with the largest r_k / E_k, E_k = -log(1 - u_k), wins with probability r_k / sum r, so no
//             sum over r and no search in running sums is needed, and the answer hangs on a comparison of two numbers, not on the rounding of a sum
//             of a hundred thousand terms
//
// A row's numbers e^(z/T) are 2^((z - m) c), c = log2(e) / T, m the running maximum (differences first: an offset that all logits share is no
// loss, and masks of the type's lowest value are zeros beside anything else).  Threads sum in fp32, their sums are joined in fp64.
//
// A cluster of blocks takes a sequence.  It goes through the positions in rounds: the rows of a round (the target's and the drafter's of some
// positions) are cut into segments that the cluster's warps share out evenly, whatever the number of rows, so that all of them are under way at
// once; then the warps' statistics are joined through shared memory, the blocks' through the cluster's, and every block takes the same decisions.
// Rounds of many positions read rows that turn out not to be reached, but wait once; they are for batches that leave the device half empty.
//
// Bound: by bytes HBM, 300 MB or 46 us for 256 sequences of up to 5 drafts and 131072 tokens in bf16; as measured 144 us.  Three pipes have 35 us of work
// each (an exponential a logit; the generator's wide products, 20 cycles a token and scheduler; conversions and maxima), its 55 M warp instructions
// 48 us, and phases that follow one another with barriers between them leave the issue slots half idle.  256 draws of 131072 tokens: 56 us, of which
// the generator needs 19; 4 drafts of one sequence, 32768 tokens in fp32: 12.5 us, by the eight blocks that a cluster has at most.  Without the
// drafter's logits: 256 sequences of 5 drafts 127 us of 39, 64 of 4 39 of 9.  Two blocks of 512 leave a thread 64 registers, and what the statistics and
// the race keep side by side spills 204 bytes (bf16) and 244 (fp32).  Decisions by the first block alone, told to the others, are 1.2 us and
// 2 % of these; without them (140 us) equal or slower: three blocks of 512 threads an SM at 40
// registers (138 - 145 us), four of 256 (130, but 21 us for one sequence of 131072 tokens against 18), one of 1024 (145), vectors asked for one
// by one as others are taken (135), a second exponential a token in the race (168), its fp64 keys for every candidate (206).
#include <algorithm>
#include <cfloat>

#include "tm_philox.cuh"
#include "tm_rows.cuh"

namespace tmask {
namespace {

constexpr uint32_t kTestBlocks = 0x80000000u;      // the generator's blocks of the acceptance tests; the draw's are tokens / 4, far below
constexpr int kThreads = 512, kBlocks = 2, kWarps = kThreads / 32, kMaxCluster = 8;
constexpr int kPositions = 8, kRows = 2 * kPositions;      // of a round: the target's rows, then the drafter's
constexpr int kLoads = 4;                          // 16-byte vectors that a lane asks for at once: a segment of a row is 32 kLoads of them
// What fp32 may be off by, relative.  A probability: 2^-22 of the exponential, and three roundings of an exponent of 126 at most (difference, c, product), 3 *
// 126 * 2^-24 ln 2 = 1.6e-5; kOff is above it.  1 / E: 2^-15 (race_gain).  A key has both, 5e-5, which is below half of kNear: keys further apart than kNear
// are in the right order, and nearer ones are told apart in fp64.
constexpr float kOff = 6e-5f, kNear = 4e-4f;
// log2 p - log2 q up to which p - q counts as nothing.  The rows' sums are fp32 sums: a thread adds up to vocab / 512 numbers (where one block
// has the sequence; an eighth of that where eight have; 128 where all positions are one round) one after the other, each addition off by 2^-24 at
// most, so 131072 tokens have 2^-16 if all were off the same way, and some 2^-21 as they fall.  Rows that are equal but for that then differ by one
// factor in all tokens: p - q is nothing, or p times a constant, and both mean a draw from p.
constexpr double kEqual = 0x1p-20;
constexpr float kSlack = 1e-3f;                    // of a logarithm in the race's screening, eight of its units

struct RowStat { float m; double s; };             // largest logit, sum of 2^((z - m) c); m is Inf where NaN or +Inf are among them, or nothing but -Inf

// N logits whose largest is top: into (m, s)
template <int N> __device__ __forceinline__ void take_logits(const float (&v)[N], float m, float c, float& s) {
    const float2 less = make_float2(-m, -m), by = make_float2(c, c);
    float2 add = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int j = 0; j + 1 < N; j += 2) {
        const float2 x = __fmul2_rn(__fadd2_rn(make_float2(v[j], v[j + 1]), less), by);
        add = __fadd2_rn(add, make_float2(exp2_fast(x.x), exp2_fast(x.y)));
    }
    if constexpr (N % 2) add.x += exp2_fast((v[N - 1] - m) * c);
    s += add.x + add.y;
}
__device__ __forceinline__ void raise(float top, float c, float& m, float& s, bool& bad) {
    bad |= !(top < INFINITY);
    if (top > m) { s *= exp2_fast((m - top) * c); m = top; }
}

// A warp's part of a row: vectors [from, to)
template <int DT> __device__ __forceinline__ void take_range(const RowVectors<DT>& row, int from, int to, float c, float& m, float& s, bool& bad) {
    constexpr int V = RowType<DT>::kVec;
    const RowPart<DT> part(row, from, to);
    const int lane = threadIdx.x & 31;
    const uint4* p = reinterpret_cast<const uint4*>(row.base + part.column) + lane;
    int i = lane;
    for (; i + 32 * (kLoads - 1) < part.inside; i += 32 * kLoads, p += 32 * kLoads) {
        uint4 u[kLoads];
        float top = -INFINITY;
#pragma unroll
        for (int k = 0; k < kLoads; ++k) u[k] = p[32 * k];
#pragma unroll
        for (int k = 0; k < kLoads; ++k) top = max_nan(top, vector_max_nan<DT>(u[k]));
        raise(top, c, m, s, bad);
#pragma unroll
        for (int k = 0; k < kLoads; ++k) {
            float v[V];
            unpack_vector<DT>(u[k], v);
            take_logits<V>(v, m, c, s);
        }
    }
    for (; i < part.inside; i += 32, p += 32) {
        const uint4 u = *p;
        float v[V];
        unpack_vector<DT>(u, v);
        raise(vector_max_nan<DT>(u), c, m, s, bad);
        take_logits<V>(v, m, c, s);
    }
    if (lane < part.head + part.tail) {
        const float v[1] = {to_float(row.base[part.edge(lane)])};
        raise(v[0], c, m, s, bad);
        take_logits<1>(v, m, c, s);
    }
}

// (m, s) of the lanes joined; m is Inf where a lane saw a bad logit
__device__ __forceinline__ float2 join_lanes(float m, float s, bool bad, float c) {
    const float all = group_max<32>(m);
    s = group_sum<32>(s * exp2_fast((m - all) * c));
    return make_float2(__any_sync(0xFFFFFFFFu, bad) ? INFINITY : all, s);
}

// Key of one token, r / E, in fp64.  x: log2 p, y: log2 q (-Inf: none), both relative to the largest p
__device__ __noinline__ double race_key(double x, double y, uint32_t word) {
    const double r = x - y > kEqual ? exp2(x) - exp2(y) : 0.0;
    return r > 0.0 ? r / -log1p(-((double)word + 0.5) * 0x1p-32) : 0.0;
}
// 1 / E in fp32, u = (word + 1/2) / 2^32.  Near 0 by E's series (its next term is 2^-26 of it).  Else by the logarithm of 1 - u, which __log2f has to 2^-22
// and 1 - u itself to 2^-24, absolute: at u = 1/64, where E is least, 2^-16.5 and 2^-18 of E.  So 2^-15 with the product and the quotient, and better from there on.
__device__ __forceinline__ float race_gain(uint32_t word) {
    const float u = fmaf((float)word, 0x1p-32f, 0x1p-33f);
    const float e = u < 0.015625f ? u * fmaf(u, fmaf(u, fmaf(u, 0.25f, 0.33333333f), 0.5f), 1.0f) : -0.69314718f * __log2f(fmaf((float)~word, 0x1p-32f, 0x1p-33f));
    return __fdividef(1.0f, e);
}
// 2^13 (127 + log2 of the word's upper 23 bits), from below (the bits of the float that they are)
__device__ __forceinline__ int passed(uint32_t word) { return (int)(__float_as_uint(__uint_as_float(0x4B000000u | word >> 9) - 0x1p23f) >> 10); }
// Whether a token's key may reach `best`.  No key is above p / u.  A float's bits, taken as a whole number, are a chord of 2^23 (127 + log2),
// below it; so log2 p - log2 best is compared with those of u's upper 23 bits, both in units of 2^-13: the float that holds the former ends in
// it as a whole number.
struct Screen {
    static constexpr float kUnit = 8192.0f, kWhole = 12582912.0f;
    static constexpr int kZero = 0x4B400000 - (127 + 23) * 8192;       // kWhole's bits, less u's 2^-23
    float add, by, m;
    __device__ __forceinline__ Screen(float best, float c, float m_) {
        add = kWhole + (kSlack - __log2f(best)) * kUnit;
        by = c * kUnit;
        m = m_;
    }
    __device__ __forceinline__ bool operator()(float z, uint32_t word) const { return (int)__float_as_uint(fmaf(z - m, by, add)) > passed(word) + kZero; }
};
// u q < p in fp64, x = log2 p, y = log2 q
__device__ __noinline__ bool stays(double u, double x, double y) { return u * exp2(y - x) < 1.0; }

__device__ __forceinline__ void faster(double& key, int& at, double other, int other_at) {
    if (other > key || (other == key && (unsigned)other_at < (unsigned)at)) { key = other; at = other_at; }
}

// The smallest of a generator's words
__device__ __forceinline__ uint32_t least(const uint4& w) { return min(min(w.x, w.y), min(w.z, w.w)); }

// The largest of eight logits from k0 on (a multiple of 8); vec: the row is on a 16-byte boundary
template <int DT> __device__ __forceinline__ float largest(const typename RowType<DT>::T* row, bool vec, int k0, int vocab) {
    if (vec && k0 + 8 <= vocab) {
        const uint4* u = reinterpret_cast<const uint4*>(row + k0);
        return RowType<DT>::kVec == 8 ? vector_max<DT>(u[0]) : fmaxf(vector_max<DT>(u[0]), vector_max<DT>(u[1]));
    }
    float top = -INFINITY;
#pragma unroll
    for (int j = 0; j < 8; ++j) if (k0 + j < vocab) top = fmaxf(top, to_float(row[k0 + j]));
    return top;
}

// Those logits, -Inf past the last
template <int DT> __device__ __forceinline__ void load_tokens(const typename RowType<DT>::T* row, bool vec, int k0, int vocab, float (&z)[8]) {
    constexpr int V = RowType<DT>::kVec;
    if (vec && k0 + 8 <= vocab) {
#pragma unroll
        for (int i = 0; i < 8; i += V) unpack_vector<DT>(*reinterpret_cast<const uint4*>(row + k0 + i), z + i);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) z[j] = k0 + j < vocab ? to_float(row[k0 + j]) : -INFINITY;
    }
}

struct Verify : VerifyArgs {
    double cp64, cq64;                             // log2(e) / T
    int cluster, round;                            // blocks of a sequence; positions of a round
};

// One row's race, as its rare steps need it
template <int DT> struct Race {
    const typename RowType<DT>::T *rp, *rq;        // rq null: no q
    double shift;                                  // q in units of 2^(m c) of p
    float pm, qm;                                  // largest logits
    int b, without;                                // without: a token that cannot win
};

template <int DT> __device__ __forceinline__ double exact_key(const Verify& a, const Race<DT>& race, int k) {
    const uint4 w = Philox(a.keys, a.offset, a.offset_dev)((uint32_t)k / 4, race.b);
    const int j = k & 3;
    return race_key(((double)to_float(race.rp[k]) - (double)race.pm) * a.cp64, race.rq ? ((double)to_float(race.rq[k]) - (double)race.qm) * a.cq64 + race.shift : -INFINITY,
                    j == 0 ? w.x : j == 1 ? w.y : j == 2 ? w.z : w.w);
}

// Eight tokens one by one, their keys good to less than half of kNear: raises this thread's best key and its token where one is above `best`
template <int DT> __device__ __noinline__ float2 look(const Verify& a, const Race<DT> race, int k0, uint4 w0, uint4 w1, float best, float mine, int at) {
    const uint32_t word[8] = {w0.x, w0.y, w0.z, w0.w, w1.x, w1.y, w1.z, w1.w};
    const float cp = (float)a.cp64;
    float z[8];
    load_tokens<DT>(race.rp, ((uintptr_t)race.rp & 15) == 0, k0, (int)a.vocab, z);
    const Screen screen(best, cp, race.pm);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        if (!screen(z[j], word[j])) continue;
        float r = exp2_fast((z[j] - race.pm) * cp);
        const float gain = race_gain(word[j]);
        if (!(r * gain * (1.0f + kOff) > best) || k0 + j == race.without) continue;
        if (race.rq) {                             // p - q = p (1 - 2^-d): d in fp64, so that nothing is lost where q is near p
            const double d = ((double)z[j] - (double)race.pm) * a.cp64 - (((double)to_float(race.rq[k0 + j]) - (double)race.qm) * a.cq64 + race.shift);
            r = d > kEqual ? r * -expm1f((float)d * -0.69314718f) : 0.0f;
        }
        const float k = r * gain;
        if (!(k > best)) continue;
        if (k > mine * (1.0f + kNear)) { mine = k; at = k0 + j; }
        else if (k >= mine * (1.0f - kNear) && exact_key<DT>(a, race, k0 + j) > exact_key<DT>(a, race, at)) { mine = fmaxf(k, mine); at = k0 + j; }
    }
    return make_float2(mine, __int_as_float(at));
}

// What a block knows of the race: its best key (fp32), that token, and how many of its threads have one within kNear of it
struct Front { float key; int at, near; };

template <int DT> __global__ void __launch_bounds__(kThreads, kBlocks) verify_kernel(const __grid_constant__ Verify a) {
    using T = typename RowType<DT>::T;
    __shared__ float2 warp_part[kRows][kWarps], block_part[2][kRows];
    __shared__ RowStat stat[kRows];
    __shared__ float front_key[kWarps];
    __shared__ Front front[2];
    __shared__ double exact_best[kWarps];
    __shared__ int exact_at[kWarps];
    __shared__ unsigned long long exact_block[2][2];
    __shared__ int decided[3];                     // of the first block, for all: drafts that stay, how the sequence ends (or that it goes on), drafts of the next round
    __shared__ float bound;
    const Philox key(a.keys, a.offset, a.offset_dev);
    const int cluster = a.cluster, b = blockIdx.x / cluster, rank = cluster > 1 ? (int)cluster_rank() : 0, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int vocab = (int)a.vocab;
    const float cp = (float)a.cp64, cq = (float)a.cq64, ln2 = 0.69314718f;
    const auto target = [&](int n) { return static_cast<const T*>(a.logits) + ((long long)b * (a.drafted + 1) + n) * a.ld; };
    const auto draft = [&](int n) { return static_cast<const T*>(a.draft_logits) + ((long long)b * a.drafted + n) * a.ld_draft; };
    const int* ids = a.ids + (long long)b * a.drafted;
    int* tokens = a.tokens + (long long)b * (a.drafted + 1);
    float* logp = a.logp ? a.logp + (long long)b * (a.drafted + 1) : nullptr;
    const auto sync_all = [&] { if (cluster > 1) cluster_sync(); else __syncthreads(); };

    constexpr int kGoOn = 0, kDrawTarget = 1, kDrawRest = 2, kBad = 3;
    // What decides how often the blocks wait for each other is read from memory by the first of them alone: others might see other numbers, should
    // somebody write to them meanwhile, and would wait for good.
    const auto drafts_from = [&](int k) {
        int more = 0;
        while (more < a.round && k + more < a.drafted && (unsigned)ids[k + more] < (unsigned)vocab) ++more;
        return more;
    };
    const auto told = [&](int k) { return cluster > 1 ? __float_as_int(cluster_load_float(reinterpret_cast<const float*>(decided + k), 0)) : decided[k]; };
    int n = 0, turn = 0, end = kGoOn;
    RowStat p, q;
    if (threadIdx.x == 0) {
        bound = 0.0f;
        if (rank == 0) decided[2] = drafts_from(0);
    }
    sync_all();
    for (;; turn ^= 1) {
        // the round's positions: up to the first that has no draft, with it
        const int drafts = told(2);
        const int positions = min(a.round, drafts + 1), rows = positions + (a.draft_logits ? drafts : 0);
        // what the tests need besides: thread k its position's
        int id = 0;
        float zp = 0.0f, zq = 0.0f;
        if (rank == 0 && (int)threadIdx.x < drafts) {
            id = min(max(ids[n + threadIdx.x], 0), vocab - 1);
            zp = to_float(target(n + threadIdx.x)[id]);
            if (a.draft_logits) zq = to_float(draft(n + threadIdx.x)[id]);
        }
        if (lane < kRows) warp_part[lane][warp] = make_float2(-FLT_MAX, 0.0f);
        __syncwarp();
        // segments of all rows, in a row for each warp; a row's vectors are one more where it starts off a boundary
        constexpr int kSegment = 32 * kLoads;
        const int segments = (vocab / RowType<DT>::kVec + 1 + kSegment) / kSegment;
        const unsigned all = rows * segments, warps = cluster * kWarps, me = rank * kWarps + warp;
        int at = all * me / warps;
        const int stop = all * (me + 1) / warps;
        while (at < stop) {
            const int row = at / segments, first = at - row * segments, last = min(segments, first + (stop - at));
            const bool theirs = row >= positions;                 // the drafter's
            const float c = theirs ? cq : cp;
            const RowVectors<DT> vectors(theirs ? draft(n + row - positions) : target(n + row), vocab);
            float m = -FLT_MAX, s = 0.0f;
            bool bad = false;
            const int from = first * kSegment, to = min((int)vectors.count, last * kSegment);
            if (from < to) take_range<DT>(vectors, from, to, c, m, s, bad);
            const float2 part = join_lanes(m, s, bad, c);
            if (lane == 0) warp_part[theirs ? kPositions + row - positions : row][warp] = part;
            at += last - first;
        }
        __syncthreads();
        static_assert(kRows * kWarps <= kThreads && kRows * kMaxCluster <= kThreads, "the joins below give a thread to each part");
        if (threadIdx.x < kRows * kWarps) {
            const int row = threadIdx.x / kWarps;
            const float2 v = warp_part[row][threadIdx.x % kWarps];
            const float c = row < kPositions ? cp : cq;
            float m = v.x;
#pragma unroll
            for (int o = kWarps / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
            const float s = group_sum<kWarps>(v.y * exp2_fast((v.x - m) * c));
            if (threadIdx.x % kWarps == 0) block_part[turn][row] = make_float2(m, s);
        }
        sync_all();
        if (threadIdx.x < kRows * kMaxCluster) {
            const int row = threadIdx.x / kMaxCluster, k = threadIdx.x % kMaxCluster;
            const float c = row < kPositions ? cp : cq;
            float2 v = make_float2(-FLT_MAX, 0.0f);
            if (k < cluster) v = cluster > 1 ? cluster_load2(&block_part[turn][row], k) : block_part[turn][row];
            float m = v.x;
#pragma unroll
            for (int o = kMaxCluster / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
            double s = (double)(v.y * exp2_fast((v.x - m) * c));
#pragma unroll
            for (int o = kMaxCluster / 2; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
            if (k == 0) stat[row] = RowStat{s > 0.0 ? m : INFINITY, s};
        }
        __syncthreads();
        if (rank == 0 && warp == 0) {
            // lane k: position n + k
            int what = kGoOn;
            float lp = 0.0f;
            if (lane < positions) {
                const RowStat sp = stat[lane], sq = stat[kPositions + lane];
                if (!(sp.m < INFINITY)) what = kBad;
                else if (lane >= drafts) what = kDrawTarget;
                else if (a.draft_logits && !(sq.m < INFINITY)) what = kBad;
                else {
                    const uint4 w = key(kTestBlocks + (n + lane) / 4, b);
                    const int j = (n + lane) & 3;
                    const uint32_t word = j == 0 ? w.x : j == 1 ? w.y : j == 2 ? w.z : w.w;
                    // u q(x) against p(x), both times the sum of p's numbers
                    const float mass = a.draft_logits ? (float)sp.s * exp2_fast((zq - sq.m) * cq) / (float)sq.s : (float)sp.s;
                    const float over = fmaf((float)word, 0x1p-32f, 0x1p-33f) * mass, own = exp2_fast((zp - sp.m) * cp);
                    bool stay = over < own;
                    if (!(fabsf(over - own) > kNear * own) || own < 1e-30f)
                        stay = stays(((double)word + 0.5) * 0x1p-32, ((double)zp - (double)sp.m) * a.cp64 - log2(sp.s),
                                     a.draft_logits ? ((double)zq - (double)sq.m) * a.cq64 - log2(sq.s) : 0.0);
                    if (!stay) what = kDrawRest;
                    lp = fmaf(zp - sp.m, cp * ln2, -logf((float)sp.s));
                }
            }
            const unsigned ends = __ballot_sync(0xFFFFFFFFu, what != kGoOn);
            const int stay = ends ? __ffs(ends) - 1 : positions;
            const int how = __shfl_sync(0xFFFFFFFFu, what, ends ? stay : 0);
            if (lane < stay) {
                tokens[n + lane] = id;
                if (logp) logp[n + lane] = lp;
            }
            if (lane == 0) {
                decided[0] = stay;
                decided[1] = how;
                decided[2] = how == kGoOn ? drafts_from(n + stay) : 0;
            }
        }
        sync_all();
        const int stay = told(0);
        end = told(1);
        n += stay;
        if (end != kGoOn) { p = stat[stay]; q = stat[kPositions + stay]; break; }
    }

    int token = -1;
    const T* rp = target(n);
    if (end != kBad) {
        const bool vec = ((uintptr_t)rp & 15) == 0;
        const double shift = end == kDrawRest && a.draft_logits ? log2(p.s) - log2(q.s) : 0.0;      // q in units of 2^(m c) of p
        // The best key is above sum r / t but for a chance of e^-t.  So what lies below a part of p's sum is left aside at first, and looked at in a
        // further attempt should nothing have been found; of p - q the sum is not known, and may be a small part of p's.  Where p - q leaves
        // nothing, p itself is drawn from.
        constexpr float kFloor[5] = {0x1p-6f, 0x1p-14f, 0.0f, 0x1p-3f, 0.0f};
        for (int attempt = end == kDrawRest ? 0 : 3; attempt < 5; ++attempt) {
            const int pass = attempt & 1;
            const bool minus = attempt < 3 && a.draft_logits;
            const Race<DT> race = {rp, minus ? draft(n) : nullptr, shift, p.m, q.m, b, attempt < 3 && !a.draft_logits ? ids[n] : -1};
            float mine = 0.0f;                     // this thread's best key
            int at = -1;
            const int step = cluster * kThreads * 8;
            float best = kFloor[attempt] * (float)p.s;      // what keys have to reach: this, or the block's best so far, less twice kNear
            for (int base = (rank * kWarps + warp) * 256; base < vocab; base += step) {
                const int k0 = base + lane * 8;
                const float top = largest<DT>(rp, vec, k0, vocab);
                const uint4 w0 = key((uint32_t)k0 / 4, b), w1 = key((uint32_t)k0 / 4 + 1, b);
                best = fmaxf(best, *(volatile float*)&bound);
                // no key of the eight is above the largest p over the smallest u
                if (!__any_sync(0xFFFFFFFFu, Screen(best, cp, p.m)(top, min(least(w0), least(w1))))) continue;
                const float2 found = look<DT>(a, race, k0, w0, w1, best, mine, at);
                mine = found.x;
                at = __float_as_int(found.y);
                const float now = group_max<32>(mine) * (1.0f - 2.0f * kNear);
                if (now > best) {
                    best = now;
                    if (lane == 0) atomicMax(reinterpret_cast<int*>(&bound), __float_as_int(best));      // from zero up floats order like whole numbers
                }
            }
            // the block's best, then the cluster's
            float top = group_max<32>(mine);
            if (lane == 0) front_key[warp] = top;
            __syncthreads();
            top = group_max<32>(front_key[lane % kWarps]);
            const int near = __syncthreads_count(top > 0.0f && mine >= top * (1.0f - kNear));
            if (mine == top && top > 0.0f) front[pass].at = at;
            if (threadIdx.x == 0) {
                front[pass].key = top;
                front[pass].near = near;
                bound = 0.0f;
            }
            sync_all();
            Front f = {0.0f, -1, 0};
            if (lane < cluster) {
                f = front[pass];
                if (cluster > 1) {
                    f.key = cluster_load_float(&front[pass].key, lane);
                    f.at = __float_as_int(cluster_load_float(reinterpret_cast<const float*>(&front[pass].at), lane));
                    f.near = __float_as_int(cluster_load_float(reinterpret_cast<const float*>(&front[pass].near), lane));
                }
            }
            const float first = group_max<32>(f.key);
            if (first == 0.0f) continue;           // nothing to draw from
            const unsigned ahead = __ballot_sync(0xFFFFFFFFu, f.key >= first * (1.0f - kNear));
            token = __shfl_sync(0xFFFFFFFFu, f.at, __ffs(ahead) - 1);
            if (__popc(ahead) == 1 && __shfl_sync(0xFFFFFFFFu, f.near, __ffs(ahead) - 1) == 1) break;
            // too near for fp32: every thread whose best may be the winner gives its key in fp64
            double k = mine >= first * (1.0f - 2.0f * kNear) ? exact_key<DT>(a, race, at) : 0.0;
            if (k == 0.0) at = -1;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                const double other = __shfl_xor_sync(0xFFFFFFFFu, k, o);
                faster(k, at, other, __shfl_xor_sync(0xFFFFFFFFu, at, o));
            }
            if (lane == 0) { exact_best[warp] = k; exact_at[warp] = at; }
            __syncthreads();
            if (threadIdx.x == 0) {
                for (int w = 1; w < kWarps; ++w) faster(k, at, exact_best[w], exact_at[w]);
                exact_block[pass][0] = (unsigned long long)__double_as_longlong(k);
                exact_block[pass][1] = (unsigned long long)(long long)at;
            }
            sync_all();
            k = 0.0;
            token = -1;
            for (int r = 0; r < cluster; ++r) {
                const unsigned long long other = cluster > 1 ? cluster_load64(&exact_block[pass][0], r) : exact_block[pass][0];
                const unsigned long long where = cluster > 1 ? cluster_load64(&exact_block[pass][1], r) : exact_block[pass][1];
                faster(k, token, __longlong_as_double((long long)other), (int)(long long)where);
            }
            if (token >= 0) break;
        }
    }
    if (rank == 0) {
        if (threadIdx.x == 0) {
            a.accepted[b] = n;
            tokens[n] = token;
            if (logp) logp[n] = token < 0 ? __int_as_float(0x7FC00000) : fmaf(to_float(rp[token]) - p.m, cp * ln2, -logf((float)p.s));
            const int flags = (end == kBad ? kDevNonFinite : 0) | (n < a.drafted && end != kDrawRest && ids[n] >= vocab ? kDevBadId : 0);
            if (flags && a.status) atomicOr(a.status, flags);
        }
        for (int k = n + 1 + threadIdx.x; k <= a.drafted; k += kThreads) {
            tokens[k] = -1;
            if (logp) logp[k] = 0.0f;
        }
    }
    if (cluster > 1) cluster_sync();               // no block ends while another reads its shared memory
}

}  // namespace

cudaError_t launch_verify(const VerifyArgs& args, int dtype, int sms, cudaStream_t stream) {
    if (args.batch == 0) return cudaSuccess;
    Verify a;
    static_cast<VerifyArgs&>(a) = args;
    a.cp64 = 1.4426950408889634 / (double)a.temperature;
    a.cq64 = 1.4426950408889634 / (double)a.draft_temperature;
    // Blocks of a sequence: as many as the device holds (two an SM), up to a portable cluster's eight, each with more than 2048 tokens; twice that where rows
    // are long and sequences end at different positions.  us by 1, 2, 4, 8 blocks (before decisions were the first block's, 1 us a round less): 256 sequences of 5 drafts and fewer, 131072 tokens bf16 157, 140, 142, 187; 256 of 3, 32001
    // 49, 59, 83, 136; 256 of none, 131072 56, 62, 75, 113; 64 of 4, 131072 97, 61, 52, 66; 1 of 4, 32768 fp32 25, 19, 14, 11.
    int cluster = 1;
    const long long room = 2ll * sms;
    while (cluster < kMaxCluster && a.vocab > 4096ll * cluster &&
           2ll * a.batch * cluster <= (a.drafted > 0 && a.vocab > 65536ll * cluster ? 2 * room : room)) cluster *= 2;
    // Positions of a round: two, or all where their rows are short and the device has room.  Two and eight: 8 sequences of 4 drafts, 32001 bf16, by
    // eight blocks 17.8 and 12.7, 256 of 8, 4096 23.9 and 17.3; 256 of 5 and fewer, 131072, by two blocks 140 and 144 (one: 148).
    a.round = a.batch * (long long)cluster <= room && a.vocab <= 16384ll * cluster ? kPositions : 2;
    a.cluster = cluster;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(a.batch * cluster));
    cfg.blockDim = dim3(kThreads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)cluster; attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 1 : 0;
    return dtype == kF32 ? cudaLaunchKernelEx(&cfg, verify_kernel<kF32>, a) : cudaLaunchKernelEx(&cfg, verify_kernel<kBF16>, a);
}

}  // namespace tmask
