// Layer normalisation with an optional residual sum, forward and backward.
//
//   forward    h = x (+ residual);  mu = mean_c h;  r = (mean_c (h - mu)^2 + eps)^(-1/2);  y = (h - mu) r w + b
//   backward   g = dy w;  xh = (h - mu) r;  dx = r (g - mean_c g - xh mean_c (g xh)) (+ dsum);
//              dw = sum_rows dy xh;  db = sum_rows dy
//
// Bound: HBM by bytes (8 respectively 14 operations an element against 4 to 16 bytes); as measured the latency of a row's loads and
// reductions, after the number of instructions was cut (backward, 16384 x 1024 bf16: from 25.0 to 13.3 million warp instructions; 16.4 with
// the next row asked for ahead, which is faster): two elements an instruction wherever there is a packed form, parameters in registers
// over all rows, nothing worked out twice.
// A row belongs to a group of threads -- 8 or 32 of a warp, or up to 1024, by its width -- and stays in their registers between the
// reductions and the output: it is read once.  Groups go through the rows with a stride and ask for the next row before they
// reduce this one; several groups an SM cover each other's latency.
// Measured in a replayed graph, copy bandwidth 6.55 TB/s, fp32 weights: forward with residual and sum 16384 x 1024 bf16 23.1 us (5.8 TB/s),
// without them 8000 x 4096 bf16 26.1 us (5.0), 4097 x 1001 fp32 7.6 us (4.3), 2047 x 8191 bf16 22.5 us (3.0; with bf16 weights 25.8),
// 2000 x 20000 bf16 135 us; backward 16384 x 1024 bf16 with dsum 32.9 us (4.1), fp32 36.2 us (5.6), 2047 x 8191 bf16 54.0 us (1.9; with bf16
// weights 57.0), 2000 x 20000 bf16 242 us.  The figures at the forms below are of weights of the matrix's type.
// The centred squares are summed after the mean is known (no difference of large numbers); the normalised value uses the sum
// before it is rounded for sum_out: one rounding, at the end.
// A thread owns the same columns of every row, so the backward pass keeps its share of dw and db in registers over all rows
// that its block takes; blocks leave one partial row each, which a second kernel adds up in a fixed order (same input, same bits).
// The backward pass of rows too wide for that reads them from a ring of stages in shared memory that bulk copies fill (ring kernel);
// rows wider still are read again from L2 for every step (wide_* kernels).
#include <algorithm>

#include "tm_launch.h"
#include "tm_row_regs.cuh"
#include "tm_tma.cuh"

namespace tmask {

// Partial rows of the parameters' gradients, one a block of the backward kernel: as many as the device holds, up to the memory that
// they are worth.
int norm_partial_rows(long long rows, long long cols) {
    const long long cap = cols <= 4096 ? 888 : (cols <= 65536 ? 296 : 64);
    return (int)std::max<long long>(1, std::min(rows, cap));
}

namespace {

constexpr int kMaxStages = 4, kMaxStreams = 3;

// The rows of one input matrix as they are copied: [begin, end) is the memory that the matrix covers, first to last element.
struct Stream {
    const char *begin, *end;
    long long pitch;               // bytes
};
// A row in a stage: the bytes [lo, hi) that are copied, rounded outwards to 16-byte boundaries where that stays inside the matrix, else
// inwards (only its first and last row can be so).
struct RowBytes {
    const char *start, *lo;
    uint32_t bytes;
    __device__ __forceinline__ RowBytes(const Stream& m, long long r, uint32_t row_bytes) {
        start = m.begin + r * m.pitch;
        const char* down = reinterpret_cast<const char*>(reinterpret_cast<uintptr_t>(start) & ~(uintptr_t)15);
        const char* up = reinterpret_cast<const char*>((reinterpret_cast<uintptr_t>(start) + row_bytes + 15) & ~(uintptr_t)15);
        lo = down < m.begin ? down + 16 : down;
        if (up > m.end) up -= 16;
        bytes = up > lo ? (uint32_t)(up - lo) : 0u;
    }
};
struct RingPlan {
    int stages, streams;
    uint32_t row_bytes, stage_bytes;           // of one stream: a row, a stage
    Stream in[kMaxStreams];
};

// A block's ring: its rows go through the stages in turn.
struct RowRing {
    const RingPlan& plan;
    char* stage0;
    uint64_t* bars;
    __device__ __forceinline__ char* stage(int slot, int stream) const { return stage0 + (size_t)(slot * plan.streams + stream) * plan.stage_bytes; }
    // one thread: asks for a row
    __device__ __forceinline__ void ask(int slot, long long r) const {
        uint32_t all = 0;
        for (int k = 0; k < plan.streams; ++k) all += RowBytes(plan.in[k], r, plan.row_bytes).bytes;
        fence_proxy_async_smem();
        mbar_expect_tx(bars + slot, all);
        for (int k = 0; k < plan.streams; ++k) {
            const RowBytes b(plan.in[k], r, plan.row_bytes);
            if (b.bytes) asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                                      ::"r"(smem_addr(stage(slot, k))), "l"(b.lo), "r"(b.bytes), "r"(smem_addr(bars + slot)) : "memory");
        }
    }
};
// A stream's row in its stage: elements by column.  Those that the copy left out (at most 7 at either end of the matrix) come from the row.
template <int DT, int VB> struct RowInStage {
    const char *start, *copy;      // the row, and where it would start in the stage
    int from, to;                  // columns that are in the stage
    __device__ __forceinline__ RowInStage(const Stream& m, long long r, uint32_t row_bytes, const char* stage) {
        const RowBytes b(m, r, row_bytes);
        constexpr int B = RowType<DT>::kBytes;
        start = b.start;
        copy = stage + (b.start - b.lo);
        from = b.lo > b.start ? (int)((b.lo - b.start) / B) : 0;
        to = min((int)(row_bytes / B), (int)((b.lo + b.bytes - b.start) / B));
    }
    __device__ __forceinline__ void load(int c, float* v) const {
        const char* p = copy + (long long)c * RowType<DT>::kBytes;
        if constexpr (VB != 16) { if (c < from || c >= to) p = start + (long long)c * RowType<DT>::kBytes; }
        Access<DT, VB>::load(p, v);
    }
};

constexpr long long kRingWidth = 16384;

// Sets a block's ring up and asks for its first rows
__device__ __forceinline__ RowRing start_ring(const RingPlan& plan, char* smem, uint64_t* bars, long long first, long long step, long long rows) {
    const RowRing ring{plan, smem, bars};
    if (threadIdx.x == 0) {
        for (int i = 0; i < plan.stages; ++i) mbar_init(bars + i, 1);
        fence_mbar_init();
    }
    __syncthreads();
    if (threadIdx.x == 0)
        for (int k = 0; k < plan.stages; ++k) { const long long r = first + k * step; if (r < rows) ring.ask(k, r); }
    return ring;
}

// Threads of a block whose rows are shared by TPR threads each, and blocks an SM (the registers they may use).  Backward: a block
// leaves one partial row of parameter gradients, so the groups of rows up to 2048 columns share larger blocks.
template <int TPR> constexpr int kForwardThreads = TPR <= 32 ? 128 : TPR;
template <int TPR, int E> constexpr int kBackwardThreads = TPR <= 32 ? 128 : TPR <= 128 ? 384 : TPR <= 256 ? (E <= 8 ? 768 : 256) : TPR;
template <int TPR, int E> constexpr int kForwardBlocks = std::max(1, (E <= 8 ? 1024 : 768) / kForwardThreads<TPR>);
template <int TPR, int E> constexpr int kBackwardBlocks = std::max(1, (E <= 8 ? 768 : 512) / kBackwardThreads<TPR, E>);

template <int DT, int VB, int TPR, int E>
__global__ void __launch_bounds__(kForwardThreads<TPR>, kForwardBlocks<TPR, E>) norm_forward_kernel(const NormArgs a) {
    using R = RowRegs<DT, VB, TPR, E>;
    constexpr int P = E / 2, kGroups = kForwardThreads<TPR> / TPR;
    // kAhead: the next row is asked for before this one is reduced, where the registers suffice; kFetch: else it is brought to L2.  Neither
    // and as here, us: 16384 x 1024 bf16 31.3 and 23.1, 8000 x 4096 bf16 34.9 and 27.1, 2047 x 8191 bf16 41.5 and 26.1, 2048 x 8192 fp32
    // 37.7 and 29.6, 3000 x 9000 fp32 64.4 and 49.2; 200 x 12000 bf16 8.6 and 9.2.  kKeep: weight and bias stay in registers over all rows.
    constexpr bool kAhead = VB == 16 ? DT == kBF16 || R::NV <= 2 : E == 16 && (TPR == 256 || TPR == 512), kKeep = E < 32, kFetch = !kAhead && TPR >= 128;
    __shared__ float buf[2][32];
    const int t = threadIdx.x % TPR, g = threadIdx.x / TPR, cols = (int)a.cols;
    const float inv_n = 1.0f / (float)a.cols;
    const long long step = (long long)gridDim.x * kGroups;
    float2 w[P], b[P];
    if constexpr (kKeep) {
        R::params(a.weight, a.weight_f32, a.weight_vec, cols, w, 1.0f);
        R::params(a.bias, a.weight_f32, a.bias_vec, cols, b, 0.0f);
    }
    typename R::Raw ux[R::NV], us[R::NV];
    const auto ask = [&](long long r) {
        if constexpr (kAhead) {
            const int n = r < a.rows ? cols : 0;
            R::ask(row_of<DT>(a.x, a.ld_x, r), n, ux);
            if (a.residual) R::ask(row_of<DT>(a.residual, a.ld_residual, r), n, us);
        }
    };
    ask((long long)blockIdx.x * kGroups + g);
    for (long long r0 = (long long)blockIdx.x * kGroups; r0 < a.rows; r0 += step) {
        const long long r = r0 + g;
        const bool on = r < a.rows;                       // whole groups idle together, but take part in the shuffles and barriers
        float2 h[P];
        if constexpr (kAhead) R::take(ux, h);
        else R::load(row_of<DT>(a.x, a.ld_x, r), on ? cols : 0, h);
        if (a.residual) {
            float2 s[P];
            if constexpr (kAhead) R::take(us, s);
            else R::load(row_of<DT>(a.residual, a.ld_residual, r), on ? cols : 0, s);
#pragma unroll
            for (int k = 0; k < P; ++k) h[k] = __fadd2_rn(h[k], s[k]);
        }
        ask(r + step);
        if constexpr (kFetch) R::fetch(a.x, a.ld_x, a.residual ? a.residual : a.x, a.residual ? a.ld_residual : a.ld_x, r + step, a.rows, cols);
        if (a.sum && on) R::store(row_of<DT>(a.sum, a.ld_sum, r), cols, h);
        float2 add = h[0];
#pragma unroll
        for (int k = 1; k < P; ++k) add = __fadd2_rn(add, h[k]);
        const float mean = row_sum<TPR, kGroups>(add.x + add.y, buf[0]) * inv_n;
        float2 sq = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int k = 0; k < P; ++k) {
            h[k] = __fadd2_rn(h[k], R::inside(k, cols, -mean));      // the zeros past the last column stay zeros
            sq = __ffma2_rn(h[k], h[k], sq);
        }
        const float rstd = rsqrtf(row_sum<TPR, kGroups>(sq.x + sq.y, buf[1]) * inv_n + a.eps);
        if (!on) continue;
        if (t == 0) {
            if (a.mean) a.mean[r] = mean;
            if (a.rstd) a.rstd[r] = rstd;
        }
        if constexpr (!kKeep) {
            R::params(a.weight, a.weight_f32, a.weight_vec, cols, w, 1.0f);
            R::params(a.bias, a.weight_f32, a.bias_vec, cols, b, 0.0f);
        }
        const float2 rr = make_float2(rstd, rstd);
#pragma unroll
        for (int k = 0; k < P; ++k) h[k] = __ffma2_rn(__fmul2_rn(h[k], rr), w[k], b[k]);
        R::store(row_of<DT>(a.y, a.ld_y, r), cols, h);
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
__global__ void __launch_bounds__(kBackwardThreads<TPR, E>, kBackwardBlocks<TPR, E>) norm_backward_kernel(const NormBackArgs a) {
    using R = RowRegs<DT, VB, TPR, E>;
    constexpr int P = E / 2, kThreads = kBackwardThreads<TPR, E>, kGroups = kThreads / TPR;
    // As in the forward kernel.  Without and with asking ahead, us: 16384 x 1024 bf16 38.3 and 32.7; fp32 spills: 30000 x 100 20.1
    // and 26.2.  kFetch without and with: 2048 x 8192 fp32 58.0 and 43.5, 2047 x 8191 bf16 63.6 and 57.0; but 4097 x 1001 fp32, in accesses
    // of one and 128 threads a row, 15.8 and 18.3.
    constexpr bool kAhead = VB == 16 && DT == kBF16, kKeep = TPR < 1024, kFetch = !kAhead && (TPR == 1024 || (VB == 16 && TPR >= 128));
    __shared__ float2 buf[2][32];
    extern __shared__ float fold[];                       // kGroups > 1: [2][cols]
    const int g = threadIdx.x / TPR, cols = (int)a.cols;
    const float inv_n = 1.0f / (float)a.cols;
    const long long step = (long long)gridDim.x * kGroups;
    float2 w[P], dw[P], db[P];
    if constexpr (kKeep) R::params(a.weight, a.weight_f32, a.weight_vec, cols, w, 1.0f);
#pragma unroll
    for (int k = 0; k < P; ++k) dw[k] = db[k] = make_float2(0.0f, 0.0f);
    int turn = 0;
    typename R::Raw ud[R::NV], ux[R::NV], ue[R::NV];
    float next_mean = 0.0f, next_rstd = 0.0f;
    const auto ask = [&](long long r) {
        if constexpr (kAhead) {
            const bool on = r < a.rows;
            R::ask(row_of<DT>(a.dy, a.ld_dy, r), on ? cols : 0, ud);
            R::ask(row_of<DT>(a.h, a.ld_h, r), on ? cols : 0, ux);
            R::ask(row_of<DT>(a.dsum, a.ld_dsum, r), on && a.dsum ? cols : 0, ue);
            next_mean = on ? a.mean[r] : 0.0f;
            next_rstd = on ? a.rstd[r] : 0.0f;
        }
    };
    ask((long long)blockIdx.x * kGroups + g);
    for (long long r0 = (long long)blockIdx.x * kGroups; r0 < a.rows; r0 += step, turn ^= 1) {
        const long long r = r0 + g;
        const bool on = r < a.rows;
        float2 d[P], x[P], e[P];
        float mean, rstd;
        if constexpr (kAhead) {
            R::take(ud, d);
            R::take(ux, x);
            R::take(ue, e);                               // zeros without a dsum
            mean = next_mean;
            rstd = next_rstd;
        } else {
            R::load(row_of<DT>(a.dy, a.ld_dy, r), on ? cols : 0, d);
            R::load(row_of<DT>(a.h, a.ld_h, r), on ? cols : 0, x);
            mean = on ? a.mean[r] : 0.0f;
            rstd = on ? a.rstd[r] : 0.0f;
            R::load(row_of<DT>(a.dsum, a.ld_dsum, r), on && a.dsum ? cols : 0, e);
        }
        if constexpr (kFetch) {
            R::fetch(a.dy, a.ld_dy, a.h, a.ld_h, r + step, a.rows, cols);
            if constexpr (VB == 16) if (a.dsum) R::fetch(a.dsum, a.ld_dsum, a.dsum, a.ld_dsum, r + step, a.rows, cols);
        }
        ask(r + step);
        const float2 minus = make_float2(-mean, -mean), rs = make_float2(rstd, rstd);
        if constexpr (!kKeep) R::params(a.weight, a.weight_f32, a.weight_vec, cols, w, 1.0f);
        float2 s1 = make_float2(0.0f, 0.0f), s2 = s1;
#pragma unroll
        for (int k = 0; k < P; ++k) {
            x[k] = __fmul2_rn(__fadd2_rn(x[k], minus), R::inside(k, cols, rstd));      // zero past the last column
            dw[k] = __ffma2_rn(d[k], x[k], dw[k]);
            db[k] = __fadd2_rn(db[k], d[k]);
            d[k] = __fmul2_rn(d[k], w[k]);
            s1 = __fadd2_rn(s1, d[k]);
            s2 = __ffma2_rn(d[k], x[k], s2);
        }
        const float2 both = row_sum2<TPR, kGroups>(make_float2(s1.x + s1.y, s2.x + s2.y), buf[turn]);
        if (!on) continue;
        const float m1 = -both.x * inv_n, m2 = -both.y * inv_n;
        const float2 mm1 = make_float2(m1, m1), mm2 = make_float2(m2, m2);
#pragma unroll
        for (int k = 0; k < P; ++k) {
            const float2 v = __fadd2_rn(__ffma2_rn(x[k], mm2, d[k]), mm1);
            d[k] = __ffma2_rn(v, rs, e[k]);
        }
        R::store(row_of<DT>(a.dx, a.ld_dx, r), cols, d);
    }
    if (!a.partials) return;
    float* out = a.partials + (long long)blockIdx.x * 2 * a.cols;
    const float *fw = reinterpret_cast<const float*>(dw), *fb = reinterpret_cast<const float*>(db);
    // the groups add their columns one after the other
#pragma unroll 1
    for (int k = 0; k < kGroups; ++k) {
        if (kGroups > 1) __syncthreads();
        if (g != k) continue;
        float* to = k + 1 == kGroups ? out : fold;
#pragma unroll
        for (int q = 0; q < E; ++q) {
            const int c = R::column(q / R::VE) + q % R::VE;
            if (c < cols) {
                to[c] = fw[q] + (k ? fold[c] : 0.0f);
                to[cols + c] = fb[q] + (k ? fold[cols + c] : 0.0f);
            }
        }
    }
}

// Rows of 8193 to kRingWidth columns: two rows' inputs do not fit the registers beside the parameters' gradients, so bulk copies bring the
// next rows to shared memory.  2000 x 16384 bf16 86 us, 3000 x 9000 fp32 86 us; with every step read from L2 again 198 and 186 us.  For
// narrower rows the registers are faster: 16384 x 1024 bf16 77 us by this kernel, 32.7 us by the one above.
// streams: dy, h and, with a third one, dsum
constexpr int kRingThreads = 512;
template <int DT, int VB, int E>
__global__ void __launch_bounds__(kRingThreads, 1) ring_norm_backward_kernel(const __grid_constant__ NormBackArgs a, const __grid_constant__ RingPlan plan) {
    using A = Access<DT, VB>;
    constexpr int VE = A::kElems, NV = E / VE, TPR = kRingThreads;
    extern __shared__ __align__(128) char smem[];
    __shared__ __align__(8) uint64_t bars[kMaxStages];
    __shared__ float2 buf[2][32];
    const int t = threadIdx.x, cols = (int)a.cols;
    const float inv_n = 1.0f / (float)a.cols;
    const long long first = blockIdx.x, step = gridDim.x;
    const RowRing ring = start_ring(plan, smem, bars, first, step, a.rows);
    float dw[E], db[E];
#pragma unroll
    for (int k = 0; k < E; ++k) dw[k] = db[k] = 0.0f;
    int slot = 0, turn = 0;
    uint32_t phase = 0;
    float next_mean = 0.0f, next_rstd = 0.0f;
    if (first < a.rows) { next_mean = a.mean[first]; next_rstd = a.rstd[first]; }
    for (long long r = first; r < a.rows; r += step, turn ^= 1) {
        const float mean = next_mean, rstd = next_rstd;
        if (r + step < a.rows) { next_mean = a.mean[r + step]; next_rstd = a.rstd[r + step]; }
        const bool late = !mbar_wait_bounded(ring.bars + slot, phase);
        const RowInStage<DT, VB> dy(plan.in[0], r, plan.row_bytes, ring.stage(slot, 0)), h(plan.in[1], r, plan.row_bytes, ring.stage(slot, 1));
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * TPR + t) * VE;
            if (c < cols) {
                float w[VE], d[VE], x[VE];
                load_params<VE>(a.weight, a.weight_f32, a.weight_vec, c, w, 1.0f);
                dy.load(c, d);
                h.load(c, x);
#pragma unroll
                for (int j = 0; j < VE; ++j) {
                    const float xh = (x[j] - mean) * rstd, u = d[j] * w[j];
                    s1 += u;
                    s2 = fmaf(u, xh, s2);
                    dw[i * VE + j] = fmaf(d[j], xh, dw[i * VE + j]);
                    db[i * VE + j] += d[j];
                }
            }
        }
        const float2 both = row_sum2<TPR>(make_float2(s1, s2), buf[turn]);
        s1 = both.x * inv_n;
        s2 = both.y * inv_n;
        auto* dxr = row_of<DT>(a.dx, a.ld_dx, r);
        const RowInStage<DT, VB> e(plan.in[plan.streams - 1], r, plan.row_bytes, ring.stage(slot, plan.streams - 1));
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * TPR + t) * VE;
            if (c < cols) {
                float w[VE], d[VE], x[VE], o[VE];
                load_params<VE>(a.weight, a.weight_f32, a.weight_vec, c, w, 1.0f);
                dy.load(c, d);
                h.load(c, x);
#pragma unroll
                for (int j = 0; j < VE; ++j) o[j] = rstd * (d[j] * w[j] - s1 - (x[j] - mean) * rstd * s2);
                if (plan.streams > 2) {
                    float v[VE];
                    e.load(c, v);
#pragma unroll
                    for (int j = 0; j < VE; ++j) o[j] += v[j];
                }
                A::store(dxr + c, o);
            }
        }
        if (__syncthreads_or(late)) {
            // A copy that did not come in time: this block asks for no more and shows it, in this row, its later ones and its share of the
            // parameters' gradients.  What is still under way gets some more time before the stages go.
            const float nan = __uint_as_float(0x7FC00000u);
            if (t == 0)
                for (int i = 0; i < plan.stages; ++i) { mbar_wait_bounded(bars + i, 0, 1u << 14); mbar_wait_bounded(bars + i, 1, 1u << 14); }
            for (; r < a.rows; r += step)
                for (int c = t; c < cols; c += TPR) from_float(row_of<DT>(a.dx, a.ld_dx, r) + c, nan);
#pragma unroll
            for (int k = 0; k < E; ++k) dw[k] = db[k] = nan;
            break;
        }
        if (t == 0 && r + plan.stages * step < a.rows) ring.ask(slot, r + plan.stages * step);
        if (++slot == plan.stages) { slot = 0; phase ^= 1u; }
    }
    if (!a.partials) return;
    float* out = a.partials + (long long)blockIdx.x * 2 * a.cols;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < VE; ++j) {
            const int c = (i * TPR + t) * VE + j;
            if (c < cols) {
                out[c] = dw[i * VE + j];
                out[cols + c] = db[i * VE + j];
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
#pragma unroll 8
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

constexpr size_t kRingSmem = 208 * 1024;       // of a block's 227 KB

// As many stages as fit, for rows of `row_bytes` in `streams` matrices (at least one: 3 x 64 KB)
RingPlan ring_plan(const Stream* in, int streams, uint32_t row_bytes) {
    RingPlan p = {};
    for (int k = 0; k < streams; ++k) p.in[k] = in[k];
    p.streams = streams;
    p.row_bytes = row_bytes;
    p.stage_bytes = (row_bytes + 15 + 16) / 16 * 16;
    p.stages = (int)std::min<size_t>(kMaxStages, kRingSmem / ((size_t)p.stage_bytes * streams));
    return p;
}
Stream stream_of(const void* base, long long ld, long long rows, long long cols, int elem) {
    const char* b = static_cast<const char*>(base);
    return {b, b + ((rows - 1) * ld + cols) * elem, ld * elem};
}

template <int DT, int VB, int TPR, int E> cudaError_t forward(const NormArgs& a, int sms, cudaStream_t stream) {
    constexpr int kThreads = kForwardThreads<TPR>, kGroups = kThreads / TPR;
    const long long want = (a.rows + kGroups - 1) / kGroups, cap = (long long)kForwardBlocks<TPR, E> * sms;
    norm_forward_kernel<DT, VB, TPR, E><<<(unsigned)std::min(want, cap), kThreads, 0, stream>>>(a);
    return cudaGetLastError();
}

template <int DT, int VB, int TPR, int E> cudaError_t backward(const NormBackArgs& a, int sms, int* used, cudaStream_t stream) {
    constexpr int kThreads = kBackwardThreads<TPR, E>, kGroups = kThreads / TPR;
    const long long want = (a.rows + kGroups - 1) / kGroups, cap = std::min<long long>((long long)kBackwardBlocks<TPR, E> * sms, norm_partial_rows(a.rows, a.cols));
    *used = (int)std::min(want, cap);
    const size_t smem = kGroups > 1 && a.partials ? 2 * sizeof(float) * (size_t)a.cols : 0;      // at most 16 KB: these rows have 2048 columns or fewer
    norm_backward_kernel<DT, VB, TPR, E><<<(unsigned)*used, kThreads, smem, stream>>>(a);
    return cudaGetLastError();
}

template <int DT, int VB, int E> cudaError_t ring_backward(const NormBackArgs& a, int sms, int* used, cudaStream_t stream) {
    constexpr int kBytes = RowType<DT>::kBytes;
    auto kernel = ring_norm_backward_kernel<DT, VB, E>;
    static PerDeviceOnce once;
    const cudaError_t e = once.run([&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kRingSmem); });
    if (e != cudaSuccess) return e;
    const Stream in[3] = {stream_of(a.dy, a.ld_dy, a.rows, a.cols, kBytes), stream_of(a.h, a.ld_h, a.rows, a.cols, kBytes),
                          stream_of(a.dsum, a.ld_dsum, a.rows, a.cols, kBytes)};
    const RingPlan p = ring_plan(in, a.dsum ? 3 : 2, (uint32_t)(a.cols * kBytes));
    *used = std::min(sms, norm_partial_rows(a.rows, a.cols));
    kernel<<<(unsigned)*used, kRingThreads, (size_t)p.stages * p.streams * p.stage_bytes, stream>>>(a, p);
    return cudaGetLastError();
}

// The form for a row of `cols` elements: threads that share it, elements of each; the fewest threads that keep it in registers, unless
// measured otherwise (us, the form taken and the other): forward 16384 x 1024 bf16 (128, 8) 23.1, (64, 16) 24.3; 4097 x 1001 fp32 (64, 16)
// 7.8, (128, 8) 9.1; 16384 x 2048 bf16 (128, 16) 27.8, (256, 8) 29.6; 2048 x 8192 fp32 (1024, 8) 25.6, (512, 16) 29.6; 2047 x 8191 bf16
// (512, 16) 26.1, (1024, 8) 39.0; wider bf16 (512, 32) and (1024, 16) by rows times columns: 200 x 12000 7.8 and 9.9, 444 x 16384 14.2 and
// 15.0, 600 x 12000 17.5 and 17.9, 600 x 16384 22.1 and 19.5, 2000 x 8200 42.4 and 40.3, 2000 x 16384 58.5 and 44.8; 3000 x 9000 fp32
// (1024, 16) 49.2, (512, 32) 66.0; backward 32768 x 512 bf16
// (64, 8) 30.1, (128, 8) 46.4; 8000 x 4096 bf16 (256, 16) 53.2, (512, 8) 68.4; 2047 x 8191 bf16 in accesses of one (1024, 8) 63.0,
// (512, 16) 70.1 (both without kFetch).  Accesses of 16 bytes around such a row's elements, shifted into place, were no faster there
// (61.2) and slower forward (38.0 against 25.7).
template <int DT, int VB> cudaError_t forward_by_width(const NormArgs& a, int sms, cudaStream_t stream) {
    if (a.cols <= 64) return forward<DT, VB, 8, 8>(a, sms, stream);
    if (a.cols <= 256) return forward<DT, VB, 32, 8>(a, sms, stream);
    if (a.cols <= 512) return forward<DT, VB, 32, 16>(a, sms, stream);
    if (a.cols <= 1024) return forward<DT, VB, VB == 16 ? 128 : 64, VB == 16 ? 8 : 16>(a, sms, stream);
    if (a.cols <= 2048) return forward<DT, VB, 128, 16>(a, sms, stream);
    if (a.cols <= 4096) return forward<DT, VB, 256, 16>(a, sms, stream);
    constexpr bool kWords = VB == 16 && DT == kF32;
    if (a.cols <= 8192) return forward<DT, VB, kWords ? 1024 : 512, kWords ? 8 : 16>(a, sms, stream);
    // few wide bf16 rows by fewer threads (a shorter chain for a row), many by more (a row's loads cover another's reductions)
    if constexpr (DT == kBF16) { if (a.rows * a.cols <= 55000ll * sms) return forward<DT, VB, 512, 32>(a, sms, stream); }
    return forward<DT, VB, 1024, 16>(a, sms, stream);
}
template <int DT, int VB> cudaError_t backward_by_width(const NormBackArgs& a, int sms, int* used, cudaStream_t stream) {
    if (a.cols <= 64) return backward<DT, VB, 8, 8>(a, sms, used, stream);
    if (a.cols <= 256) return backward<DT, VB, 32, 8>(a, sms, used, stream);
    if (a.cols <= 512) return backward<DT, VB, 64, 8>(a, sms, used, stream);
    if (a.cols <= 1024) return backward<DT, VB, 128, 8>(a, sms, used, stream);
    if (a.cols <= 2048) return backward<DT, VB, 256, 8>(a, sms, used, stream);
    if (a.cols <= 4096) return backward<DT, VB, 256, 16>(a, sms, used, stream);
    if (a.cols <= 8192) return backward<DT, VB, VB == 16 ? 512 : 1024, VB == 16 ? 16 : 8>(a, sms, used, stream);
    return ring_backward<DT, VB, 32>(a, sms, used, stream);
}

bool aligned(const void* p, long long ld, int elem, int bytes) {
    return !p || ((uintptr_t)p % bytes == 0 && (ld * elem) % bytes == 0);
}

}  // namespace


cudaError_t launch_norm_forward(NormArgs a, int dtype, int sms, cudaStream_t stream) {
    if (a.rows == 0 || a.cols == 0) return cudaSuccess;
    const int e = dtype == kF32 ? 4 : 2;
    a.weight_vec = (uintptr_t)a.weight % 16 == 0;
    a.bias_vec = (uintptr_t)a.bias % 16 == 0;
    if (a.cols > kRingWidth) {
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
    return all(16) ? forward_by_width<kBF16, 16>(a, sms, stream) : forward_by_width<kBF16, 2>(a, sms, stream);
}

cudaError_t launch_norm_backward(NormBackArgs a, int dtype, void* dweight, void* dbias, int sms, cudaStream_t stream) {
    if (a.cols == 0) return cudaSuccess;
    if (!dweight && !dbias) a.partials = nullptr;
    const int e = dtype == kF32 ? 4 : 2;
    a.weight_vec = (uintptr_t)a.weight % 16 == 0;
    int used = 0;
    cudaError_t err = cudaSuccess;
    if (a.rows > 0 && a.cols > kRingWidth) {
        if (a.partials) {
            used = norm_partial_rows(a.rows, a.cols);
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
        if (dtype == kF32) err = all(16) ? backward_by_width<kF32, 16>(a, sms, &used, stream) : backward_by_width<kF32, 4>(a, sms, &used, stream);
        else err = all(16) ? backward_by_width<kBF16, 16>(a, sms, &used, stream) : backward_by_width<kBF16, 2>(a, sms, &used, stream);
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
