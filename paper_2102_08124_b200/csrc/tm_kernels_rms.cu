// The residual branch: dropout from a counter-based generator, and the root-mean-square norm of the residual sum.
//
//   dropout    d(x)_c = x_c / (1 - p) where column c of the row stays, else 0;  y = d(x) (+ residual)
//   forward    h = d(x) (+ residual);  r = (mean_c h^2 + eps)^(-1/2);  y = h r w
//              8 bits: a scale s = max(max |y| / 448, 2^-126) for every group of columns, and y / s rounded to e4m3
//   backward   g = dy w;  xh = h r;  dh = r (g - xh mean_c (g xh)) (+ dsum);  dx = d(dh);  dw = sum_rows dy xh
//
// Which columns stay is worked out again from the seed wherever it is needed, the backward pass included.  A block of the generator is eight columns of
// 16 bits, so that its ten rounds (80 cycles a warp and scheduler, the wide products) come to 10 cycles a column, below what memory takes.
//
// Bound: HBM by bytes, and with wide rows or single-element accesses the number of instructions and the latency of a row.  A row belongs to a group
// of 32 to 1024 threads, by its width, and stays in their registers between the one reduction and the output: the largest magnitude that an 8-bit
// scale needs is reduced with the squares, since the row's factor is above zero.  Groups go through the rows with a stride; the next row is asked for, or
// brought to L2, before this one is reduced; weights stay in registers; a thread owns its columns in all rows, so the weight's gradient grows in
// registers and a block leaves one partial row, which a second kernel adds up in a fixed order (or few rows' one cluster itself).
// Measured in a replayed graph (copy bandwidth 6.53 TB/s): dropout with residual 16384 x 1024 bf16 18.3 us (5.5 TB/s), without 16384 x 1024 fp32 23.3 us
// (5.8); forward with dropout, residual and sum 16384 x 1024 bf16 24.6 us (5.5), 8000 x 4096 43.1 us (6.1), 2000 x 16384 52.4 us (5.0), plain 4097 x
// 1001 fp32 5.9 us (5.5), 2047 x 8191 bf16 21.6 us (3.1); 8 bits with residual and sum, 128 columns a scale, 8192 x 4096 bf16 39.0 us (6.0); backward with
// dropout and dsum 16384 x 1024 bf16 33.3 us (5.0, of which about 3 for the second kernel), 8000 x 4096 58.2 us (5.6), plain 2047 x 8191 34.6 us (2.9).
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
__device__ __forceinline__ void drop_block(const Philox& key, const DropSpec& d, long long r, long long c, float (&v)[8]) {
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

// x / d rounded down for x below 2^31, by a product: m = ceil(2^(31 + bits) / d) with d <= 2^bits
struct Divide {
    uint32_t d, m, shift;
    explicit Divide(uint32_t d_) : d(d_) {
        uint32_t bits = 0;
        while (bits < 31 && (1u << bits) < d) ++bits;
        shift = bits;
        m = (uint32_t)(((1ull << (31 + bits)) + d - 1) / d);
    }
    __device__ __forceinline__ uint32_t operator()(uint32_t x) const { return (uint32_t)(((unsigned long long)x * m) >> (31 + shift)); }
};

// What is added where there is no residual: -0, which leaves a zero its sign
template <int DT> constexpr uint32_t kNothing = DT == kF32 ? 0x80000000u : 0x80008000u;

// A thread a block of eight columns (16 bytes of bf16; twice that of fp32, the last half perhaps past the row), kEach of them at a time
constexpr int kDropThreads = 256, kDropBlocks = 5;
template <int DT, bool DROP> __global__ void __launch_bounds__(kDropThreads, kDropBlocks) dropout_kernel(const DropoutArgs a, const Divide by, uint32_t all) {
    constexpr int kEach = DT == kBF16 ? 2 : 1, V = RowType<DT>::kVec, N = 8 / V;
    const Philox key(a.drop.keys, a.drop.offset, a.drop.offset_dev);
    const uint32_t step = gridDim.x * kDropThreads, high = a.drop.limit << 16;
    const int cols = (int)min(a.cols, (long long)INT32_MAX);
    for (uint32_t i0 = blockIdx.x * kDropThreads + threadIdx.x; i0 < all; i0 += kEach * step) {
        uint4 x[kEach][N], s[kEach][N];
        uint32_t r[kEach], c[kEach];
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            const uint32_t i = i0 + k * step;
            r[k] = by(i);
            c[k] = (i - r[k] * by.d) * 8;
#pragma unroll
            for (int q = 0; q < N; ++q) {
                x[k][q] = make_uint4(0, 0, 0, 0);
                s[k][q] = make_uint4(kNothing<DT>, kNothing<DT>, kNothing<DT>, kNothing<DT>);
                if (i < all && (int)c[k] + q * V < cols) {
                    x[k][q] = *reinterpret_cast<const uint4*>(row_of<DT>(a.x, a.ld_x, r[k]) + c[k] + q * V);
                    if (a.residual) s[k][q] = *reinterpret_cast<const uint4*>(row_of<DT>(a.residual, a.ld_residual, r[k]) + c[k] + q * V);
                }
            }
        }
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            const uint4 w = DROP ? key(c[k] / 8, r[k]) : make_uint4(0, 0, 0, 0);
            const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int q = 0; q < N; ++q) {
                float v[V], t[V];
                unpack_vector<DT>(x[k][q], v);
                unpack_vector<DT>(s[k][q], t);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const uint32_t word = u[(q * V + j) / 2];
                    if (DROP) v[j] = (j & 1 ? word : word << 16) >= high ? v[j] * a.drop.scale : 0.0f;      // a dropped Inf or NaN is gone
                    v[j] += t[j];
                }
                uint32_t o[4];
                pack_words<DT, 4>(v, o);
                if (i0 + k * step < all && (int)c[k] + q * V < cols)
                    *reinterpret_cast<uint4*>(row_of<DT>(a.y, a.ld_y, r[k]) + c[k] + q * V) = make_uint4(o[0], o[1], o[2], o[3]);
            }
        }
    }
}
// Rows that start anywhere, or more blocks than 32 bits count: a warp takes 256 columns of a row in eight accesses side by side.  Lane k
// works out which columns of block k stay; a column's bit comes from there.
template <int DT> __global__ void __launch_bounds__(kDropThreads) dropout_any_kernel(const DropoutArgs a) {
    using T = typename RowType<DT>::T;
    const Philox key(a.drop.keys, a.drop.offset, a.drop.offset_dev);
    const long long parts = (a.cols + 255) / 256, all = a.rows * parts, step = (long long)gridDim.x * (kDropThreads / 32);
    const int lane = threadIdx.x & 31;
    for (long long i = (long long)blockIdx.x * (kDropThreads / 32) + (threadIdx.x >> 5); i < all; i += step) {
        const long long r = i / parts, c0 = (i - r * parts) * 256;
        const T *x = row_of<DT>(a.x, a.ld_x, r) + c0 + lane, *s = a.residual ? row_of<DT>(a.residual, a.ld_residual, r) + c0 + lane : nullptr;
        T* y = row_of<DT>(a.y, a.ld_y, r) + c0 + lane;
        const int left = (int)min(256ll, a.cols - c0) - lane;
        float v[8], w[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            v[j] = 32 * j < left ? to_float(x[32 * j]) : 0.0f;
            w[j] = s && 32 * j < left ? to_float(s[32 * j]) : -0.0f;
        }
        const uint32_t kept = a.drop.limit ? kept_bits(key((uint32_t)(c0 / 8) + lane, (uint32_t)r), a.drop.limit) : 0xFFu;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t bits = __shfl_sync(0xFFFFFFFFu, kept, 4 * j + lane / 8);
            if (32 * j < left) from_float(y + 32 * j, ((bits >> (lane & 7)) & 1u ? v[j] * a.drop.scale : 0.0f) + w[j]);
        }
    }
}

// ---- a row in registers --------------------------------------------------------------------------------------------

constexpr int kPlain = 0, kDrop = 1, kE4m3 = 2;      // forms of the kernels below

// How a row is accessed: VB = 16: all rows of all matrices start on 16-byte boundaries; VB = kLead: every matrix's row starts `lead` elements behind
// such a boundary, and the threads' columns start at -lead, so that accesses are whole vectors but at the row's ends; VB = kAny: an element
// at a time.  With kLead a group of threads keeps to rows of one lead (rows repeat it), so that its columns' weights, sums and random numbers stay its own.
constexpr int kLead = 0;
template <int DT> constexpr int kAny = RowType<DT>::kBytes;

// A row's address from 32-bit numbers is one instruction; matrices of more rows or longer pitches go to the wide kernels
template <int DT> __device__ __forceinline__ const typename RowType<DT>::T* row_at(const void* p, uint32_t pitch, uint32_t r) {
    return reinterpret_cast<const typename RowType<DT>::T*>(static_cast<const char*>(p) + (unsigned long long)pitch * r);
}
template <int DT> __device__ __forceinline__ typename RowType<DT>::T* row_at(void* p, uint32_t pitch, uint32_t r) {
    return reinterpret_cast<typename RowType<DT>::T*>(static_cast<char*>(p) + (unsigned long long)pitch * r);
}
// A matrix that is read
struct Of {
    const void* p;
    uint32_t pitch, rows;
    template <int DT> __device__ __forceinline__ const typename RowType<DT>::T* row(uint32_t r) const { return row_at<DT>(p, pitch, r); }
};

// A vector from column c on, an element at a time: at the matrix's very first and last elements
template <int DT> __device__ __noinline__ uint4 first_or_last(const typename RowType<DT>::T* row, int c, int cols) {
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < RowType<DT>::kVec; ++j) {
        if (c + j < 0 || c + j >= cols) continue;
        if constexpr (DT == kF32) w[j] = __float_as_uint(row[c + j]);
        else w[j / 2] |= (uint32_t)__bfloat16_as_ushort(row[c + j]) << (16 * (j & 1));
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

template <int DT, int VB, int TPR, int E> struct Row : RowRegs<DT, VB, TPR, E> {
    using R = RowRegs<DT, VB, TPR, E>;
    using T = typename RowType<DT>::T;
    using Raw = typename R::Raw;
    static __device__ __forceinline__ int column(int i, int) { return R::column(i); }
    static __device__ __forceinline__ void load(const Of& m, uint32_t r, int cols, int, float2 (&v)[E / 2]) { R::load(m.row<DT>(r), cols, v); }
    static __device__ __forceinline__ void ask(const Of& m, uint32_t r, int cols, int, Raw (&u)[R::NV]) { R::ask(m.row<DT>(r), cols, u); }
    static __device__ __forceinline__ void ends(const Of&, long long, int, int, Raw (&)[R::NV]) {}
    static __device__ __forceinline__ void inside(int, int, float2 (&)[E / 2]) {}
    static __device__ __forceinline__ void store(T* row, int cols, int, const float2 (&v)[E / 2]) { R::store(row, cols, v); }
    static __device__ __forceinline__ void params(const void* p, bool f32, bool vec, int cols, int, float2 (&v)[E / 2]) { R::params(p, f32, vec, cols, v, 1.0f); }
    // VE values of row from column c on
    static __device__ __forceinline__ void some(const Of& m, uint32_t r, int c, int, float* v) { R::A::load(reinterpret_cast<const char*>(m.row<DT>(r) + c), v); }
    static __device__ __forceinline__ bool any(int c, int cols) { return c < cols; }
};
template <int DT, int TPR, int E> struct Row<DT, kLead, TPR, E> : RowRegs<DT, 16, TPR, E> {
    using R = RowRegs<DT, 16, TPR, E>;
    using T = typename RowType<DT>::T;
    using Raw = uint4;
    static constexpr int VE = R::VE, NV = R::NV;
    static __device__ __forceinline__ int column(int i, int lead) { return R::column(i) - lead; }
    static __device__ __forceinline__ bool any(int c, int cols) { return cols > 0 && c + VE > 0 && c < cols; }      // cols is 0 where there is no row
    // Vectors at a row's ends reach into its neighbours (rows are a vector long at least), and are read whole; but for those that would lie before the
    // matrix's first element or behind its last one, whose elements ends() adds
    static __device__ __forceinline__ bool whole(uint32_t r, uint32_t rows, int c, int cols) {
        return any(c, cols) && (c >= 0 || r > 0) && (c + VE <= cols || r + 1 < rows);
    }
    static __device__ __forceinline__ uint4 vector(const Of& m, uint32_t r, int c, int cols) {
        uint4 u = make_uint4(0, 0, 0, 0);
        if (whole(r, m.rows, c, cols)) u = *reinterpret_cast<const uint4*>(m.row<DT>(r) + c);
        return u;
    }
    static __device__ __forceinline__ void ends(const Of& m, uint32_t r, int cols, int lead, uint4 (&u)[NV]) {
        if (r > 0 && r + 1 < m.rows) return;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = column(i, lead);
            if (any(c, cols) && !whole(r, m.rows, c, cols)) u[i] = first_or_last<DT>(m.row<DT>(r), c, cols);
        }
    }
    static __device__ __forceinline__ void ask(const Of& m, uint32_t r, int cols, int lead, uint4 (&u)[NV]) {
#pragma unroll
        for (int i = 0; i < NV; ++i) u[i] = vector(m, r, column(i, lead), cols);
    }
    static __device__ __forceinline__ void load(const Of& m, uint32_t r, int cols, int lead, float2 (&v)[E / 2]) {
        uint4 u[NV];
        ask(m, r, cols, lead, u);
        ends(m, r, cols, lead, u);
        R::take(u, v);
    }
    static __device__ __forceinline__ void some(const Of& m, uint32_t r, int c, int cols, float* v) {
        uint4 u = vector(m, r, c, cols);
        if (any(c, cols) && !whole(r, m.rows, c, cols)) u = first_or_last<DT>(m.row<DT>(r), c, cols);
        unpack_vector<DT>(u, v);
    }
    // zeros in the place of what lies before and behind the row
    static __device__ __forceinline__ void inside(int cols, int lead, float2 (&v)[E / 2]) {
        float* f = reinterpret_cast<float*>(v);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = column(i, lead);
            if (c >= 0 && c + VE <= cols) continue;
#pragma unroll
            for (int j = 0; j < VE; ++j) f[i * VE + j] = c + j >= 0 && c + j < cols ? f[i * VE + j] : 0.0f;
        }
    }
    static __device__ __forceinline__ void store(T* row, int cols, int lead, const float2 (&v)[E / 2]) {
        const float* f = reinterpret_cast<const float*>(v);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = column(i, lead);
            if (c >= 0 && c + VE <= cols) R::A::store(row + c, f + i * VE);
            else if (any(c, cols)) {
#pragma unroll
                for (int j = 0; j < VE; ++j) if (c + j >= 0 && c + j < cols) from_float(row + c + j, f[i * VE + j]);
            }
        }
    }
    static __device__ __forceinline__ void params(const void* p, bool f32, bool, int cols, int lead, float2 (&v)[E / 2]) {
        float* f = reinterpret_cast<float*>(v);
#pragma unroll
        for (int k = 0; k < E; ++k) {
            const int c = column(k / VE, lead) + k % VE;
            f[k] = 0.0f;
            if (c >= 0 && c < cols) load_params<1>(p, f32, false, c, f + k, 1.0f);
        }
    }
};

// brings row r of two matrices to L2, a line a thread: half the threads cover a row of 16 elements a thread
template <int DT, int TPR> __device__ __forceinline__ void fetch_rows(const void* a, uint32_t pitch_a, const void* b, uint32_t pitch_b, uint32_t r, uint32_t rows, int cols) {
    const int t = threadIdx.x % TPR, c = (t & (TPR / 2 - 1)) * (128 / RowType<DT>::kBytes);
    if (r < rows && c < cols) asm volatile("prefetch.global.L2 [%0];" ::"l"((t < TPR / 2 ? row_at<DT>(a, pitch_a, r) : row_at<DT>(b, pitch_b, r)) + c));
}

// Dropout of what TPR >= 32 threads hold of a row.  A warp's lanes work out one block of eight columns each; accesses that are narrower than a
// block, or start inside one, take their columns' bits from the lanes that have them (with a lead, an access touches one block more: lane i has
// access i's).
template <int DT, int VB, int TPR, int E> __device__ __forceinline__ void drop_row(const Philox& key, const DropSpec& d, uint32_t r, int lead, float2 (&v)[E / 2]) {
    using R = Row<DT, VB, TPR, E>;
    constexpr int VE = R::VE, NV = R::NV, A = 8 / VE, B = 4 * VE;      // accesses that a warp's 32 blocks are, and blocks of each
    float* f = reinterpret_cast<float*>(v);
    const int t = threadIdx.x % TPR, lane = threadIdx.x & 31;
    const auto first = [&](int i) { return (i * TPR + t - lane) * VE - lead; };      // the warp's first column in access i
    uint32_t more = 0;
    if constexpr (VB == kLead) more = kept_bits(key((uint32_t)((first(min(lane, NV - 1)) >> 3) + B), r), d.limit);
#pragma unroll
    for (int k = 0; k < NV / A; ++k) {
        const uint4 w = key((uint32_t)((first(k * A + lane / B) >> 3) + lane % B), r);
        if constexpr (VE == 8 && VB != kLead) {
            const uint32_t high = d.limit << 16, u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int j = 0; j < 8; ++j) f[8 * k + j] = (j & 1 ? u[j / 2] : u[j / 2] << 16) >= high ? f[8 * k + j] : 0.0f;
        } else {
            const uint32_t kept = kept_bits(w, d.limit);
#pragma unroll
            for (int i = 0; i < A; ++i) {
                uint32_t bits;
                if constexpr (VB != kLead) bits = __shfl_sync(0xFFFFFFFFu, kept, i * B + lane * VE / 8) >> (lane * VE & 7);
                else {
                    const int at = (first(k * A + i) & 7) + lane * VE, q = at >> 3;      // columns from the first block's start on; block
                    const uint32_t lo = __shfl_sync(0xFFFFFFFFu, kept, i * B + min(q, B - 1)), hi = __shfl_sync(0xFFFFFFFFu, kept, i * B + min(q + 1, B - 1));
                    const uint32_t past = __shfl_sync(0xFFFFFFFFu, more, k * A + i);
                    bits = ((q < B ? lo : past) | (q + 1 < B ? hi : past) << 8) >> (at & 7);
                }
#pragma unroll
                for (int j = 0; j < VE; ++j) f[(k * A + i) * VE + j] = (bits >> j) & 1u ? f[(k * A + i) * VE + j] : 0.0f;
            }
        }
    }
    const float2 scale = make_float2(d.scale, d.scale);
#pragma unroll
    for (int k = 0; k < E / 2; ++k) v[k] = __fmul2_rn(v[k], scale);
}

// v times the parameters of its columns, an access after the other: rows whose parameters have no registers of their own.  With a lead they lie
// in shared memory as the columns do in the accesses (a block has one lead where it has one group).
template <int DT, int VB, int TPR, int E> __device__ __forceinline__ void times_params(const void* p, bool f32, bool vec, int cols, const float* shared, float2 (&v)[E / 2]) {
    using R = Row<DT, VB, TPR, E>;
    float* f = reinterpret_cast<float*>(v);
#pragma unroll
    for (int i = 0; i < R::NV; ++i) {
        float w[R::VE];
        if constexpr (VB == kLead) load_params<R::VE>(shared, true, true, R::column(i, 0), w, 1.0f);
        else if (R::column(i, 0) < cols) load_params<R::VE>(p, f32, vec, R::column(i, 0), w, 1.0f);
        else continue;
#pragma unroll
        for (int j = 0; j < R::VE; ++j) f[i * R::VE + j] *= w[j];
    }
}
template <int TPR, int E> __device__ __forceinline__ void share_params(const void* p, bool f32, int cols, int lead, float* shared) {
    for (int k = threadIdx.x; k < TPR * E; k += TPR) {
        float w = 0.0f;
        if (k >= lead && k - lead < cols) load_params<1>(p, f32, false, k - lead, &w, 1.0f);
        shared[k] = w;
    }
    __syncthreads();
}

// (sum of v.x, largest v.y) over the TPR threads of a row; buf as for row_sum2
template <int TPR, int GROUPS> __device__ __forceinline__ float2 row_sum_max(float2 v, float2* buf) {
    v = make_float2(group_sum<32>(v.x), group_max<32>(v.y));
    if constexpr (TPR <= 32) return v;
    else {
        constexpr int W = TPR / 32;
        if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = v;
        row_barrier<TPR, GROUPS>();
        const float2 t = buf[(threadIdx.x / TPR) * W + (threadIdx.x & (W - 1))];
        return make_float2(group_sum<W>(t.x), group_max<32>(t.y));
    }
}

// Threads of a block whose rows are shared by TPR threads each, and blocks an SM
template <int TPR> constexpr int kForwardThreads = TPR <= 32 ? 128 : TPR;
template <int TPR, int E> constexpr int kForwardBlocks = std::max(1, (E <= 8 ? 1024 : 768) / kForwardThreads<TPR>);
template <int TPR, int E> constexpr int kBackwardThreads = TPR <= 32 ? 128 : TPR <= 128 ? 384 : TPR <= 256 ? (E <= 8 ? 768 : 256) : TPR;
template <int TPR, int E> constexpr int kBackwardBlocks = std::max(1, (E <= 8 ? 768 : 512) / kBackwardThreads<TPR, E>);

template <int DT, int VB, int TPR, int E, int FORM>
__global__ void __launch_bounds__(kForwardThreads<TPR>, kForwardBlocks<TPR, E>) rms_forward_kernel(const RmsArgs a, bool vec8) {
    using R = Row<DT, VB, TPR, E>;
    constexpr int P = E / 2, VE = R::VE, kGroups = kForwardThreads<TPR> / TPR;
    // kAhead: the next row is asked for before this one is reduced, where the registers suffice; kFetch: else it is brought to L2
    constexpr bool kAhead = VB != kAny<DT> ? (DT == kBF16 && !(TPR == 1024 && E == 16)) || (DT == kF32 && R::NV <= 2) : E == 16 && (TPR == 256 || TPR == 512), kKeep = TPR < 1024 || E < 16, kFetch = !kAhead && TPR >= 128;
    extern __shared__ __align__(16) float shared[];       // kLead without kKeep: the weights
    __shared__ float2 buf[2][32];
    __shared__ float tops[FORM == kE4m3 && VE == 1 ? kGroups * TPR * E / 32 : 1];
    const Philox key(a.drop.keys, a.drop.offset, FORM == kDrop ? a.drop.offset_dev : nullptr);
    const int t = threadIdx.x % TPR, g = threadIdx.x / TPR, cols = (int)a.cols, lane = threadIdx.x & 31;
    const float inv_n = 1.0f / (float)a.cols;
    const uint32_t rows = (uint32_t)a.rows, step = gridDim.x * kGroups;
    constexpr uint32_t B = RowType<DT>::kBytes;
    const uint32_t pitch_x = (uint32_t)a.ld_x * B, pitch_residual = (uint32_t)a.ld_residual * B, pitch_sum = (uint32_t)a.ld_sum * B, pitch_y = (uint32_t)a.ld_y * B;
    const int lead = VB == kLead ? (int)((reinterpret_cast<uintptr_t>(row_at<DT>(a.x, pitch_x, blockIdx.x * kGroups + g)) & 15) / sizeof(typename R::T)) : 0;
    float2 w[P];
    if constexpr (VB == kLead && !kKeep) share_params<TPR, E>(a.weight, a.weight_f32, cols, lead, shared);
    if constexpr (kKeep) R::params(a.weight, a.weight_f32, a.weight_vec, cols, lead, w);
    typename R::Raw ux[R::NV], us[R::NV];
    const auto ask = [&](uint32_t r) {
        if constexpr (kAhead) {
            const int n = r < rows ? cols : 0;
            R::ask(Of{a.x, pitch_x, rows}, r, n, lead, ux);
            if (a.residual) R::ask(Of{a.residual, pitch_residual, rows}, r, n, lead, us);
        }
    };
    ask(blockIdx.x * kGroups + g);
    int turn = 0;
    for (uint32_t r0 = blockIdx.x * kGroups; r0 < rows; r0 += step, turn ^= 1) {
        const uint32_t r = r0 + g;
        const bool on = r < rows;                       // whole groups idle together, but take part in the shuffles and barriers
        float2 h[P];
        if constexpr (kAhead) {
            R::ends(Of{a.x, pitch_x, rows}, r, on ? cols : 0, lead, ux);
            R::take(ux, h);
        } else R::load(Of{a.x, pitch_x, rows}, r, on ? cols : 0, lead, h);
        if constexpr (FORM == kDrop) drop_row<DT, VB, TPR, E>(key, a.drop, r, lead, h);
        if (a.residual) {
            float2 s[P];
            if constexpr (kAhead) {
                R::ends(Of{a.residual, pitch_residual, rows}, r, on ? cols : 0, lead, us);
                R::take(us, s);
            } else R::load(Of{a.residual, pitch_residual, rows}, r, on ? cols : 0, lead, s);
#pragma unroll
            for (int k = 0; k < P; ++k) h[k] = __fadd2_rn(h[k], s[k]);
        }
        R::inside(cols, lead, h);
        ask(r + step);
        if constexpr (kFetch) fetch_rows<DT, TPR>(a.x, pitch_x, a.residual ? a.residual : a.x, a.residual ? pitch_residual : pitch_x, r + step, rows, cols);
        if (a.sum && on) R::store(row_at<DT>(a.sum, pitch_sum, r), cols, lead, h);
        float2 sq = make_float2(0.0f, 0.0f);
        float top = 0.0f;
#pragma unroll
        for (int k = 0; k < P; ++k) sq = __ffma2_rn(h[k], h[k], sq);
        if constexpr (!kKeep) times_params<DT, VB, TPR, E>(a.weight, a.weight_f32, a.weight_vec, cols, shared, h);
#pragma unroll
        for (int k = 0; k < P; ++k) {
            if constexpr (kKeep) h[k] = __fmul2_rn(h[k], w[k]);      // zeros past the last column
            if constexpr (FORM == kE4m3) top = fmaxf(top, fmaxf(fabsf(h[k].x), fabsf(h[k].y)));
        }
        float rstd;
        if constexpr (FORM == kE4m3) {
            const float2 both = row_sum_max<TPR, kGroups>(make_float2(sq.x + sq.y, top), buf[turn]);
            rstd = 1.0f / sqrtf(both.x * inv_n + a.eps);
            top = both.y;
        } else rstd = 1.0f / sqrtf(row_sum<TPR, kGroups>(sq.x + sq.y, reinterpret_cast<float*>(buf[turn])) * inv_n + a.eps);
        if (t == 0 && on && a.rstd) a.rstd[r] = rstd;
        if constexpr (FORM != kE4m3) {
            if (!on) continue;
            const float2 rr = make_float2(rstd, rstd);
#pragma unroll
            for (int k = 0; k < P; ++k) h[k] = __fmul2_rn(h[k], rr);
            R::store(row_at<DT>(a.y, pitch_y, r), cols, lead, h);
        } else {
            const float* f = reinterpret_cast<const float*>(h);
            uint8_t* y = static_cast<uint8_t*>(a.y) + (unsigned long long)(uint32_t)a.ld_y * r;
            const int shift = __ffs(a.group) - 1;          // a.group is a power of two, or 0
            float* scales = a.scales + (unsigned long long)r * (uint32_t)(a.group ? (cols + a.group - 1) >> shift : 1);
            float scale = scale_of(top * rstd);
            if (a.group == 0 && t == 0 && on) scales[0] = scale;
            if (VE == 1 && a.group) {                     // a warp's accesses are 32 columns each
                constexpr int kTops = TPR * E / 32;
                float* mine = tops + g * kTops;
#pragma unroll
                for (int i = 0; i < R::NV; ++i) {
                    const float m = group_max<32>(fabsf(f[i]));
                    if (lane == 0) mine[(i * TPR + t) / 32] = m;
                }
                row_barrier<TPR, kGroups>();
                const int n = a.group / 32, groups = kTops >> (shift - 5);
                float m = 0.0f;
                if (t < groups) {
                    for (int k = 0; k < n; ++k) m = fmaxf(m, mine[t * n + k]);
                    scale = scale_of(m * rstd);
                    if (on && t * a.group < cols) scales[t] = scale;
                    m = __fdividef(1.0f, scale);
                }
                row_barrier<TPR, kGroups>();
                if (t < groups) mine[t] = m;           // from here on the groups' inverses
                row_barrier<TPR, kGroups>();               // the next row's writes come behind its reduction, which waits for these reads
            }
            // Up to 2^126: times rstd it could leave fp32's range.  The quick inverse is good to two units; with an exact one, and an exact quotient by 448, as
            // many of 33 million values (500 and 460 to 770) fall to another neighbour than in another order of the products: those that lie on a tie but for
            // roundings.  2047 x 8191 bf16 37.2 and 39.6 to 41.6 us.
            float by = __fdividef(1.0f, scale);
#pragma unroll
            for (int i = 0; i < R::NV; ++i) {
                const int c = R::column(i, lead);
                if (a.group) {
                    if constexpr (VB == kLead) {}          // the launch takes these rows an element at a time: groups would not start with accesses
                    else if constexpr (VE == 1) by = tops[g * (TPR * E / 32) + (c >> shift)];
                    else {
                        float m = 0.0f;
#pragma unroll
                        for (int j = 0; j < VE; ++j) m = fmaxf(m, fabsf(f[i * VE + j]));
                        for (int o = a.group / VE / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
                        scale = scale_of(m * rstd);
                        by = __fdividef(1.0f, scale);
                        if (on && c < cols && (c & (a.group - 1)) == 0) scales[c >> shift] = scale;
                    }
                }
                if (!on || !R::any(c, cols)) continue;    // behind the shuffles of this access
                float q[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) q[j] = j < VE ? f[i * VE + j % VE] * rstd * by : 0.0f;
                const uint32_t lo = pack_e4m3(q[0], q[1], q[2], q[3]), hi = pack_e4m3(q[4], q[5], q[6], q[7]);
                const bool whole = VB == kLead ? c >= 0 && c + VE <= cols && (reinterpret_cast<uintptr_t>(y + c) & (VE - 1)) == 0 : vec8;
                if (VE == 8 && whole) *reinterpret_cast<uint2*>(y + c) = make_uint2(lo, hi);
                else if (VE == 4 && whole) *reinterpret_cast<uint32_t*>(y + c) = lo;
                else {
#pragma unroll
                    for (int j = 0; j < VE; ++j) if (VB != kLead || (c + j >= 0 && c + j < cols)) y[c + j] = (uint8_t)((j < 4 ? lo : hi) >> (8 * (j & 3)));
                }
            }
        }
    }
}

constexpr int kClusterWidth = 4096;                   // columns up to which few rows are one cluster's

template <int DT, int VB, int TPR, int E, int FORM>
__global__ void __launch_bounds__(kBackwardThreads<TPR, E>, kBackwardBlocks<TPR, E>) rms_backward_kernel(const RmsBackArgs a) {
    using R = Row<DT, VB, TPR, E>;
    constexpr int P = E / 2, kThreads = kBackwardThreads<TPR, E>, kGroups = kThreads / TPR;
    constexpr bool kAhead = VB != kAny<DT> && DT == kBF16 && TPR < 1024, kKeep = TPR < 1024 || E == 8, kFetch = !kAhead && (TPR == 1024 || (VB != kAny<DT> && TPR >= 128));
    __shared__ float buf[2][32];
    extern __shared__ __align__(16) float fold[];         // kGroups > 1: [cols]; kLead without kKeep: the weights
    const Philox key(a.drop.keys, a.drop.offset, FORM == kDrop ? a.drop.offset_dev : nullptr);
    const int g = threadIdx.x / TPR, cols = (int)a.cols;
    const float inv_n = 1.0f / (float)a.cols;
    const uint32_t rows = (uint32_t)a.rows, step = gridDim.x * kGroups;
    constexpr uint32_t B = RowType<DT>::kBytes;
    const uint32_t pitch_dy = (uint32_t)a.ld_dy * B, pitch_h = (uint32_t)a.ld_h * B, pitch_dsum = (uint32_t)a.ld_dsum * B, pitch_dh = (uint32_t)a.ld_dh * B, pitch_dx = (uint32_t)a.ld_dx * B;
    const int lead = VB == kLead ? (int)((reinterpret_cast<uintptr_t>(row_at<DT>(a.h, pitch_h, blockIdx.x * kGroups + g)) & 15) / sizeof(typename R::T)) : 0;
    float2 w[P], dw[P];
    if constexpr (VB == kLead && !kKeep) share_params<TPR, E>(a.weight, a.weight_f32, cols, lead, fold);
    if constexpr (kKeep) R::params(a.weight, a.weight_f32, a.weight_vec, cols, lead, w);
#pragma unroll
    for (int k = 0; k < P; ++k) dw[k] = make_float2(0.0f, 0.0f);
    int turn = 0;
    typename R::Raw ud[R::NV], ux[R::NV], ue[R::NV];
    float next_rstd = 0.0f;
    const auto ask = [&](uint32_t r) {
        if constexpr (kAhead) {
            const bool on = r < rows;
            R::ask(Of{a.dy, pitch_dy, rows}, r, on ? cols : 0, lead, ud);
            R::ask(Of{a.h, pitch_h, rows}, r, on ? cols : 0, lead, ux);
            R::ask(Of{a.dsum, pitch_dsum, rows}, r, on && a.dsum ? cols : 0, lead, ue);
            next_rstd = on ? a.rstd[r] : 0.0f;
        }
    };
    ask(blockIdx.x * kGroups + g);
    for (uint32_t r0 = blockIdx.x * kGroups; r0 < rows; r0 += step, turn ^= 1) {
        const uint32_t r = r0 + g;
        const bool on = r < rows;
        constexpr bool kLate = TPR == 1024;               // dsum is read behind the reduction
        float2 d[P], x[P], e[kLate ? 1 : P];
        float rstd;
        if constexpr (kAhead) {
            R::ends(Of{a.dy, pitch_dy, rows}, r, on ? cols : 0, lead, ud);
            R::take(ud, d);
            R::ends(Of{a.h, pitch_h, rows}, r, on ? cols : 0, lead, ux);
            R::take(ux, x);
            if constexpr (!kLate) {
                R::ends(Of{a.dsum, pitch_dsum, rows}, r, on && a.dsum ? cols : 0, lead, ue);
                R::take(ue, e);                           // zeros without a dsum
            }
            rstd = next_rstd;
        } else {
            R::load(Of{a.dy, pitch_dy, rows}, r, on ? cols : 0, lead, d);
            R::load(Of{a.h, pitch_h, rows}, r, on ? cols : 0, lead, x);
            rstd = on ? a.rstd[r] : 0.0f;
            if constexpr (!kLate) R::load(Of{a.dsum, pitch_dsum, rows}, r, on && a.dsum ? cols : 0, lead, e);
        }
        if constexpr (kFetch) {
            fetch_rows<DT, TPR>(a.dy, pitch_dy, a.h, pitch_h, r + step, rows, cols);
            if constexpr (VB != kAny<DT>) if (a.dsum) fetch_rows<DT, TPR>(a.dsum, pitch_dsum, a.dsum, pitch_dsum, r + step, rows, cols);
        }
        ask(r + step);
        R::inside(cols, lead, d);
        R::inside(cols, lead, x);
        const float2 rs = make_float2(rstd, rstd);
        float2 s2 = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int k = 0; k < P; ++k) {
            x[k] = __fmul2_rn(x[k], rs);
            dw[k] = __ffma2_rn(d[k], x[k], dw[k]);
            if constexpr (kKeep) d[k] = __fmul2_rn(d[k], w[k]);
        }
        if constexpr (!kKeep) times_params<DT, VB, TPR, E>(a.weight, a.weight_f32, a.weight_vec, cols, fold, d);
#pragma unroll
        for (int k = 0; k < P; ++k) s2 = __ffma2_rn(d[k], x[k], s2);
        const float m2 = -row_sum<TPR, kGroups>(s2.x + s2.y, buf[turn]) * inv_n;
        const float2 mm2 = make_float2(m2, m2);
#pragma unroll
        for (int k = 0; k < P; ++k) {
            d[k] = __ffma2_rn(x[k], mm2, d[k]);
            if constexpr (kLate) d[k] = __fmul2_rn(d[k], rs);
            else d[k] = __ffma2_rn(d[k], rs, e[k]);
        }
        if constexpr (kLate) {
            if (a.dsum) {
                float* f = reinterpret_cast<float*>(d);
#pragma unroll
                for (int i = 0; i < R::NV; ++i)
                    if (on && R::any(R::column(i, lead), cols)) {
                        float v[R::VE];
                        R::some(Of{a.dsum, pitch_dsum, rows}, r, R::column(i, lead), cols, v);
#pragma unroll
                        for (int j = 0; j < R::VE; ++j) f[i * R::VE + j] += v[j];
                    }
            }
        }
        if (on && a.dh) R::store(row_at<DT>(a.dh, pitch_dh, r), cols, lead, d);
        if constexpr (FORM == kDrop) drop_row<DT, VB, TPR, E>(key, a.drop, r, lead, d);
        if (on && a.dx) R::store(row_at<DT>(a.dx, pitch_dx, r), cols, lead, d);
    }
    if (!a.partials) return;
    float* out = a.dweight ? fold : a.partials + (long long)blockIdx.x * a.cols;
    const float* fw = reinterpret_cast<const float*>(dw);
    // the groups add their columns one after the other
#pragma unroll 1
    for (int k = 0; k < kGroups; ++k) {
        if (kGroups > 1) __syncthreads();
        if (g != k) continue;
        float* to = k + 1 == kGroups ? out : fold;
#pragma unroll
        for (int q = 0; q < E; ++q) {
            const int c = R::column(q / R::VE, lead) + q % R::VE;
            if (c >= 0 && c < cols) to[c] = fw[q] + (k ? fold[c] : 0.0f);
        }
    }
    if constexpr (E * TPR <= kClusterWidth) {
        if (!a.dweight) return;
        cluster_sync();
        for (int c = blockIdx.x * kThreads + threadIdx.x; c < cols; c += gridDim.x * kThreads) {
            float v = 0.0f;
            for (uint32_t k = 0; k < gridDim.x; ++k) v += cluster_load_float(fold + c, k);
            if (a.weight_f32) static_cast<float*>(a.dweight)[c] = v;
            else static_cast<__nv_bfloat16*>(a.dweight)[c] = __float2bfloat16_rn(v);
        }
        cluster_sync();                                   // no block ends while another reads its shared memory
    }
}

// Rows wider than the registers hold, and matrices that 32 bits do not count: a block a row, the row read twice.  2000 x 20000 bf16: forward with
// dropout 115 us, backward 190 us (floors 49 and 61).
constexpr int kWide = 512;
template <int DT, bool VEC, bool E8> __global__ void __launch_bounds__(kWide) wide_rms_forward_kernel(const RmsArgs a, bool vec8) {
    __shared__ float2 buf[2][32];
    const Philox key(a.drop.keys, a.drop.offset, a.drop.offset_dev);
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
    const Philox key(a.drop.keys, a.drop.offset, a.drop.offset_dev);
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

// Adds up `n` partial rows: 32 columns a block, its warps share the rows, always in the same order
constexpr int kFoldWarps = 32;
__global__ void __launch_bounds__(32 * kFoldWarps) rms_fold_kernel(const float* partials, int n, long long cols, void* dweight, int weight_f32) {
    __shared__ float s[kFoldWarps][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long c = (long long)blockIdx.x * 32 + lane;
    cudaGridDependencySynchronize();
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

constexpr long long kRegisterWidth = 16384, kMostRows = 1ll << 31;      // columns and rows of the register form

// Blocks of `rows` rows each, at most `cap`; with a lead, blocks that come round again come to rows of the same lead: those are `period` apart
unsigned blocks_of(long long rows, int groups, long long cap, int period) {
    const long long want = (rows + groups - 1) / groups;
    return (unsigned)(want <= cap ? want : std::max<long long>(cap / period, 1) * period);
}
int period_of(long long ld, int elem) {            // rows after which the lead comes again
    int n = 1;
    while (ld * elem * n % 16) n *= 2;
    return n;
}

template <int DT, int VB, int TPR, int E, int FORM> cudaError_t forward(const RmsArgs& a, int sms, cudaStream_t stream) {
    constexpr int kThreads = kForwardThreads<TPR>, kGroups = kThreads / TPR;
    const unsigned grid = blocks_of(a.rows, kGroups, (long long)kForwardBlocks<TPR, E> * sms, VB == kLead ? period_of(a.ld_x, RowType<DT>::kBytes) : 1);
    const int bytes = VB == kLead ? 1 : VB / RowType<DT>::kBytes;      // that a thread stores of y8 at a time
    auto kernel = rms_forward_kernel<DT, VB, TPR, E, FORM>;
    const size_t smem = VB == kLead && TPR == 1024 && E == 16 ? sizeof(float) * TPR * E : 0;      // the weights
    if (smem) {
        static PerDeviceOnce once;
        const cudaError_t e = once.run([&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem); });
        if (e != cudaSuccess) return e;
    }
    kernel<<<grid, kThreads, smem, stream>>>(a, (uintptr_t)a.y % bytes == 0 && a.ld_y % bytes == 0);
    return cudaGetLastError();
}
template <int DT, int VB, int TPR, int E, int FORM> cudaError_t backward(RmsBackArgs a, void* dweight, int sms, int* used, cudaStream_t stream) {
    constexpr int kThreads = kBackwardThreads<TPR, E>, kGroups = kThreads / TPR, kMost = 8;
    auto kernel = rms_backward_kernel<DT, VB, TPR, E, FORM>;
    size_t smem = kGroups > 1 && a.partials ? sizeof(float) * (size_t)a.cols : 0;                // at most 8 KB: these rows have 2048 columns or fewer
    // Few rows, three a group where a block has several groups, else one: one cluster, which needs no second launch for the weight's gradient.  64 x 1024
    // fp32: a call from Python 2 to 3 us less (17.7 us), the kernels alone 5.1 and 6.7.  24 x 3001 bf16 alone: 8.1 and, three rows
    // each, 10.8.
    if (TPR * E <= kClusterWidth && a.partials && a.rows <= (kGroups > 1 ? 3 : 1) * kMost * kGroups) {
        a.dweight = dweight;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)std::min<long long>(kMost, (a.rows + kGroups - 1) / kGroups));
        cfg.blockDim = dim3(kThreads);
        cfg.dynamicSmemBytes = sizeof(float) * (size_t)a.cols;
        cfg.stream = stream;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = cfg.gridDim.x; attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        *used = -1;
        return cudaLaunchKernelEx(&cfg, kernel, a);
    }
    const long long cap = std::min<long long>((long long)kBackwardBlocks<TPR, E> * sms, rms_partial_rows(a.rows, a.cols));
    *used = (int)blocks_of(a.rows, kGroups, cap, VB == kLead ? period_of(a.ld_h, RowType<DT>::kBytes) : 1);
    if (VB == kLead && TPR == 1024 && E == 16) {
        smem = sizeof(float) * TPR * E;                   // the weights
        static PerDeviceOnce once;
        const cudaError_t e = once.run([&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem); });
        if (e != cudaSuccess) return e;
    }
    kernel<<<(unsigned)*used, kThreads, smem, stream>>>(a);
    return cudaGetLastError();
}

// The form for a row of `cols` elements, and with a lead up to a vector less one in front of them: threads that share it, elements of each.
// Of the forms with a lead those stand here that the launches below take.
template <int DT, int VB, int FORM> cudaError_t forward_by_width(const RmsArgs& a, int sms, cudaStream_t stream) {
    if constexpr (VB == kLead && DT == kF32) return forward<DT, VB, 256, 16, FORM>(a, sms, stream);
    else {
        constexpr bool kVector = VB != kAny<DT>, kWords = kVector && DT == kF32;
        const long long width = a.cols + (VB == kLead ? RowType<DT>::kVec - 1 : 0);
        if (width <= 256) return forward<DT, VB, 32, 8, FORM>(a, sms, stream);
        if (width <= 512) return forward<DT, VB, 32, 16, FORM>(a, sms, stream);
        // an element at a time with dropout, by 16 and by 8 elements a thread: fp32 4097 x 1001 25.5 and 14.6, bf16 8000 x 3001 (rows of two leads)
        // 67.2 and 63.7
        constexpr bool kFew = !kVector && FORM == kDrop;
        if (width <= 1024) return forward<DT, VB, kVector || kFew ? 128 : 64, kVector || kFew ? 8 : 16, FORM>(a, sms, stream);
        if (width <= 2048) return forward<DT, VB, kFew ? 256 : 128, kFew ? 8 : 16, FORM>(a, sms, stream);
        if (width <= 4096) return forward<DT, VB, kFew ? 512 : 256, kFew ? 8 : 16, FORM>(a, sms, stream);
        if (width <= 8192) return forward<DT, VB, kWords ? 1024 : 512, kWords ? 8 : 16, FORM>(a, sms, stream);
        return forward<DT, VB, 1024, 16, FORM>(a, sms, stream);
    }
}
template <int DT, int VB, int FORM> cudaError_t backward_by_width(const RmsBackArgs& a, void* dweight, int sms, int* used, cudaStream_t stream) {
    const long long width = a.cols + (VB == kLead ? RowType<DT>::kVec - 1 : 0);
    if (width <= 256) return backward<DT, VB, 32, 8, FORM>(a, dweight, sms, used, stream);
    if (width <= 512) return backward<DT, VB, 64, 8, FORM>(a, dweight, sms, used, stream);
    if (width <= 1024) return backward<DT, VB, 128, 8, FORM>(a, dweight, sms, used, stream);
    if (width <= 2048) return backward<DT, VB, 256, 8, FORM>(a, dweight, sms, used, stream);
    // an element at a time, rows of two leads: bf16 8000 x 3001 by (256, 16) 259 us, (512, 8) 142; fp32 61 and 90
    constexpr bool kHalves = VB == kAny<DT> && DT == kBF16;
    if (width <= 4096) return backward<DT, VB, kHalves ? 512 : 256, kHalves ? 8 : 16, FORM>(a, dweight, sms, used, stream);
    if (width <= 8192) return backward<DT, VB, VB == 16 ? 512 : 1024, VB == 16 ? 16 : 8, FORM>(a, dweight, sms, used, stream);
    return backward<DT, VB, 1024, 16, FORM>(a, dweight, sms, used, stream);
}
template <int DT, int VB> cudaError_t forward_by_form(const RmsArgs& a, int sms, cudaStream_t stream) {
    if (a.scales) return forward_by_width<DT, VB, kE4m3>(a, sms, stream);
    if constexpr (VB != kLead || DT == kBF16) { if (a.drop.limit) return forward_by_width<DT, VB, kDrop>(a, sms, stream); }
    return forward_by_width<DT, VB, kPlain>(a, sms, stream);
}
template <int DT, int VB> cudaError_t backward_by_form(const RmsBackArgs& a, void* dweight, int sms, int* used, cudaStream_t stream) {
    return a.drop.limit && a.dx ? backward_by_width<DT, VB, kDrop>(a, dweight, sms, used, stream) : backward_by_width<DT, VB, kPlain>(a, dweight, sms, used, stream);
}
template <int DT> cudaError_t forward_by_access(const RmsArgs& a, int access, int sms, cudaStream_t stream) {
    return access == 16 ? forward_by_form<DT, 16>(a, sms, stream) : access == kLead ? forward_by_form<DT, kLead>(a, sms, stream) : forward_by_form<DT, kAny<DT>>(a, sms, stream);
}
template <int DT> cudaError_t backward_by_access(const RmsBackArgs& a, int access, void* dweight, int sms, int* used, cudaStream_t stream) {
    if constexpr (DT == kBF16) { if (access == kLead) return backward_by_form<DT, kLead>(a, dweight, sms, used, stream); }
    return access == 16 ? backward_by_form<DT, 16>(a, dweight, sms, used, stream) : backward_by_form<DT, kAny<DT>>(a, dweight, sms, used, stream);
}

// How the rows of some matrices can be accessed, all alike: 16, kLead or (for more than one element's bytes) kAny
struct Matrices {
    int elem, start = -1, step = -1;
    bool same = true, narrow = true;               // pitches that 32 bits hold
    void add(const void* p, long long ld) {
        if (!p) return;
        narrow = narrow && ld * elem <= INT32_MAX;
        const int at = (int)((uintptr_t)p % 16), by = (int)(ld * elem % 16);
        if (start < 0) { start = at; step = by; }
        same = same && at == start && by == step;
    }
    int access(long long cols) const { return !same || cols * elem < 16 ? elem : start == 0 && step == 0 && cols * elem % 16 == 0 ? 16 : kLead; }
};

template <int DT> cudaError_t dropout(const DropoutArgs& a, bool vec, int sms, cudaStream_t stream) {
    const long long blocks = (a.cols + 7) / 8;
    if (vec && a.cols <= 1 << 30 && a.rows <= (1ll << 30) / blocks) {          // counted in 31 bits, a stride beyond the last included
        const uint32_t all = (uint32_t)(a.rows * blocks);
        const unsigned grid = (unsigned)std::min<long long>((all + kDropThreads - 1) / kDropThreads, (long long)kDropBlocks * sms);
        if (a.drop.limit) dropout_kernel<DT, true><<<grid, kDropThreads, 0, stream>>>(a, Divide((uint32_t)blocks), all);
        else dropout_kernel<DT, false><<<grid, kDropThreads, 0, stream>>>(a, Divide((uint32_t)blocks), all);
    } else {
        const long long all = (a.cols + 255) / 256 * a.rows;
        dropout_any_kernel<DT><<<(unsigned)std::min<long long>((all + kDropThreads / 32 - 1) / (kDropThreads / 32), 6ll * sms), kDropThreads, 0, stream>>>(a);
    }
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_dropout(const DropoutArgs& a, int dtype, int sms, cudaStream_t stream) {
    if (a.rows == 0 || a.cols == 0) return cudaSuccess;
    const int e = dtype == kF32 ? 4 : 2;
    const bool vec = a.cols * e % 16 == 0 && aligned(a.x, a.ld_x, e) && aligned(a.residual, a.ld_residual, e) && aligned(a.y, a.ld_y, e);
    return dtype == kF32 ? dropout<kF32>(a, vec, sms, stream) : dropout<kBF16>(a, vec, sms, stream);
}

cudaError_t launch_rms_forward(RmsArgs a, int dtype, int sms, cudaStream_t stream) {
    if (a.rows == 0 || a.cols == 0) return cudaSuccess;
    const int e = dtype == kF32 ? 4 : 2;
    a.weight_vec = (uintptr_t)a.weight % 16 == 0;
    const bool e8 = a.scales != nullptr;
    const bool vec = aligned(a.x, a.ld_x, e) && aligned(a.residual, a.ld_residual, e) && aligned(a.sum, a.ld_sum, e) && (e8 || aligned(a.y, a.ld_y, e));
    Matrices m = {e};
    m.add(a.x, a.ld_x);
    m.add(a.residual, a.ld_residual);
    m.add(a.sum, a.ld_sum);
    if (!e8) m.add(a.y, a.ld_y);
    if (a.cols <= kRegisterWidth && m.narrow && a.rows <= kMostRows && a.ld_y <= INT32_MAX) {
        // With a lead, groups of columns would start inside accesses, and the widest rows have no room for it.  Else, us an element at a time and with
        // it: bf16 16000 x 999 18.3 and 16.7, 8000 x 3001 47.0 and 36.4, 4000 x 7001 60.8 and 45.4, 3000 x 9001 with dropout 119 and 91; but 2047 x
        // 8191, where it takes the next form, 21.4 and 35.9.  fp32, whose single elements fill a line a warp, 8000 x 3001 39.9 and 34.2, but with
        // dropout 59.4 and 71.0, and 4097 x 1001 5.9 and 6.8.
        int access = m.access(a.cols);
        const long long width = a.cols + 16 / e - 1;
        const bool gains = dtype == kF32 ? a.cols > 2048 && width <= 4096 && !a.drop.limit : a.cols > 8192 || width <= 8192;
        if (access == kLead && ((e8 && a.group) || width > kRegisterWidth || !gains)) access = e;
        return dtype == kF32 ? forward_by_access<kF32>(a, access, sms, stream) : forward_by_access<kBF16>(a, access, sms, stream);
    }
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
    cudaError_t err = cudaSuccess;
    const bool vec = aligned(a.dy, a.ld_dy, e) && aligned(a.h, a.ld_h, e) && aligned(a.dsum, a.ld_dsum, e) && aligned(a.dh, a.ld_dh, e) && aligned(a.dx, a.ld_dx, e);
    Matrices m = {e};
    m.add(a.dy, a.ld_dy);
    m.add(a.h, a.ld_h);
    m.add(a.dsum, a.ld_dsum);
    m.add(a.dh, a.ld_dh);
    m.add(a.dx, a.ld_dx);
    if (a.rows > 0 && a.cols <= kRegisterWidth && m.narrow && a.rows <= kMostRows) {
        // As above: bf16 16000 x 999 51.7 and 29.1, 8000 x 3001 150 and 44.5, 8000 x 5001 with dsum 149 and 102, 2047 x 8181 34.8 and 35.1, 3000 x 9001
        // with dsum 93.6 and 77.7, but 200 x 5001 8.1 and 10.4; fp32, before, 8000 x 3001 76.2 and 77.5, 4097 x 1001 18.4 and 23.6
        int access = m.access(a.cols);
        const long long width = a.cols + 16 / e - 1;
        if (access == kLead && (dtype == kF32 || width > kRegisterWidth || (width > 8192 && a.cols <= 8192))) access = e;
        err = dtype == kF32 ? backward_by_access<kF32>(a, access, dweight, sms, &used, stream) : backward_by_access<kBF16>(a, access, dweight, sms, &used, stream);
    } else if (a.rows > 0) {
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
    }
    if (err != cudaSuccess || !dweight || used < 0) return err;      // used < 0: the cluster has written it
    // rows == 0: nothing was launched and the sum over no rows is zeros (used == 0)
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((a.cols + 31) / 32));
    cfg.blockDim = dim3(32 * kFoldWarps);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, rms_fold_kernel, (const float*)a.partials, used, a.cols, dweight, (int)a.weight_f32);
}

}  // namespace tmask
