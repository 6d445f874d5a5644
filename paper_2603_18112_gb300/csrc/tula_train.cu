// The global gradient norm, clipping and AdamW over a list of tensors, for sm_103a.
//
//   k_norm   sum of squares of every gradient; the last CTA to finish turns it into the norm, the
//            clipping coefficient and the step's scalars
//   k_clip   g = coef * g
//   k_adamw  the update of w, m, v and the weights' copies
//
// All three stream: a few operations for 2 to 30 bytes, so HBM bounds them, or, for lists of a few
// hundred thousand elements, the launches.  The plan's device table (a row per tile) makes each
// pass one launch with a few bytes of parameters whatever the number of tensors, and a tile's
// addresses one load away.  Code that runs over a tile is there once for each type, so that all of a
// thread's loads are issued before the first is converted: with the type looked at vector by vector
// the norm of 184 M bf16 gradients took 101 us, 3.6 TB/s.
#include "tula_common.h"
#include "tula_train.h"

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <memory>
#include <new>
#include <vector>

namespace {

constexpr unsigned kFull = 0xffffffffu;
// Threads of a CTA that takes tiles of VPT vectors a thread: small lists want few rounds of latency, large
// ones small CTAs that come and go (with 256 threads for both, four tiles to a CTA of the norm and 8192
// elements to a tile, clipping 443 M fp16 gradients took 411 us instead of 397).
template <int VPT>
constexpr int kThreadsOf = VPT == 1 ? 256 : 128;
constexpr int kVec = 8;             // elements a thread moves at once: 16 bytes of a 16-bit type
constexpr int kSmallTile = 2048;    // elements per tile: one vector a thread
constexpr int kLargeTile = 4096;    // four
constexpr int kMaxGroup = 2;        // tiles of a CTA of the norm
constexpr int kClipGroup = 4;       // tiles of a CTA of clipping, in large lists
constexpr int kFan = 256;           // partial sums that one warp adds up
constexpr float kNormEps = 1e-6f;

// A tile of a tensor: addresses of its first element in each buffer, of which [lo, hi) are the
// tensor's.  vec: a vector of kVec elements lies on a boundary of as many bytes in every buffer.
// The tensor's first element is then at the index (its lead) at which that is so, and the first
// tile's addresses may lie before the buffers.
struct Row {
    unsigned long long g, w, m, v, copy;
    int lo, hi;
    short gtype, ctype;
    int vec;
    unsigned long long spare;
};
static_assert(sizeof(Row) == 64, "half an L2 line");

// The scalars one step's update needs, written by the norm's last CTA.
struct alignas(16) StepScalars {
    float mult, step_size, rbc2;
    int go;
};

struct Tables {
    const Row *rows;    // [n_tiles]
    int n_tiles, tile;  // elements per tile
    int group, n_groups;  // tiles per CTA of the norm
    double *part;       // [n_groups]
    double *part2;      // [ceil(n_groups / kFan)]
    unsigned *tickets;  // [1 + ceil(n_groups / kFan)], zero between launches
    StepScalars *scal;
};

__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void let_next_start() {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// ----------------------------------------------------------------------------
// Elements
// ----------------------------------------------------------------------------

__device__ __forceinline__ float2 unpack_bf16(unsigned u) {
    return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u));
}
__device__ __forceinline__ float2 unpack_f16(unsigned u) {
    __half2 h;
    memcpy(&h, &u, 4);
    return __half22float2(h);
}
__device__ __forceinline__ unsigned pack_bf16(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    unsigned u;
    memcpy(&u, &h, 4);
    return u;
}
__device__ __forceinline__ unsigned pack_f16(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    unsigned u;
    memcpy(&u, &h, 4);
    return u;
}

// kVec elements of a type as they lie in memory, at index i (a multiple of kVec).  Past L1: nothing is
// read twice, and AdamW over 184 M elements takes 744 us, 749 with streaming loads through it.
template <int Type>
struct Raw {
    static constexpr bool kWide = Type == TULA_TYPE_F32;
    unsigned w[kWide ? 8 : 4];
    __device__ __forceinline__ void load(unsigned long long base, int i) {
        if (kWide) {
            constexpr int kHalf = kWide ? 4 : 0;
            asm volatile("ld.global.cg.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                         : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[kHalf]), "=r"(w[kHalf + 1]),
                           "=r"(w[kHalf + 2]), "=r"(w[kHalf + 3])
                         : "l"(base + 4ull * i)
                         : "memory");
        } else {
            const uint4 q = __ldcg(reinterpret_cast<const uint4 *>(base + 2ull * i));
            w[0] = q.x, w[1] = q.y, w[2] = q.z, w[3] = q.w;
        }
    }
    __device__ __forceinline__ unsigned bits() const {  // or'd, with a 16-bit type's in the upper half
        unsigned b = (w[0] | w[1]) | (w[2] | w[3]);
        if (kWide) b |= (w[kWide ? 4 : 0] | w[kWide ? 5 : 0]) | (w[kWide ? 6 : 0] | w[kWide ? 7 : 0]);
        return kWide ? b : b | b << 16;
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (unsigned &u : w) u = 0;
    }
    // element k from index i, or 0
    __device__ __forceinline__ void set(int k, unsigned long long base, int i, bool there) {
        if (kWide) {
            w[k & (kWide ? 7 : 3)] = there ? __ldcg(reinterpret_cast<const unsigned *>(base) + i) : 0u;
        } else {
            const unsigned u = there ? __ldcg(reinterpret_cast<const unsigned short *>(base) + i) : 0u;
            w[k / 2 & 3] = k & 1 ? w[k / 2 & 3] | u << 16 : u;
        }
    }
    __device__ __forceinline__ void floats(float (&x)[kVec]) const {
        if (kWide) {
#pragma unroll
            for (int k = 0; k < kVec; ++k) x[k] = __uint_as_float(w[k & (kWide ? 7 : 3)]);
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float2 f = Type == TULA_TYPE_BF16 ? unpack_bf16(w[k]) : unpack_f16(w[k]);
                x[2 * k] = f.x;
                x[2 * k + 1] = f.y;
            }
        }
    }
};
__device__ __forceinline__ void load8(float (&x)[kVec], unsigned long long base, int type, int i) {
    if (type == TULA_TYPE_F32) {
        Raw<TULA_TYPE_F32> r;
        r.load(base, i);
        r.floats(x);
    } else if (type == TULA_TYPE_BF16) {
        Raw<TULA_TYPE_BF16> r;
        r.load(base, i);
        r.floats(x);
    } else {
        Raw<TULA_TYPE_F16> r;
        r.load(base, i);
        r.floats(x);
    }
}
__device__ __forceinline__ void store8(const float (&x)[kVec], unsigned long long base, int type, int i) {
    if (type == TULA_TYPE_F32) {
        asm volatile("st.global.cs.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(base + 4ull * i), "f"(x[0]), "f"(x[1]),
                     "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7])
                     : "memory");
        return;
    }
    unsigned u[4];
#pragma unroll
    for (int k = 0; k < 4; ++k)
        u[k] = type == TULA_TYPE_BF16 ? pack_bf16(x[2 * k], x[2 * k + 1]) : pack_f16(x[2 * k], x[2 * k + 1]);
    __stcs(reinterpret_cast<uint4 *>(base + 2ull * i), make_uint4(u[0], u[1], u[2], u[3]));
}
__device__ __forceinline__ float load1(unsigned long long base, int type, int i) {
    if (type == TULA_TYPE_F32) return __ldcg(reinterpret_cast<const float *>(base) + i);
    const unsigned short u = __ldcg(reinterpret_cast<const unsigned short *>(base) + i);
    return type == TULA_TYPE_BF16 ? __uint_as_float((unsigned)u << 16) : __half2float(__ushort_as_half(u));
}
__device__ __forceinline__ void store1(float x, unsigned long long base, int type, int i) {
    if (type == TULA_TYPE_F32)
        reinterpret_cast<float *>(base)[i] = x;
    else if (type == TULA_TYPE_BF16)
        reinterpret_cast<__nv_bfloat16 *>(base)[i] = __float2bfloat16_rn(x);
    else
        reinterpret_cast<__half *>(base)[i] = __float2half_rn(x);
}

// ----------------------------------------------------------------------------
// The norm
// ----------------------------------------------------------------------------

// A thread's sum of squares of N vectors; `bits`: the elements' bits, or'd.
template <int N, int Type>
__device__ __forceinline__ float square_sum(const Raw<Type> (&raw)[N], unsigned &bits) {
    float c[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < N; ++j) {
        float x[kVec];
        raw[j].floats(x);
        bits |= raw[j].bits();
#pragma unroll
        for (int k = 0; k < kVec; ++k) c[k & 3] = __fmaf_rn(x[k], x[k], c[k & 3]);
    }
    return __fadd_rn(__fadd_rn(c[0], c[1]), __fadd_rn(c[2], c[3]));
}
// Whether it is safe as it stands: in [2^-100, 2^120] nothing overflowed, and what underflowed is
// below 2^-40 of it; so is a sum of zeros.
__device__ __forceinline__ bool safe(float s, unsigned bits) {
    return (s >= 0x1p-100f && s <= 0x1p120f) || (bits << 1) == 0;
}
// Else the elements are squared again, scaled by an exact power of two: below, every element is under
// 2^-50 and is taken times 2^100; above (inf and NaN too), times 2^-72.
template <int Type>
__device__ double scaled_sum(const Raw<Type> &raw, float s) {
    const float f = s < 0x1p-100f ? 0x1p100f : 0x1p-72f;
    float x[kVec], r = 0.f;
    raw.floats(x);
#pragma unroll
    for (int k = 0; k < kVec; ++k) {
        const float y = __fmul_rn(x[k], f);
        r = __fmaf_rn(y, y, r);
    }
    return (double)r * (s < 0x1p-100f ? 0x1p-200 : 0x1p144);
}

// A warp's sum, in lane 0.  fp32 lane sums of at most 2^120 add to at most 2^125; the
// fp64 part is there in the rare warps that have one.
__device__ __forceinline__ double warp_sum(float s, double d) {
#pragma unroll
    for (int o = 16; o; o >>= 1) s = __fadd_rn(s, __shfl_xor_sync(kFull, s, o));
    if (__any_sync(kFull, d != 0.0)) {  // NaN too
#pragma unroll
        for (int o = 16; o; o >>= 1) d += __shfl_xor_sync(kFull, d, o);
        return d + (double)s;
    }
    return (double)s;
}

struct NormArgs {
    double grad_scale, max_norm;
    float inv_scale;  // 1 / grad_scale
    bool in_fp32;     // what follows from an ordinary sum of squares stays in fp32's normal range
    float *record;
    // the step's scalars (steps NULL: a norm alone)
    long long *steps;
    double log_beta1, log_beta2, lr;
    int skip;
};

// -(beta^t - 1) to fp32's precision.
__device__ __forceinline__ float one_minus_pow(double log_beta, long long t) {
    return -expm1f((float)((double)t * log_beta));
}
__device__ __forceinline__ float step_size(const NormArgs &a, long long t) {
    return __fdiv_rn((float)a.lr, one_minus_pow(a.log_beta1, t));
}
__device__ __forceinline__ float root_correction(const NormArgs &a, long long t) {
    return __fdiv_rn(1.f, __fsqrt_rn(one_minus_pow(a.log_beta2, t)));
}

__device__ void finish_norm(double total, const Tables &tb, const NormArgs &a) {
    float norm, coef = 1.f, mult;
    bool finite = true;
    if (a.in_fp32 && total >= 0x1p-100 && total <= 0x1p100) {
        // in fp32 (its root and quotients take a tenth of the time that fp64's take on this part)
        norm = __fmul_rn(__fsqrt_rn((float)total), a.inv_scale);
        if (a.max_norm > 0.0) coef = fminf(__fdiv_rn((float)a.max_norm, __fadd_rn(norm, kNormEps)), 1.f);
        mult = __fmul_rn(coef, a.inv_scale);
    } else {
        const double n = sqrt(total) / a.grad_scale;
        finite = n <= 1.7e308;
        double c = 1.0;
        if (a.max_norm > 0.0) {
            c = a.max_norm / (n + (double)kNormEps);
            if (c > 1.0) c = 1.0;      // a NaN stays
            if (n > 1.7e308) c = 0.0;  // also below an infinite threshold
        }
        norm = (float)n;
        coef = (float)c;
        mult = (float)(c / a.grad_scale);
    }
    if (a.record) {
        a.record[TULA_RECORD_NORM] = norm;
        a.record[TULA_RECORD_COEF] = coef;
        a.record[TULA_RECORD_FINITE] = finite ? 1.f : 0.f;
    }
    if (a.steps) {
        const bool go = finite || !a.skip;
        const long long t = a.steps[0] + 1;
        StepScalars s;
        s.mult = mult;
        s.step_size = step_size(a, t);
        s.rbc2 = root_correction(a, t);
        s.go = go;
        *tb.scal = s;
        if (go)
            a.steps[0] = t;
        else
            a.steps[1] += 1;
    } else {
        tb.scal->mult = coef;
    }
}

// Sum of n doubles, kFan at most, by one warp in a fixed order; in every lane.
__device__ __forceinline__ double sum_fan(const double *p, int n) {
    const int lane = threadIdx.x & 31;
    double v[kFan / 32];
#pragma unroll
    for (int k = 0; k < kFan / 32; ++k) v[k] = lane + 32 * k < n ? __ldcg(p + lane + 32 * k) : 0.0;
#pragma unroll
    for (int k = 1; k < kFan / 32; ++k) v[0] += v[k];
#pragma unroll
    for (int o = 16; o; o >>= 1) v[0] += __shfl_xor_sync(kFull, v[0], o);
    return v[0];
}

// Of a tile whose tensor begins or ends within a vector, the one vector at each end that is the tensor's
// in part: whether vector j of this thread is one.  The others are whole or not the tensor's at all.
template <int VPT>
__device__ __forceinline__ bool in_part(const Row &row, int j) {
    const int i = (j * kThreadsOf<VPT> + (int)threadIdx.x) * kVec;
    return row.vec && !(i >= row.lo && i + kVec <= row.hi) && i + kVec > row.lo && i < row.hi;
}
// Vector j of a thread's of a tile; 0 unless it is whole.
template <int VPT, int Type>
__device__ __forceinline__ bool load_whole(Raw<Type> &raw, const Row &row, int j) {
    const int i = (j * kThreadsOf<VPT> + (int)threadIdx.x) * kVec;
    const bool whole = row.vec && i >= row.lo && i + kVec <= row.hi;
    if (whole)
        raw.load(row.g, i);
    else
        raw.clear();
    return whole;
}
// Vector j element by element, those that are not the tensor's as 0.
template <int VPT, int Type>
__device__ __forceinline__ void load_elements(Raw<Type> &raw, const Row &row, int j) {
    constexpr int kThreads = kThreadsOf<VPT>;
    const int tid = threadIdx.x;
#pragma unroll
    for (int k = 0; k < kVec; ++k) {
        const int e = row.vec ? (j * kThreads + tid) * kVec + k : (j * kVec + k) * kThreads + tid;
        raw.set(k, row.g, e, e >= row.lo && e < row.hi);
    }
}

// One warp's sum over a tile, in lane 0.  Nothing but a sum stays of the elements, so that registers
// leave room for all the threads that an SM holds; where it is not safe they are loaded again.
template <int VPT, int Type>
__device__ __forceinline__ double tile_sum(const Row &row) {
    constexpr int kThreads = kThreadsOf<VPT>;
    // vectors at a time: 64 bytes a thread (in 32 registers, of which one spills as it is)
    constexpr int kAtOnce = Raw<Type>::kWide && VPT > 1 ? VPT / 2 : VPT;
    const bool full = row.vec && row.lo == 0 && row.hi == VPT * kThreads * kVec;
    float s = 0.f;
    unsigned bits = 0;
#pragma unroll 1
    for (int j0 = 0; j0 < VPT; j0 += kAtOnce) {
        Raw<Type> raw[kAtOnce];
        if (full) {
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) raw[j].load(row.g, ((j0 + j) * kThreads + (int)threadIdx.x) * kVec);
        } else {
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) load_whole<VPT>(raw[j], row, j0 + j);
        }
        s = __fadd_rn(s, square_sum(raw, bits));
    }
    if (!row.vec || row.lo % kVec || row.hi % kVec)
#pragma unroll 1
        for (int j = 0; j < VPT; ++j)
            if (!row.vec || in_part<VPT>(row, j)) {
                Raw<Type> one[1];
                load_elements<VPT>(one[0], row, j);
                s = __fadd_rn(s, square_sum(one, bits));
            }
    double d = 0.0;
    if (!safe(s, bits)) {
#pragma unroll 1
        for (int j = 0; j < VPT; ++j) {
            Raw<Type> raw;
            if (!load_whole<VPT>(raw, row, j)) load_elements<VPT>(raw, row, j);
            d += scaled_sum(raw, s);
        }
        s = 0.f;
    }
    return warp_sum(s, d);
}

// A group's rows to shared memory.  Nothing has written the table since the plan was made, so it is
// read before the kernel ahead has completed.
__device__ __forceinline__ void fetch_rows(Row (&rows)[kMaxGroup], const Tables &tb, int first, int n) {
    constexpr int kParts = sizeof(Row) / 16;
    if ((int)threadIdx.x < n * kParts)
        reinterpret_cast<uint4 *>(rows)[threadIdx.x] = __ldg(reinterpret_cast<const uint4 *>(tb.rows + first) + threadIdx.x);
    __syncthreads();
}

template <int VPT>
__global__ void __launch_bounds__(kThreadsOf<VPT>, 2048 / kThreadsOf<VPT>) k_norm(const Tables tb, const NormArgs a) {
    constexpr int kThreads = kThreadsOf<VPT>;
    __shared__ double sums[kThreads / 32];
    __shared__ __align__(16) Row rows[kMaxGroup];
    let_next_start();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int first = blockIdx.x * tb.group, n = min(tb.group, tb.n_tiles - first);
    fetch_rows(rows, tb, first, n);
    wait_for_previous();
    double acc = 0.0;  // lane 0: the warp's
    for (int t = 0; t < n; ++t) {
        const Row &row = rows[t];
        const int type = row.gtype;
        acc += type == TULA_TYPE_F32    ? tile_sum<VPT, TULA_TYPE_F32>(row)
               : type == TULA_TYPE_BF16 ? tile_sum<VPT, TULA_TYPE_BF16>(row)
                                        : tile_sum<VPT, TULA_TYPE_F16>(row);
    }
    if (lane == 0) sums[warp] = acc;
    __syncthreads();
    if (warp != 0) return;
    // The CTA's partial sum; the last of kFan CTAs adds up theirs, and the last of those all.
    const int node = blockIdx.x / kFan, n_nodes = (tb.n_groups + kFan - 1) / kFan;
    const int in_node = min(kFan, tb.n_groups - node * kFan);
    bool last_here = false;
    if (lane == 0) {
        double s = 0.0;
        for (int k = 0; k < kThreads / 32; ++k) s += sums[k];
        __stcg(tb.part + blockIdx.x, s);
        __threadfence();
        last_here = atomicAdd(tb.tickets + 1 + node, 1u) == (unsigned)in_node - 1;
    }
    if (!__shfl_sync(kFull, last_here, 0)) return;
    __threadfence();
    double total = sum_fan(tb.part + (size_t)node * kFan, in_node);
    if (lane == 0) tb.tickets[1 + node] = 0;
    if (n_nodes > 1) {
        if (lane == 0) {
            __stcg(tb.part2 + node, total);
            __threadfence();
            last_here = atomicAdd(tb.tickets, 1u) == (unsigned)n_nodes - 1;
        }
        if (!__shfl_sync(kFull, last_here, 0)) return;
        __threadfence();
        total = 0.0;
        for (int k = 0; k < n_nodes; k += kFan) total += sum_fan(tb.part2 + k, min(kFan, n_nodes - k));
        if (lane == 0) tb.tickets[0] = 0;
    }
    if (lane == 0) finish_norm(total, tb, a);
}

// ----------------------------------------------------------------------------
// Clipping
// ----------------------------------------------------------------------------

__device__ __forceinline__ void scale1(unsigned long long g, int type, int i, float c) {
    store1(__fmul_rn(load1(g, type, i), c), g, type, i);
}

template <int VPT, int Type>
__device__ __forceinline__ void tile_scale(const Row &row, float c) {
    constexpr int kThreads = kThreadsOf<VPT>;
    const int tid = threadIdx.x;
    Raw<Type> raw[VPT];
    bool whole[VPT];
#pragma unroll
    for (int j = 0; j < VPT; ++j) whole[j] = load_whole<VPT>(raw[j], row, j);
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        float x[kVec];
        raw[j].floats(x);
#pragma unroll
        for (int k = 0; k < kVec; ++k) x[k] = __fmul_rn(x[k], c);
        if (whole[j]) store8(x, row.g, Type, (j * kThreads + tid) * kVec);
    }
    if (row.vec && row.lo % kVec == 0 && row.hi % kVec == 0) return;
#pragma unroll 1
    for (int j = 0; j < VPT; ++j) {
        if (row.vec && !in_part<VPT>(row, j)) continue;
        for (int k = 0; k < kVec; ++k) {
            const int e = row.vec ? (j * kThreads + tid) * kVec + k : (j * kVec + k) * kThreads + tid;
            if (e >= row.lo && e < row.hi) scale1(row.g, Type, e, c);
        }
    }
}

// Tiles from the last to the first: what the norm read last is still in L2.  `per` of them a CTA: fewer CTAs
// have less to start where there is nothing to scale, more are dealt out more evenly where there is (443 M
// fp16 gradients, with the norm's 134 us: 161 us and 402 us with four, 147 and 410 with eight).
template <int VPT>
__global__ void __launch_bounds__(kThreadsOf<VPT>) k_clip(const Tables tb, int per) {
    let_next_start();
    wait_for_previous();
    const float c = __ldcg(&tb.scal->mult);
    if (c == 1.f) return;
    const int first = tb.n_tiles - 1 - (int)blockIdx.x * per;
    for (int t = first; t > first - per && t >= 0; --t) {
        const Row row = tb.rows[t];
        if (row.gtype == TULA_TYPE_F32)
            tile_scale<VPT, TULA_TYPE_F32>(row, c);
        else if (row.gtype == TULA_TYPE_BF16)
            tile_scale<VPT, TULA_TYPE_BF16>(row, c);
        else
            tile_scale<VPT, TULA_TYPE_F16>(row, c);
    }
}

// ----------------------------------------------------------------------------
// AdamW
// ----------------------------------------------------------------------------

struct Adam {
    float beta1, beta2, ob1, ob2, decay, eps;  // ob: 1 - beta; decay: 1 - lr * weight_decay
};

// Each operation rounds as fp32's, the root and the quotient too: a weight near zero is mostly its update,
// whose error the instructions of 2^-22 relative error would make several units in its last place.  They would
// save nothing where HBM bounds the pass (806 us for 184 M elements either way), and of a step over 0.27 M
// elements in 65 tensors 0.8 of 6.5 us.
__device__ __forceinline__ void adamw1(float g, float &w, float &m, float &v, const Adam &h,
                                       const StepScalars &s) {
    const float d = __fmul_rn(g, s.mult);
    m = __fmaf_rn(h.beta1, m, __fmul_rn(h.ob1, d));
    v = __fmaf_rn(h.beta2, v, __fmul_rn(__fmul_rn(h.ob2, d), d));
    const float den = __fmaf_rn(__fsqrt_rn(v), s.rbc2, h.eps);
    w = __fmaf_rn(-s.step_size, __fdiv_rn(m, den), __fmul_rn(w, h.decay));
}

// kVec elements' weights, moments and gradients.
struct AdamVec {
    float g[kVec], w[kVec], m[kVec], v[kVec];
    __device__ __forceinline__ void load(const Row &r, int i) {
        load8(w, r.w, TULA_TYPE_F32, i);
        load8(m, r.m, TULA_TYPE_F32, i);
        load8(v, r.v, TULA_TYPE_F32, i);
        load8(g, r.g, r.gtype, i);
    }
    __device__ __forceinline__ void update(const Row &r, int i, const Adam &h, const StepScalars &s) {
#pragma unroll
        for (int k = 0; k < kVec; ++k) adamw1(g[k], w[k], m[k], v[k], h, s);
        store8(w, r.w, TULA_TYPE_F32, i);
        store8(m, r.m, TULA_TYPE_F32, i);
        store8(v, r.v, TULA_TYPE_F32, i);
        if (r.copy) store8(w, r.copy, r.ctype, i);
    }
};
__device__ __forceinline__ void adamw_one(const Row &r, bool copy, int i, const Adam &h,
                                          const StepScalars &s) {
    float w = load1(r.w, TULA_TYPE_F32, i), m = load1(r.m, TULA_TYPE_F32, i);
    float v = load1(r.v, TULA_TYPE_F32, i);
    adamw1(load1(r.g, r.gtype, i), w, m, v, h, s);
    store1(w, r.w, TULA_TYPE_F32, i);
    store1(m, r.m, TULA_TYPE_F32, i);
    store1(v, r.v, TULA_TYPE_F32, i);
    if (copy) store1(w, r.copy, r.ctype, i);
}

// Normed: the norm's last CTA has left the step's scalars.  Else each CTA takes them from the step
// count, which the last CTA to have read it moves on.
template <int VPT, bool Normed>
__global__ void __launch_bounds__(kThreadsOf<VPT>) k_adamw(const Tables tb, const Adam h, const NormArgs a) {
    constexpr int kThreads = kThreadsOf<VPT>;
    let_next_start();
    const Row row = tb.rows[tb.n_tiles - 1 - (int)blockIdx.x];  // before the wait, as fetch_rows
    wait_for_previous();
    const int tid = threadIdx.x;
    const bool copy = row.copy != 0;
    // the first vector's loads go ahead of what the scalars wait for
    auto fits = [&](int i) { return row.vec && i >= row.lo && i + kVec <= row.hi; };
    AdamVec x;
    if (fits(tid * kVec)) x.load(row, tid * kVec);
    StepScalars s;
    if (Normed) {
        const float4 q = __ldcg(reinterpret_cast<const float4 *>(tb.scal));
        s.mult = q.x, s.step_size = q.y, s.rbc2 = q.z, s.go = __float_as_int(q.w);
        if (!s.go) return;
    } else {
        __shared__ float scalars[2];
        const long long t = *(volatile long long *)a.steps + 1;
        if (tid == 0) scalars[0] = step_size(a, t);
        if (tid == 32) scalars[1] = root_correction(a, t);
        __syncthreads();
        s.mult = a.inv_scale;
        s.step_size = scalars[0];
        s.rbc2 = scalars[1];
        // every thread has its t: the last CTA to come here moves it on
        if (tid == 64) {
            __threadfence();
            if (atomicAdd(tb.tickets, 1u) == gridDim.x - 1) {
                tb.tickets[0] = 0;
                a.steps[0] = t;
            }
        }
    }
    if (row.vec) {
#pragma unroll 1
        for (int j = 0; j < VPT; ++j) {
            const int i = (j * kThreads + tid) * kVec;
            if (fits(i)) {
                if (j > 0) x.load(row, i);
                x.update(row, i, h, s);
            } else {
                for (int k = 0; k < kVec; ++k)
                    if (i + k >= row.lo && i + k < row.hi) adamw_one(row, copy, i + k, h, s);
            }
        }
    } else {
#pragma unroll 4
        for (int k = 0; k < VPT * kVec; ++k) {
            const int i = k * kThreads + tid;
            if (i < row.hi) adamw_one(row, copy, i, h, s);
        }
    }
}

// A list without elements: the norm is 0, the step counts.
__global__ void k_empty(const Tables tb, const NormArgs a) {
    wait_for_previous();
    finish_norm(0.0, tb, a);
}

// ----------------------------------------------------------------------------
// Host side
// ----------------------------------------------------------------------------

struct Layout {
    size_t scal, tickets, part2, part, rows, total;
    int tile, group, n_groups;
};

// Tiles of the whole list at `tile` elements each, at any alignment.
bool count_tiles(const int64_t *numels, int n, int tile, long long *out) {
    long long t = 0;
    for (int i = 0; i < n; ++i) {
        if (numels[i] < 0) return false;
        if (numels[i]) t += numels[i] / tile + (numels[i] % tile + kVec - 1 + tile - 1) / tile;
        if (t >= (1LL << 31) - 1) return false;
    }
    *out = t;
    return true;
}

bool layout(const int64_t *numels, int n, Layout *L) {
    if (!numels || n < 1) return false;
    long long t;
    // Up to eight CTAs an SM small tiles spread a list over more SMs; beyond, large ones have
    // more bytes in flight and fewer partial sums.
    L->tile = kSmallTile;
    if (!count_tiles(numels, n, kSmallTile, &t) || t > 8 * 152) {
        L->tile = kLargeTile;
        if (!count_tiles(numels, n, kLargeTile, &t)) return false;
    }
    // The norm's CTAs take one tile up to 32 CTAs an SM, then two.
    const long long per = t / (16 * 152);
    L->group = per < 1 ? 1 : per > kMaxGroup ? kMaxGroup : (int)per;
    L->n_groups = (int)((t + L->group - 1) / L->group);
    const size_t nodes = ((size_t)L->n_groups + kFan - 1) / kFan;
    size_t off = 0;
    auto take = [&](size_t bytes) {
        const size_t o = off;
        off = (off + bytes + 255) & ~size_t(255);
        return o;
    };
    L->scal = take(sizeof(StepScalars));
    L->tickets = take(4 * (1 + nodes));
    L->part2 = take(8 * nodes);
    L->part = take(8 * (size_t)L->n_groups);
    L->rows = take(sizeof(Row) * (size_t)t);
    L->total = off;
    return true;
}

inline int size_of(int type) { return type == TULA_TYPE_F32 ? 4 : 2; }

int cuda_failed(cudaError_t e) {
    tula::note_cuda_error((int)e);
    return TULA_ERR_CUDA;
}

}  // namespace

struct tula_train_plan {
    int dev;
    bool weights;
    Tables tb;
};

namespace {

// The index at which the tensor starts so that vectors lie on boundaries of as many bytes in all of
// its buffers, or -1.
int lead_of(const unsigned long long *ptrs, const int *sizes, int count) {
    const int lead = (int)(ptrs[0] / (unsigned)sizes[0] % kVec);
    for (int k = 0; k < count; ++k)
        if (ptrs[k] / (unsigned)sizes[k] % kVec != (unsigned)lead) return -1;
    return lead;
}

int check_plan(tula_train_plan *plan) {
    if (!plan) return TULA_ERR_ARG;
    int dev = 0;
    const cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return cuda_failed(e);
    return dev == plan->dev ? TULA_OK : TULA_ERR_ARG;
}

// Whether finish_norm may go on from a root in [2^-50, 2^50] in fp32.  With 1 / grad_scale within 2^+-32 the
// norm is within 2^+-82, and with a threshold of 2^-32 or more the coefficient is 2^-114 or more (above fp32's
// range the threshold is inf, and the coefficient 1 all the same); the two factors' product is what an
// element is multiplied by, threshold / root or 1 / grad_scale.
bool stays_in_fp32(const NormArgs &a) {
    return a.inv_scale >= 0x1p-32f && a.inv_scale <= 0x1p32f && (a.max_norm == 0.0 || a.max_norm >= 0x1p-32);
}

int run_norm(const Tables &tb, const NormArgs &a, cudaStream_t s) {
    if (tb.n_tiles == 0) return tula::launch(k_empty, dim3(1), 1, 0, s, 1, tb, a);
    return tula::launch(tb.tile == kSmallTile ? k_norm<1> : k_norm<4>, dim3((unsigned)tb.n_groups),
                        tb.tile == kSmallTile ? kThreadsOf<1> : kThreadsOf<4>, 0, s, 1, tb, a);
}

}  // namespace

extern "C" {

int tula_train_workspace_size(const int64_t *numels, int n_tensors, size_t *bytes) {
    Layout L;
    if (!bytes || !layout(numels, n_tensors, &L)) return TULA_ERR_ARG;
    *bytes = L.total;
    return TULA_OK;
}

int tula_train_plan_create(const tula_train_tensors *t, void *workspace, size_t workspace_bytes,
                           void *stream, tula_train_plan **plan_out) {
    if (!plan_out) return TULA_ERR_ARG;
    *plan_out = nullptr;
    Layout L;
    if (!t || !t->grad_ptrs || !layout(t->numels, t->n_tensors, &L)) return TULA_ERR_ARG;
    const bool weights = t->param_ptrs != nullptr;
    if ((t->exp_avg_ptrs != nullptr) != weights || (t->exp_avg_sq_ptrs != nullptr) != weights ||
        (t->copy_ptrs && !weights))
        return TULA_ERR_ARG;
    const int n = t->n_tensors;
    std::unique_ptr<tula_train_plan> plan(new (std::nothrow) tula_train_plan());
    std::vector<Row> rows;
    if (!plan) return TULA_ERR_NO_MEMORY;
    try {
        rows.reserve((L.total - L.rows) / sizeof(Row));
        for (int i = 0; i < n; ++i) {
            const int gtype = t->grad_types ? t->grad_types[i] : TULA_TYPE_F32;
            const int ctype = t->copy_types ? t->copy_types[i] : TULA_TYPE_BF16;
            if (gtype < TULA_TYPE_F32 || gtype > TULA_TYPE_F16) return TULA_ERR_ARG;
            if (t->copy_ptrs && ctype != TULA_TYPE_BF16 && ctype != TULA_TYPE_F16) return TULA_ERR_ARG;
            const long long numel = t->numels[i];
            if (numel == 0) continue;
            unsigned long long p[5];
            int size[5], count = 0;
            auto add = [&](const void *q, int bytes) {
                p[count] = reinterpret_cast<unsigned long long>(q);
                size[count++] = bytes;
            };
            add(t->grad_ptrs[i], size_of(gtype));
            if (weights) {
                add(t->param_ptrs[i], 4);
                add(t->exp_avg_ptrs[i], 4);
                add(t->exp_avg_sq_ptrs[i], 4);
                if (t->copy_ptrs) add(t->copy_ptrs[i], 2);
            }
            for (int k = 0; k < count; ++k)
                if (!p[k] || p[k] % (unsigned)size[k]) return TULA_ERR_ARG;
            const int at = lead_of(p, size, count), lead = at < 0 ? 0 : at;
            const long long ends = numel + lead;  // index behind the tensor
            Row r;
            std::memset(&r, 0, sizeof(r));
            r.gtype = (short)gtype;
            r.ctype = (short)ctype;
            r.vec = at >= 0;
            unsigned long long *dst[5] = {&r.g, &r.w, &r.m, &r.v, &r.copy};
            for (int k = 0; k < count; ++k) *dst[k] = p[k] - (unsigned long long)(lead * size[k]);
            for (long long i0 = 0; i0 < ends; i0 += L.tile) {
                r.lo = i0 == 0 ? lead : 0;
                r.hi = (int)std::min<long long>(L.tile, ends - i0);
                rows.push_back(r);
                for (int k = 0; k < count; ++k) *dst[k] += (unsigned long long)L.tile * (unsigned)size[k];
            }
        }
    } catch (const std::bad_alloc &) {
        return TULA_ERR_NO_MEMORY;
    }
    if (!workspace || workspace_bytes < L.total || (reinterpret_cast<uintptr_t>(workspace) & 255u))
        return TULA_ERR_WORKSPACE;
    cudaError_t e = cudaGetDevice(&plan->dev);
    if (e != cudaSuccess) return cuda_failed(e);
    char *ws = static_cast<char *>(workspace);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    Tables &tb = plan->tb;
    tb.rows = reinterpret_cast<const Row *>(ws + L.rows);
    tb.n_tiles = (int)rows.size();
    tb.tile = L.tile;
    tb.group = L.group;
    tb.n_groups = (tb.n_tiles + L.group - 1) / L.group;
    tb.part = reinterpret_cast<double *>(ws + L.part);
    tb.part2 = reinterpret_cast<double *>(ws + L.part2);
    tb.tickets = reinterpret_cast<unsigned *>(ws + L.tickets);
    tb.scal = reinterpret_cast<StepScalars *>(ws + L.scal);
    plan->weights = weights;
    e = cudaMemsetAsync(ws, 0, L.part2, s);
    if (e == cudaSuccess && !rows.empty())
        e = cudaMemcpyAsync(ws + L.rows, rows.data(), sizeof(Row) * rows.size(), cudaMemcpyHostToDevice, s);
    if (e == cudaSuccess) e = cudaStreamSynchronize(s);
    if (e != cudaSuccess) return cuda_failed(e);
    *plan_out = plan.release();
    return TULA_OK;
}

int tula_train_plan_destroy(tula_train_plan *plan) {
    delete plan;
    return TULA_OK;
}

int tula_grad_norm(tula_train_plan *plan, float grad_scale, float max_norm, float *record, void *stream) {
    if (!plan || !record || (reinterpret_cast<uintptr_t>(record) & 3u) || !(grad_scale >= 0x1p-100f) || !(grad_scale <= 0x1p100f) || !(max_norm >= 0.f))
        return TULA_ERR_ARG;
    const int rc = check_plan(plan);
    if (rc) return rc;
    NormArgs a = {};
    a.grad_scale = grad_scale;
    a.inv_scale = 1.f / grad_scale;
    a.max_norm = max_norm;
    a.in_fp32 = stays_in_fp32(a);
    a.record = record;
    return run_norm(plan->tb, a, static_cast<cudaStream_t>(stream));
}

int tula_grad_clip(tula_train_plan *plan, float max_norm, float *record, void *stream) {
    if (!(max_norm > 0.f)) return TULA_ERR_ARG;
    const int rc = tula_grad_norm(plan, 1.f, max_norm, record, stream);
    if (rc || plan->tb.n_tiles == 0) return rc;
    const Tables &tb = plan->tb;
    const bool small = tb.tile == kSmallTile;
    const int per = small ? 1 : kClipGroup;
    return tula::launch(small ? k_clip<1> : k_clip<4>, dim3((unsigned)((tb.n_tiles + per - 1) / per)),
                        small ? kThreadsOf<1> : kThreadsOf<4>, 0, static_cast<cudaStream_t>(stream), 1, tb, per);
}

void tula_adamw_default_hparams(tula_adamw_hparams *hp) {
    if (!hp) return;
    std::memset(hp, 0, sizeof(*hp));
    hp->lr = 1e-3;
    hp->beta1 = 0.9;
    hp->beta2 = 0.999;
    hp->eps = 1e-8;
    hp->weight_decay = 0.01;
    hp->grad_scale = 1.0;
}

int tula_adamw_step(tula_train_plan *plan, const tula_adamw_hparams *hp, void *stream) {
    if (!plan || !hp || !plan->weights || !hp->steps) return TULA_ERR_ARG;
    auto at_least_0 = [](double v) { return v >= 0.0 && v <= 1.7e308; };
    if (!at_least_0(hp->lr) || !at_least_0(hp->eps) || !at_least_0(hp->weight_decay) ||
        !(hp->max_norm >= 0.0) || !(hp->grad_scale >= 0x1p-100) || !(hp->grad_scale <= 0x1p100) ||
        !(hp->beta1 >= 0.0 && hp->beta1 < 1.0) || !(hp->beta2 >= 0.0 && hp->beta2 < 1.0) ||
        (hp->skip_nonfinite != 0 && hp->skip_nonfinite != 1))
        return TULA_ERR_ARG;
    const bool normed = hp->max_norm > 0.0 || hp->skip_nonfinite;
    if (normed && !hp->record) return TULA_ERR_ARG;
    if ((reinterpret_cast<uintptr_t>(hp->steps) & 7u) || (reinterpret_cast<uintptr_t>(hp->record) & 3u))
        return TULA_ERR_ARG;
    int rc = check_plan(plan);
    if (rc) return rc;
    const Tables &tb = plan->tb;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    NormArgs a = {};
    a.grad_scale = hp->grad_scale;
    a.inv_scale = (float)(1.0 / hp->grad_scale);
    a.max_norm = hp->max_norm;
    a.in_fp32 = stays_in_fp32(a);
    a.record = normed ? hp->record : nullptr;
    a.steps = reinterpret_cast<long long *>(hp->steps);
    a.log_beta1 = std::log(hp->beta1);
    a.log_beta2 = std::log(hp->beta2);
    a.lr = hp->lr;
    a.skip = hp->skip_nonfinite;
    Adam h;
    h.beta1 = (float)hp->beta1;
    h.beta2 = (float)hp->beta2;
    h.ob1 = (float)(1.0 - hp->beta1);
    h.ob2 = (float)(1.0 - hp->beta2);
    h.decay = (float)(1.0 - hp->lr * hp->weight_decay);
    h.eps = (float)hp->eps;
    if (normed || tb.n_tiles == 0) {
        rc = run_norm(tb, a, s);
        if (rc || tb.n_tiles == 0) return rc;
    }
    const bool small = tb.tile == kSmallTile;
    return tula::launch(normed ? (small ? k_adamw<1, true> : k_adamw<4, true>)
                               : (small ? k_adamw<1, false> : k_adamw<4, false>),
                        dim3((unsigned)tb.n_tiles), small ? kThreadsOf<1> : kThreadsOf<4>, 0, s, 1, tb, h, a);
}

}  // extern "C"
