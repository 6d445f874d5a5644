// Layer norm, forward and backward, for sm_103a.
//
//   k_norm_forward    y = (x - mean) r w + b,  r = 1 / sqrt(var + eps)
//   k_norm_backward   with n = (x - mean) r and g = dy w:  dx = r (g - mean(g) - n mean(g n)), and each
//                     CTA's sums of dy n and dy over its rows
//   k_norm_params     those sums added up: the gradients of the weight and the bias
//
// HBM bounds all of it: some ten operations an element of 2 or 4 bytes read and written once.  A group of
// threads holds a row in registers, so that the mean, the variance about it and the output come from one
// reading, and keeps its columns' weights, and in the backward pass their sums, in registers from row to row.
// Rows come by bulk copies into a ring of shared memory, several ahead (with one row ahead in registers
// instead, 16384 x 4096 bf16 took 254 us forward and backward where it takes 180 now, and 50000 x 1001 fp32 316
// instead of 203).
#include "tula_ring.h"
#include "tula_tc.cuh"

namespace {

constexpr int kMostThreads = 512;  // of a CTA
// Of an SM, that registers are left for.  (Forward with 512 too, of an earlier form: 79 us instead of 71 for 16384 x
// 4096 bf16; rows off 16-byte boundaries took 78 us with 512, 160 with 768, for 50000 x 1001.)
constexpr int kForwardThreads = 768, kBackwardThreads = 512;
constexpr int forward_threads(bool vec) { return vec ? kForwardThreads : kBackwardThreads; }
constexpr int kMostCluster = 8;
// Elements that a thread holds of a row.  What each row costs every warp (exchanges, of which an SM does one a
// cycle, barriers, addresses) is spread over as many: with eight a thread 16384 x 4096 bf16 took 133 us forward.
constexpr int kN = 16;
constexpr int kMostStages = 8;

struct NormArgs {
    const void *x, *dy, *w, *b;
    void *y;                  // or dx (NULL: not wanted)
    float *stats;             // [rows][2]: mean, r
    float *parts;             // [CTAs][2][cols]: sums of dy n and of dy
    long long rows, stride, dy_stride;
    int cols, group;          // threads to a row in a CTA, a power of two: all of it, or at most that
    int cluster;              // CTAs to a row
    int share;                // columns of a CTA: all, or a multiple of 16 and none without any
    int stages;               // of the ring
    long long last_copied;    // rows off 16-byte boundaries: the last row that a round which is copied begins with
    int ptype;                // of w and b
    float eps;
};

__device__ __forceinline__ float value(float v) { return v; }
__device__ __forceinline__ float value(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float value(__half v) { return __half2float(v); }

__device__ __forceinline__ float2 pair_of(unsigned u, __half) {
    __half2 h;
    memcpy(&h, &u, 4);
    return __half22float2(h);
}
__device__ __forceinline__ float2 pair_of(unsigned u, __nv_bfloat16) {
    return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u));
}
__device__ __forceinline__ unsigned pair_from(float a, float b, __half) {
    const __half2 h = __floats2half2_rn(a, b);
    unsigned u;
    memcpy(&u, &h, 4);
    return u;
}
__device__ __forceinline__ unsigned pair_from(float a, float b, __nv_bfloat16) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    unsigned u;
    memcpy(&u, &h, 4);
    return u;
}

// What a thread takes of a row, or of a CTA's share of it: t of `group` parts.  Vec: it starts on a 16-byte
// boundary and has whole vectors of 16 bytes; the threads' vectors lie next to each other.  Else their
// elements do, and move one by one.
template <typename T, bool Vec>
struct Part {
    static constexpr int kElems = 16 / (int)sizeof(T), kStep = Vec ? kElems : 1;
    static __device__ __forceinline__ int column(int k, int t, int group) {
        return Vec ? (k / kElems * group + t) * kElems + k % kElems : k * group + t;
    }
    unsigned mask;  // of the elements (Vec: of the vectors) that the row has
    int at, next;   // the first one's column, columns to the next
    unsigned w[kN * sizeof(T) / 4];

    __device__ __forceinline__ Part(int t, int group, int cols) : mask(0), at(column(0, t, group)), next(kStep * group) {
#pragma unroll
        for (int k = 0; k < kN / kStep; ++k)
            if (at + k * next < cols) mask |= 1u << k;
    }
    __device__ __forceinline__ bool in(int k) const { return mask >> (k / kStep) & 1; }
    // Zero where there is none.
    __device__ __forceinline__ void load(const T *row, bool there) {
        const T *p = row + at;
#pragma unroll
        for (int k = 0; k < kN; ++k) {
            T v = T(0.f);
            if (there && in(k)) v = __ldcs(p + k * next);
            memcpy(reinterpret_cast<T *>(w) + k, &v, sizeof(T));
        }
    }
    __device__ __forceinline__ void load_shared(uint32_t row, bool there) {
        const uint32_t p = row + at * (int)sizeof(T);
        if constexpr (!Vec) {
#pragma unroll
            for (int k = 0; k < kN; ++k) {
                if constexpr (sizeof(T) == 4) {
                    w[k] = 0;
                    if (there && in(k)) asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w[k]) : "r"(p + 4 * k * next) : "memory");
                } else {
                    unsigned short v = 0;
                    if (there && in(k)) asm volatile("ld.shared.b16 %0, [%1];" : "=h"(v) : "r"(p + 2 * k * next) : "memory");
                    w[k / 2] = k & 1 ? w[k / 2] | (unsigned)v << 16 : v;
                }
            }
        } else {
#pragma unroll
            for (int k = 0; k < kN / kStep; ++k) {
                unsigned *q = w + 4 * k;
                q[0] = q[1] = q[2] = q[3] = 0;
                if (there && in(k * kStep))
                    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                                 : "=r"(q[0]), "=r"(q[1]), "=r"(q[2]), "=r"(q[3])
                                 : "r"(p + k * next * (int)sizeof(T))
                                 : "memory");
            }
        }
    }
    __device__ __forceinline__ void floats(float (&f)[kN]) const {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int k = 0; k < kN; ++k) f[k] = __uint_as_float(w[k]);
        } else {
#pragma unroll
            for (int k = 0; k < kN / 2; ++k) {
                const float2 v = pair_of(w[k], T());
                f[2 * k] = v.x;
                f[2 * k + 1] = v.y;
            }
        }
    }
    __device__ __forceinline__ void store(T *row, const float (&f)[kN]) const {
        T *p = row + at;
#pragma unroll
        for (int k = 0; k < kN; k += kStep) {
            if (!in(k)) continue;
            if constexpr (Vec && sizeof(T) == 4)
                __stcs(reinterpret_cast<float4 *>(p + k / kStep * next), make_float4(f[k], f[k + 1], f[k + 2], f[k + 3]));
            else if constexpr (Vec)
                __stcs(reinterpret_cast<uint4 *>(p + k / kStep * next),
                       make_uint4(pair_from(f[k], f[k + 1], T()), pair_from(f[k + 2], f[k + 3], T()), pair_from(f[k + 4], f[k + 5], T()),
                                  pair_from(f[k + 6], f[k + 7], T())));
            else
                put(p + k * next, f[k]);
        }
    }
    // The columns' parameters; `none` where there are none.
    template <typename W>
    __device__ __forceinline__ void params(float (&f)[kN], const W *p) const {
#pragma unroll
        for (int k = 0; k < kN; ++k)
            if (in(k)) f[k] = value(p[at + k / kStep * next + k % kStep]);
    }
    __device__ __forceinline__ void params(float (&f)[kN], const void *p, int type, float none) const {
#pragma unroll
        for (int k = 0; k < kN; ++k) f[k] = none;
        if (!p) return;
        if (type == TULA_TYPE_F32)
            params(f, static_cast<const float *>(p));
        else if (type == TULA_TYPE_BF16)
            params(f, static_cast<const __nv_bfloat16 *>(p));
        else
            params(f, static_cast<const __half *>(p));
    }
};
__device__ __forceinline__ float param(const void *p, int type, int c, float none) {
    if (!p) return none;
    return type == TULA_TYPE_F32    ? static_cast<const float *>(p)[c]
           : type == TULA_TYPE_BF16 ? value(static_cast<const __nv_bfloat16 *>(p)[c])
                                    : value(static_cast<const __half *>(p)[c]);
}

// Sums over the threads of a row, the same in all of them.  Within a warp by exchanges; a group's warps go by
// way of shared memory and a cluster's CTAs by way of each other's, two places in turn, so that one barrier
// a sum is enough (whoever writes a place again has passed the barrier of the sum between, which all reach
// after they have read it).
struct Sums {
    float warps[2][2][kMostThreads / 32];
    float2 ctas[2][kMostCluster];
};
template <bool Wide>  // groups of more than a warp
struct GroupSum {
    Sums *place;
    int group, cluster, turn;
    // N sums at a time: one or two.
    template <int N>
    __device__ __forceinline__ void operator()(float (&v)[N]) {
        for (int o = Wide ? 16 : group / 2; o; o >>= 1)
#pragma unroll
            for (int m = 0; m < N; ++m) v[m] += __shfl_xor_sync(kFull, v[m], o);
        if constexpr (Wide) {
            if ((threadIdx.x & 31) == 0)
#pragma unroll
                for (int m = 0; m < N; ++m) place->warps[turn][m][threadIdx.x >> 5] = v[m];
            across(v);
        }
    }
    // The same of two, in a warp's five exchanges instead of ten: the halves go on with one each after the first.
    // (16384 x 4096 bf16 forward 76 us, 87 with ten.  The gradients of parameters leave no registers for it: 105 us
    // for 102.)
    __device__ __forceinline__ void two(float (&v)[2]) {
        const int half = Wide ? 16 : group / 2;
        if (!Wide && !half) return;  // a thread has its row
        const bool upper = threadIdx.x & half;
        float mine = upper ? v[1] : v[0];
        mine += __shfl_xor_sync(kFull, upper ? v[0] : v[1], half);
        for (int o = half / 2; o; o >>= 1) mine += __shfl_xor_sync(kFull, mine, o);
        if constexpr (Wide) {
            if ((threadIdx.x & 15) == 0) place->warps[turn][upper][threadIdx.x >> 5] = mine;
            across(v);
        } else {
            const float other = __shfl_xor_sync(kFull, mine, half);
            v[0] = upper ? other : mine;
            v[1] = upper ? mine : other;
        }
    }
    template <int N>
    __device__ __forceinline__ void across(float (&v)[N]) {
        const int warp = threadIdx.x >> 5, n = group >> 5;
        __syncthreads();
#pragma unroll
        for (int m = 0; m < N; ++m) {
            const float *at = &place->warps[turn][m][warp & ~(n - 1)];  // the group's warps, by all of its threads
            if (n == 2) {
                v[m] = at[0] + at[1];
            } else {
                v[m] = 0.f;
                for (int k = 0; k < n; k += 4) {
                    const float4 q = *reinterpret_cast<const float4 *>(at + k);
                    v[m] += (q.x + q.y) + (q.z + q.w);
                }
            }
        }
        if (cluster > 1) {
            float2 *mine = place->ctas[turn];
            if (threadIdx.x < cluster)
                asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(
                                 in_cta(smem_addr(mine + blockIdx.x % cluster), threadIdx.x)),
                             "f"(v[0]), "f"(v[N - 1])
                             : "memory");
            cluster_sync();
#pragma unroll
            for (int m = 0; m < N; ++m) v[m] = 0.f;
            for (int k = 0; k < cluster; ++k) {
                v[0] += mine[k].x;
                if (N > 1) v[N - 1] += mine[k].y;
            }
        }
        turn ^= 1;
    }
    __device__ __forceinline__ float operator()(float v) {
        float one[1] = {v};
        (*this)(one);
        return one[0];
    }
};

// The ring: stage s holds the rows of one round of the CTA's groups, of each of N matrices.  Rows off 16-byte
// boundaries come with what shares their first and last 16 bytes; a round beside which the matrix may not go on so
// far is read directly.  A wait that runs out leaves what is there: the others end at once then, nothing more is
// fetched (a barrier whose phase is not over may not be armed again, nor may a copy be issued over another), and
// the error word says so.
template <typename T, int N, bool Vec>
struct Ring {
    uint32_t at, bars;  // shared addresses
    volatile int *dead;
    int stages, per, bytes;  // rows to a round; bytes of a row
    long long last;          // row that a round which is copied begins with

    __device__ __forceinline__ int pitch() const { return Vec ? bytes : (bytes + 15) / 16 * 16 + 16; }
    __device__ __forceinline__ uint32_t place(int s, int m) const { return at + (s * N + m) * per * pitch(); }
    __device__ __forceinline__ bool direct(long long r0) const { return !Vec && (r0 == 0 || r0 > last); }
    __device__ __forceinline__ bool joined(long long stride) const { return stride * (long long)sizeof(T) == bytes; }
    static __device__ __forceinline__ unsigned off(const T *p) { return Vec ? 0u : (unsigned)reinterpret_cast<unsigned long long>(p) & 15u; }
    // Where row g of the round that starts with `from` lies.
    __device__ __forceinline__ uint32_t row(int s, int m, int g, const T *from, long long stride) const {
        if constexpr (Vec) return place(s, m) + g * bytes;
        return joined(stride) ? place(s, m) + off(from) + g * bytes : place(s, m) + g * pitch() + off(from + g * stride);
    }
    // Of rows r0 to r0 + n, the first ones at `from`; by one warp.
    __device__ __forceinline__ void fetch(int s, long long r0, const T *const (&from)[N], const long long (&stride)[N], int n) {
        const int lane = threadIdx.x & 31;
        const uint32_t bar = bars + 8 * s;
        if (__any_sync(kFull, *dead)) return;  // (*dead: also if this warp's own wait for the stage ran out)
        if (direct(r0)) {
            if (lane == 0) mbar_expect(bar, 0);
            return;
        }
        unsigned total = 0;
#pragma unroll
        for (int m = 0; m < N; ++m) {
            if (joined(stride[m]))
                total += lane == 0 ? tula::bytes_copied(off(from[m]), n * bytes) : 0u;
            else
                for (int g = lane; g < n; g += 32) total += tula::bytes_copied(off(from[m] + g * stride[m]), bytes);
        }
        total = __reduce_add_sync(kFull, total);
        if (lane == 0) mbar_expect(bar, total);
        __syncwarp();
#pragma unroll
        for (int m = 0; m < N; ++m) {
            if (joined(stride[m])) {
                const unsigned o = off(from[m]);
                if (lane == 0)
                    bulk_load(place(s, m), reinterpret_cast<const unsigned char *>(from[m]) - o, tula::bytes_copied(o, n * bytes), bar);
            } else {
                for (int g = lane; g < n; g += 32) {
                    const T *p = from[m] + g * stride[m];
                    const unsigned o = off(p);
                    bulk_load(place(s, m) + g * pitch(), reinterpret_cast<const unsigned char *>(p) - o, tula::bytes_copied(o, bytes), bar);
                }
            }
        }
    }
    __device__ __forceinline__ void wait(int s, unsigned parity) { mbar_wait(bars + 8 * s, parity, dead); }
    // No copy may be in flight when the CTA ends.  Nothing was fetched after the wait that ran out had begun: every
    // copy has had its whole limit, and here a millisecond more.
    __device__ __forceinline__ void leave() const {
        if (*dead)
            for (int w = 0; w < 1000; ++w) __nanosleep(1000);
    }
};

template <typename T, int N, bool Vec>
__device__ __forceinline__ void start_ring(const Ring<T, N, Vec> &ring) {
    if (threadIdx.x == 0) {
        for (int s = 0; s < ring.stages; ++s) mbar_init(ring.bars + 8 * s, 1);
        *ring.dead = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
}

// The mean comes in two parts: `near` is off by the roundings of its sum, each of them one of the row's size, and
// what the differences to it add up to, the rest of the mean, is that but for roundings of the differences' size.
// So a row of equal values gives b (but for 1e-9), and a row's offset costs no digits.  (From `near` alone 1000 columns of 1000.0
// had a mean of 1000.00006 and outputs of -0.019 w + b.)  The variance about near + rest from the mean of the
// squares about near; a NaN stays.
__device__ __forceinline__ float variance(float squares, float rest) {
    const float v = fmaf(-rest, rest, squares);
    return v < 0.f ? 0.f : v;
}

template <typename T, bool Vec, bool Wide>
__global__ void __launch_bounds__(forward_threads(Vec)) k_norm_forward(const NormArgs a) {
    using P = Part<T, Vec>;
    extern __shared__ __align__(128) unsigned char memory[];  // the ring
    __shared__ __align__(16) Sums place;
    __shared__ __align__(8) unsigned long long bars[kMostStages];
    __shared__ volatile int dead;
    const int per = blockDim.x / a.group, g = threadIdx.x / a.group, t = threadIdx.x & (a.group - 1);
    const int col0 = blockIdx.x % a.cluster * a.share, cols = min(a.cols - col0, a.share);  // the CTA's share
    const long long block = blockIdx.x / a.cluster, step = (long long)(gridDim.x / a.cluster) * per;
    const int bytes = cols * (int)sizeof(T);
    Ring<T, 1, Vec> ring{smem_addr(memory), smem_addr(bars), &dead, a.stages, per, bytes, a.last_copied};
    start_ring(ring);
    let_next_start();
    if (a.cluster > 1) cluster_sync();  // the other CTAs' shared memory may be written to from here on
    wait_for_previous();
    GroupSum<Wide> sum{&place, a.group, a.cluster, 0};
    const float inv = 1.f / (float)a.cols;
    const T *const x[1] = {static_cast<const T *>(a.x) + col0};
    const long long stride[1] = {a.stride};
    const long long first = block * per;
    P now(t, a.group, cols);
    if (threadIdx.x < 32) {
        long long r0 = first;
        for (int s = 0; s < a.stages && r0 < a.rows; ++s, r0 += step) {
            const T *const from[1] = {x[0] + r0 * a.stride};
            ring.fetch(s, r0, from, stride, (int)min((long long)per, a.rows - r0));
        }
    }
    const int psize = a.ptype == TULA_TYPE_F32 ? 4 : 2;
    float w[kN], b[kN];
    now.params(w, a.w ? static_cast<const char *>(a.w) + col0 * psize : nullptr, a.ptype, 1.f);
    now.params(b, a.b ? static_cast<const char *>(a.b) + col0 * psize : nullptr, a.ptype, 0.f);
    int s = 0;
    unsigned parity = 0;
    // (all threads of a CTA go round as often: groups beyond the last row take part in the exchanges)
    for (long long r0 = first; r0 < a.rows; r0 += step) {
        const long long r = r0 + g;
        const bool there = r < a.rows;
        ring.wait(s, parity);
        if (ring.direct(r0))
            now.load(x[0] + r * a.stride, there);
        else
            now.load_shared(ring.row(s, 0, g, x[0] + r0 * a.stride, a.stride), there);
        float c[kN], part[2] = {0.f, 0.f};
        now.floats(c);
#pragma unroll
        for (int k = 0; k < kN; ++k) part[k & 1] += c[k];
        const float near = sum(part[0] + part[1]) * inv;
        if (!Wide) __syncthreads();
        if (threadIdx.x < 32 && r0 + a.stages * step < a.rows) {  // all have read the stage
            const long long r1 = r0 + a.stages * step;
            const T *const from[1] = {x[0] + r1 * a.stride};
            ring.fetch(s, r1, from, stride, (int)min((long long)per, a.rows - r1));
        }
        if (++s == a.stages) s = 0, parity ^= 1;
        // Chains of additions to either sum (16384 x 4096: bf16 76 us with two, 86 with one; fp32, which has no
        // registers left, 102 and 95).
        constexpr int kChains = sizeof(T) == 4 ? 1 : 2;
        float rests[2] = {0.f, 0.f}, squares[2] = {0.f, 0.f};
#pragma unroll
        for (int k = 0; k < kN; ++k) {
            c[k] -= now.in(k) ? near : 0.f;  // (what the row does not have is 0)
            rests[k % kChains] += c[k];
            squares[k % kChains] = fmaf(c[k], c[k], squares[k % kChains]);
        }
        float both[2] = {rests[0] + rests[1], squares[0] + squares[1]};
        sum.two(both);
        const float rest = both[0] * inv, rstd = rsqrtf(variance(both[1] * inv, rest) + a.eps), off = -rest * rstd;
        if (there) {
#pragma unroll
            for (int k = 0; k < kN; ++k) c[k] = fmaf(fmaf(c[k], rstd, off), w[k], b[k]);
            now.store(static_cast<T *>(a.y) + r * a.cols + col0, c);
            if (a.stats && t == 0 && col0 == 0) reinterpret_cast<float2 *>(a.stats)[r] = make_float2(near + rest, rstd);
        }
    }
    ring.leave();
}

template <typename T, bool Vec, bool Wide, bool Params>
__global__ void __launch_bounds__(kBackwardThreads) k_norm_backward(const NormArgs a) {
    using P = Part<T, Vec>;
    extern __shared__ __align__(128) unsigned char memory[];  // the ring; Params: then the groups' sums
    __shared__ __align__(16) Sums place;
    __shared__ __align__(8) unsigned long long bars[kMostStages];
    __shared__ volatile int dead;
    const int per = blockDim.x / a.group, g = threadIdx.x / a.group, t = threadIdx.x & (a.group - 1);
    const int col0 = blockIdx.x % a.cluster * a.share, cols = min(a.cols - col0, a.share);  // the CTA's share
    const long long block = blockIdx.x / a.cluster, step = (long long)(gridDim.x / a.cluster) * per;
    const int bytes = cols * (int)sizeof(T);
    Ring<T, 2, Vec> ring{smem_addr(memory), smem_addr(bars), &dead, a.stages, per, bytes, a.last_copied};
    start_ring(ring);
    let_next_start();
    if (a.cluster > 1) cluster_sync();
    wait_for_previous();
    GroupSum<Wide> sum{&place, a.group, a.cluster, 0};
    const float inv = 1.f / (float)a.cols;
    const T *const x = static_cast<const T *>(a.x) + col0, *const dy = static_cast<const T *>(a.dy) + col0;
    const long long stride[2] = {a.stride, a.dy_stride};
    const float2 *stats = reinterpret_cast<const float2 *>(a.stats);
    const long long first = block * per;
    P now_x(t, a.group, cols), now_d = now_x;
    float2 now_s = make_float2(0.f, 0.f), next_s = now_s;
    if (threadIdx.x < 32) {
        long long r0 = first;
        for (int s = 0; s < a.stages && r0 < a.rows; ++s, r0 += step) {
            const T *const from[2] = {x + r0 * a.stride, dy + r0 * a.dy_stride};
            ring.fetch(s, r0, from, stride, (int)min((long long)per, a.rows - r0));
        }
    }
    if (first + g < a.rows) now_s = __ldcs(stats + first + g);
    float w[kN], dw[kN], db[kN];
    now_x.params(w, a.w ? static_cast<const char *>(a.w) + col0 * (a.ptype == TULA_TYPE_F32 ? 4 : 2) : nullptr, a.ptype, 1.f);
#pragma unroll
    for (int k = 0; k < kN; ++k) dw[k] = db[k] = 0.f;
    int s = 0;
    unsigned parity = 0;
    for (long long r0 = first; r0 < a.rows; r0 += step) {
        const long long r = r0 + g;
        const bool there = r < a.rows;
        if (r + step < a.rows) next_s = __ldcs(stats + r + step);
        ring.wait(s, parity);
        if (ring.direct(r0)) {
            now_x.load(x + r * a.stride, there);
            now_d.load(dy + r * a.dy_stride, there);
        } else {
            now_x.load_shared(ring.row(s, 0, g, x + r0 * a.stride, a.stride), there);
            now_d.load_shared(ring.row(s, 1, g, dy + r0 * a.dy_stride, a.dy_stride), there);
        }
        const float rstd = there ? now_s.y : 0.f, mean = there ? now_s.x : 0.f;
        float n[kN], d[kN], s1 = 0.f, s2 = 0.f;
        now_x.floats(n);
        now_d.floats(d);
#pragma unroll
        for (int k = 0; k < kN; ++k) {
            n[k] = (n[k] - (now_x.in(k) ? mean : 0.f)) * rstd;  // (what the row does not have is 0)
            if (Params) {
                dw[k] = fmaf(d[k], n[k], dw[k]);
                db[k] += d[k];
            }
            d[k] *= w[k];
            s1 += d[k];
            s2 = fmaf(d[k], n[k], s2);
        }
        float sums[2] = {s1, s2};
        if (a.y) sum(sums);
        if (!a.y || !Wide) __syncthreads();
        if (threadIdx.x < 32 && r0 + a.stages * step < a.rows) {  // all have read the stage
            const long long r1 = r0 + a.stages * step;
            const T *const from[2] = {x + r1 * a.stride, dy + r1 * a.dy_stride};
            ring.fetch(s, r1, from, stride, (int)min((long long)per, a.rows - r1));
        }
        if (++s == a.stages) s = 0, parity ^= 1;
        if (a.y && there) {
            const float m1 = sums[0] * inv * rstd, m2 = sums[1] * inv * rstd;
#pragma unroll
            for (int k = 0; k < kN; ++k) d[k] = fmaf(rstd, d[k], -fmaf(n[k], m2, m1));
            now_x.store(static_cast<T *>(a.y) + r * a.cols + col0, d);
        }
        now_s = next_s;
    }
    ring.leave();
    if (!Params) return;
    float *to = a.parts + (size_t)block * 2 * a.cols + col0;
    const int group = a.group;
    if (per == 1) {
#pragma unroll
        for (int k = 0; k < kN; ++k) {
            const int c = P::column(k, t, group);
            if (c < cols) to[c] = dw[k], to[a.cols + c] = db[k];
        }
        return;
    }
    // the groups' sums, in their order
    float *sums = reinterpret_cast<float *>(memory);
    __syncthreads();  // the ring has been read
#pragma unroll
    for (int k = 0; k < kN; ++k) {
        sums[(g * kN + k) * group + t] = dw[k];
        sums[((per + g) * kN + k) * group + t] = db[k];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * kN * group; i += blockDim.x) {
        const int which = i / (kN * group), j = i - which * kN * group;
        const int c = P::column(j / group, j & (group - 1), group);
        if (c >= cols) continue;
        float v = 0.f;
        for (int q = 0; q < per; ++q) v += sums[(which * per + q) * kN * group + j];
        to[which * a.cols + c] = v;
    }
}

// Additions one after the other, at most, before a sum is added to the next one's: a sum of n of a sign is off by n
// roundings in the worst case.
constexpr int kMostChain = 128;

// N sums over a row's columns, a thread's by itself: add(column, sums).
template <int N, class Add>
__device__ __forceinline__ void over_columns(float (&v)[N], int cols, Add add) {
#pragma unroll
    for (int m = 0; m < N; ++m) v[m] = 0.f;
    for (int c0 = threadIdx.x; c0 < cols; c0 += kMostChain * blockDim.x) {
        float part[N] = {};
        const int end = min(cols, c0 + kMostChain * (int)blockDim.x);
        for (int c = c0; c < end; c += blockDim.x) add(c, part);
#pragma unroll
        for (int m = 0; m < N; ++m) v[m] += part[m];
    }
}

// Rows that registers do not hold: a CTA to a row, which is read three times, or twice, mostly from L2.
template <typename T>
__global__ void __launch_bounds__(kMostThreads) k_norm_forward_wide(const NormArgs a) {
    __shared__ __align__(16) Sums place;
    let_next_start();
    wait_for_previous();
    GroupSum<true> sum{&place, (int)blockDim.x, 1, 0};
    const int cols = a.cols;
    for (long long r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T *x = static_cast<const T *>(a.x) + r * a.stride;
        float all[1], both[2];
        over_columns(all, cols, [&](int c, float (&v)[1]) { v[0] += value(x[c]); });
        const float near = sum(all[0]) / (float)cols;
        over_columns(both, cols, [&](int c, float (&v)[2]) {
            const float d = value(x[c]) - near;
            v[0] += d;
            v[1] = fmaf(d, d, v[1]);
        });
        sum(both);
        const float rest = both[0] / (float)cols, rstd = rsqrtf(variance(both[1] / (float)cols, rest) + a.eps);
        T *y = static_cast<T *>(a.y) + r * cols;
        for (int c = threadIdx.x; c < cols; c += blockDim.x) {
            const float w = param(a.w, a.ptype, c, 1.f), b = param(a.b, a.ptype, c, 0.f);
            put(y + c, fmaf((value(x[c]) - near - rest) * rstd, w, b));
        }
        if (a.stats && threadIdx.x == 0) reinterpret_cast<float2 *>(a.stats)[r] = make_float2(near + rest, rstd);
    }
}
template <typename T>
__global__ void __launch_bounds__(kMostThreads) k_norm_backward_wide(const NormArgs a) {
    __shared__ __align__(16) Sums place;
    let_next_start();
    wait_for_previous();
    GroupSum<true> sum{&place, (int)blockDim.x, 1, 0};
    const int cols = a.cols;
    for (long long r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T *x = static_cast<const T *>(a.x) + r * a.stride, *dy = static_cast<const T *>(a.dy) + r * a.dy_stride;
        const float2 st = reinterpret_cast<const float2 *>(a.stats)[r];
        float s[2];
        over_columns(s, cols, [&](int c, float (&v)[2]) {
            const float g = value(dy[c]) * param(a.w, a.ptype, c, 1.f);
            v[0] += g;
            v[1] = fmaf(g, (value(x[c]) - st.x) * st.y, v[1]);
        });
        sum(s);
        T *dx = static_cast<T *>(a.y) + r * cols;
        for (int c = threadIdx.x; c < cols; c += blockDim.x) {
            const float g = value(dy[c]) * param(a.w, a.ptype, c, 1.f);
            put(dx + c, st.y * (g - fmaf((value(x[c]) - st.x) * st.y, s[1], s[0]) / (float)cols));
        }
    }
}
// The parameters' sums of wide rows: a CTA has 256 columns and the rows of every gridDim.y-th block of 64.
template <typename T>
__global__ void __launch_bounds__(256) k_norm_sums_wide(const NormArgs a) {
    let_next_start();
    wait_for_previous();
    const int c = blockIdx.x * 256 + threadIdx.x;
    float dw = 0.f, db = 0.f;
    if (c >= a.cols) return;
    for (long long r0 = (long long)blockIdx.y * 64; r0 < a.rows; r0 += (long long)gridDim.y * 64)
        for (long long r = r0; r < min(r0 + 64, a.rows); ++r) {
            const float2 st = reinterpret_cast<const float2 *>(a.stats)[r];
            const float d = value(static_cast<const T *>(a.dy)[r * a.dy_stride + c]);
            dw = fmaf(d, (value(static_cast<const T *>(a.x)[r * a.stride + c]) - st.x) * st.y, dw);
            db += d;
        }
    float *to = a.parts + (size_t)blockIdx.y * 2 * a.cols;
    to[c] = dw;
    to[a.cols + c] = db;
}

// The parts' sums, 32 threads to a column: each those of every 32nd, then together in their order.
template <typename W>
__global__ void __launch_bounds__(1024) k_norm_params(const float *parts, int n, int cols, W *dw, W *db) {
    __shared__ float sums[32][33];
    let_next_start();
    wait_for_previous();
    const int lane = threadIdx.x & 31, turn = threadIdx.x >> 5;
    const long long c = (long long)blockIdx.x * 32 + lane;  // of both gradients
    float v = 0.f;
    if (c < 2ll * cols)
        for (int i0 = turn; i0 < n; i0 += 32 * kMostChain) {
            const int end = min(n, i0 + 32 * kMostChain);
            float part = 0.f;
#pragma unroll 4
            for (int i = i0; i < end; i += 32) part += __ldcg(parts + (size_t)i * 2 * cols + c);
            v += part;
        }
    sums[turn][lane] = v;
    __syncthreads();
    v = sums[lane][turn];  // part `lane` of column `turn`
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
    const long long at = (long long)blockIdx.x * 32 + turn;
    if (lane || at >= 2ll * cols) return;
    W *to = at < cols ? dw : db;
    if (to) put(to + (at < cols ? at : at - cols), v);
}

// ----------------------------------------------------------------------------
// Host side
// ----------------------------------------------------------------------------

// Parts that the sums over so many rounds of rows are taken in, at least: none is of more than kMostRounds, so that a
// matrix of more than that for each CTA has more CTAs than there is room for at a time.  (2^17 x 4096 bf16 backward:
// 711 us as one chain, 732 with 256, 753 with 128; the threads' sums held in memory from time to time instead, 786,
// and fewer registers for all.  The limit of their number is far beyond what memory holds.)
constexpr int kMostRounds = 2 * kMostChain;
inline long long least_parts(long long rounds) { return std::min(up(rounds, kMostRounds), 1ll << 24); }
// Those of wide rows, of kMostChain at most.
inline long long wide_parts(long long rows) {
    return std::min(std::max(std::min(64ll, up(rows, 64)), up(rows, kMostChain)), 65535ll);
}

// How rows of so many columns are shared out: the threads of a CTA to a row, the CTAs to one.
struct Layout {
    int group, threads, cluster, share;  // cluster 0: rows that registers do not hold
    unsigned grid;
    unsigned blocks() const { return grid / (unsigned)std::max(1, cluster); }
};
Layout layout_of(long long rows, int cols, int sms, int sm_threads, bool sums = false) {
    Layout l;
    const long long ctas = up(cols, kMostThreads * kN);
    l.cluster = ctas <= kMostCluster ? (int)ctas : 0;
    l.share = ctas == 1 ? cols : (int)up(up(cols, ctas), kN) * kN;
    l.group = 1;
    while (l.group < kMostThreads && l.group * kN < l.share) l.group *= 2;
    l.threads = std::max(l.group, 256);
    if (!l.cluster) {
        l.grid = (unsigned)std::min<long long>(rows, 4ll * sms);
        return l;
    }
    const long long rounds = up(rows, l.threads / l.group), resident = std::max(1, sms * (sm_threads / l.threads) / l.cluster);
    long long blocks = std::min(rounds, resident);
    // (whole waves: 2^18 x 4112 bf16 by 2048 CTAs 2.95 ms, by 14 for each SM 2.91)
    if (sums && least_parts(rounds) > resident) blocks = up(least_parts(rounds), resident) * resident;
    l.grid = (unsigned)(l.cluster * blocks);
    return l;
}

// The ring's memory: so much a thread that all threads of an SM take 192 KB.
constexpr int kRingMost = 192 * 1024;
inline int ring_bytes(const Layout &l, bool vec, size_t size, int matrices, int sm_threads, int &stages) {
    const int bytes = l.share * (int)size, pitch = vec ? bytes : (bytes + 15) / 16 * 16 + 16;  // as Ring's
    const int stage = l.threads / l.group * pitch * matrices;
    stages = std::max(1, std::min(kMostStages, kRingMost / (sm_threads / l.threads) / stage));
    return stages * stage;
}

// (of a cluster the first CTA's share, at least; all are of some thousand columns)
inline long long last_copied(const Layout &l, long long rows, size_t size) {
    return tula::last_round_copied(rows, l.threads / l.group, l.share * (int)size);
}

inline bool lies(const void *p, long long stride, size_t size) {  // rows on 16-byte boundaries
    return (reinterpret_cast<uintptr_t>(p) | (size_t)stride * size) % 16 == 0;
}

template <typename T>
int forward_typed(NormArgs &a, cudaStream_t s) {
    const bool vec = a.cols % (16 / (int)sizeof(T)) == 0 && lies(a.x, a.stride, sizeof(T)) && lies(a.y, a.cols, sizeof(T));
    const Layout l = layout_of(a.rows, a.cols, std::max(1, sm_count()), forward_threads(vec));
    if (!l.cluster) return tula::launch(k_norm_forward_wide<T>, dim3(l.grid), l.threads, 0, s, 1, a);
    a.group = l.group;
    a.cluster = l.cluster;
    a.share = l.share;
    const bool wide = l.group > 32;
    void (*k)(const NormArgs) = vec ? (wide ? k_norm_forward<T, true, true> : k_norm_forward<T, true, false>)
                                    : (wide ? k_norm_forward<T, false, true> : k_norm_forward<T, false, false>);
    static std::atomic<uint64_t> done[4];
    const int smem = ring_bytes(l, vec, sizeof(T), 1, forward_threads(vec), a.stages);
    a.last_copied = last_copied(l, a.rows, sizeof(T));
    const int rc = allow_smem((const void *)k, kRingMost, &done[2 * vec + wide]);
    return rc ? rc : tula::launch(k, dim3(l.grid), l.threads, smem, s, l.cluster, a);
}
template <typename T, bool Params>
void (*backward_kernel(bool vec, bool wide))(const NormArgs) {
    return vec ? (wide ? k_norm_backward<T, true, true, Params> : k_norm_backward<T, true, false, Params>)
               : (wide ? k_norm_backward<T, false, true, Params> : k_norm_backward<T, false, false, Params>);
}
template <typename T>
int backward_typed(NormArgs &a, void *dw, void *db, cudaStream_t s) {
    const Layout l = layout_of(a.rows, a.cols, std::max(1, sm_count()), kBackwardThreads, a.parts != nullptr);
    const long long parts = l.cluster ? (long long)l.blocks() : wide_parts(a.rows);
    int rc = TULA_OK;
    if (l.cluster) {
        a.group = l.group;
        a.cluster = l.cluster;
        a.share = l.share;
        const bool vec = a.cols % (16 / (int)sizeof(T)) == 0 && lies(a.x, a.stride, sizeof(T)) && lies(a.dy, a.dy_stride, sizeof(T)) &&
                         (!a.y || lies(a.y, a.cols, sizeof(T)));
        const bool wide = l.group > 32;
        void (*k)(const NormArgs) = a.parts ? backward_kernel<T, true>(vec, wide) : backward_kernel<T, false>(vec, wide);
        static std::atomic<uint64_t> done[8];
        int smem = ring_bytes(l, vec, sizeof(T), 2, kBackwardThreads, a.stages);
        a.last_copied = last_copied(l, a.rows, sizeof(T));
        if (a.parts && l.threads > l.group) smem = std::max(smem, 2 * l.threads * kN * 4);  // 32 KB
        rc = allow_smem((const void *)k, kRingMost, &done[4 * vec + 2 * wide + (a.parts != nullptr)]);
        if (!rc) rc = tula::launch(k, dim3(l.grid), l.threads, smem, s, l.cluster, a);
    } else {
        if (a.y) rc = tula::launch(k_norm_backward_wide<T>, dim3(l.grid), l.threads, 0, s, 1, a);
        if (!rc && a.parts)
            rc = tula::launch(k_norm_sums_wide<T>, dim3((unsigned)up(a.cols, 256), (unsigned)parts), 256, 0, s, 1, a);
    }
    if (rc || !a.parts) return rc;
    auto params = [&](auto w) {
        using W = decltype(w);
        return tula::launch(k_norm_params<W>, dim3((unsigned)up(2ll * a.cols, 32)), 1024, 0, s, 1, (const float *)a.parts,
                            (int)parts, a.cols, static_cast<W *>(dw), static_cast<W *>(db));
    };
    if (a.ptype == TULA_TYPE_F32) return params(float());
    return a.ptype == TULA_TYPE_BF16 ? params(__nv_bfloat16()) : params(__half());
}

constexpr long long kMostCols = 1LL << 24;

bool good_sizes(long long rows, long long cols) { return rows >= 0 && cols >= 0 && cols <= kMostCols && rows < (1LL << 40); }

}  // namespace

extern "C" {

int tula_layer_norm(const void *x, int type, int64_t rows, int64_t cols, int64_t stride, const void *weight, const void *bias,
                    int param_type, float eps, void *y, float *stats, void *stream) {
    if (!good_type(type) || !good_type(param_type) || !good_sizes(rows, cols) || stride < cols || !(eps >= 0.f)) return TULA_ERR_ARG;
    if (rows == 0 || cols == 0) return TULA_OK;
    const unsigned size = type_size(type), psize = type_size(param_type);
    if (!x || !y || !aligned(x, size) || !aligned(y, size) || !aligned(weight, psize) || !aligned(bias, psize) || !aligned(stats, 8))
        return TULA_ERR_ARG;
    NormArgs a = {};
    a.x = x;
    a.w = weight;
    a.b = bias;
    a.y = y;
    a.stats = stats;
    a.rows = rows;
    a.cols = (int)cols;
    a.stride = stride;
    a.eps = eps;
    a.ptype = param_type;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (type == TULA_TYPE_F32) return forward_typed<float>(a, s);
    return type == TULA_TYPE_BF16 ? forward_typed<__nv_bfloat16>(a, s) : forward_typed<__half>(a, s);
}

int tula_layer_norm_workspace_size(int64_t rows, int64_t cols, size_t *bytes) {
    if (!bytes || !good_sizes(rows, cols)) return TULA_ERR_ARG;
    *bytes = 0;
    if (cols == 0) return TULA_OK;
    // as many parts as a GPU of up to 256 SMs has CTAs (of 256 threads, two an SM), or more of long sums
    const Layout l = layout_of(rows, (int)cols, 256, kBackwardThreads);
    const long long resident = 2 * 256, least = l.cluster ? least_parts(up(rows, l.threads / l.group)) : 0;
    long long parts = std::min(std::max<long long>(rows, 1), resident);
    if (least > 1) parts = std::max(parts, least + resident);
    if (!l.cluster) parts = wide_parts(std::max<long long>(rows, 1));
    *bytes = (size_t)parts * 2 * (size_t)cols * 4;
    return TULA_OK;
}

int tula_layer_norm_backward(const void *dy, int64_t dy_stride, const void *x, int64_t stride, int type, int64_t rows, int64_t cols,
                             const void *weight, int param_type, const float *stats, void *dx, void *dweight, void *dbias,
                             void *workspace, size_t workspace_bytes, void *stream) {
    if (!good_type(type) || !good_type(param_type) || !good_sizes(rows, cols) || stride < cols || dy_stride < cols) return TULA_ERR_ARG;
    if (cols == 0 || (!dx && !dweight && !dbias)) return TULA_OK;
    const unsigned size = type_size(type), psize = type_size(param_type);
    if (!aligned(weight, psize) || !aligned(dweight, psize) || !aligned(dbias, psize)) return TULA_ERR_ARG;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (rows == 0) {
        for (void *p : {dweight, dbias}) {
            const cudaError_t e = p ? cudaMemsetAsync(p, 0, (size_t)cols * psize, s) : cudaSuccess;
            if (e != cudaSuccess) return cuda_failed(e);
        }
        return TULA_OK;
    }
    if (!dy || !x || !stats || !aligned(dy, size) || !aligned(x, size) || !aligned(dx, size) || !aligned(stats, 8)) return TULA_ERR_ARG;
    size_t need = 0;
    tula_layer_norm_workspace_size(rows, cols, &need);
    if ((dweight || dbias) && (!workspace || workspace_bytes < need || !aligned(workspace, 16) || sm_count() > 256)) return TULA_ERR_WORKSPACE;
    NormArgs a = {};
    a.x = x;
    a.dy = dy;
    a.w = weight;
    a.y = dx;
    a.stats = const_cast<float *>(stats);
    a.parts = dweight || dbias ? static_cast<float *>(workspace) : nullptr;
    a.rows = rows;
    a.cols = (int)cols;
    a.stride = stride;
    a.dy_stride = dy_stride;
    a.ptype = param_type;
    if (type == TULA_TYPE_F32) return backward_typed<float>(a, dweight, dbias, s);
    return type == TULA_TYPE_BF16 ? backward_typed<__nv_bfloat16>(a, dweight, dbias, s) : backward_typed<__half>(a, dweight, dbias, s);
}

int tula_layer_norm_check_wait_timeout(void *stream) { return check_wait_timeout(stream); }

int tula_layer_norm_error(void *stream, int *error_out) { return read_error(stream, error_out); }

}  // extern "C"
