// Layer norm, forward and backward, for sm_103a.
//
//   k_norm_forward    y = (x - mean) r w + b,  r = 1 / sqrt(var + eps)
//   k_norm_backward   with n = (x - mean) r and g = dy w:  dx = r (g - mean(g) - n mean(g n)), and each
//                     CTA's sums of dy n and dy over its rows
//   k_norm_params     those sums added up: the gradients of the weight and the bias
//
// HBM bounds all of it: some ten operations an element of 2 or 4 bytes read and written once.  A group of
// threads holds a row in registers, so that the mean, the variance about it and the output come from one
// reading, and keeps its columns' weights, and in the backward pass their sums, in registers from row to row;
// a row's loads are issued before the one ahead of it is worked on.
#include "tula_tc.cuh"

namespace {

constexpr int kMostThreads = 1024;
constexpr int kMostCluster = 8;
constexpr int kN = 8;  // elements that a thread holds of a row

struct NormArgs {
    const void *x, *dy, *w, *b;
    void *y;                  // or dx (NULL: not wanted)
    float *stats;             // [rows][2]: mean, r
    float *parts;             // [CTAs][2][cols]: sums of dy n and of dy
    long long rows, stride, dy_stride;
    int cols, group;          // threads to a row in a CTA, a power of two: all of it, or at most that
    int cluster;              // CTAs to a row
    float eps;
};

__device__ __forceinline__ float value(float v) { return v; }
__device__ __forceinline__ float value(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float value(__half v) { return __half2float(v); }

// Part t of a row in `group` parts.  Vec: the row starts on a 16-byte boundary and has whole vectors of 16
// bytes; the threads' vectors lie next to each other.  Else their elements do, and move one by one.
template <typename T, bool Vec>
struct Part {
    static constexpr int kElems = 16 / (int)sizeof(T);
    T v[kN];
    static __device__ __forceinline__ int column(int k, int t, int group) {
        return Vec ? (k / kElems * group + t) * kElems + k % kElems : k * group + t;
    }
    __device__ __forceinline__ void load(const T *row, int t, int group, int cols) {
#pragma unroll
        for (int k = 0; k < kN; k += Vec ? kElems : 1) {
            const int c = column(k, t, group);
            if (Vec) {
                uint4 q = make_uint4(0, 0, 0, 0);
                if (c < cols) q = __ldcs(reinterpret_cast<const uint4 *>(row + c));
                memcpy(&v[k], &q, 16);
            } else {
                v[k] = T(0.f);
                if (c < cols) v[k] = __ldcs(row + c);
            }
        }
    }
    __device__ __forceinline__ void store(T *row, int t, int group, int cols, const float (&f)[kN]) {
#pragma unroll
        for (int k = 0; k < kN; k += Vec ? kElems : 1) {
            const int c = column(k, t, group);
            if (c >= cols) continue;
            if (Vec) {
                __align__(16) T y[kElems];
#pragma unroll
                for (int j = 0; j < kElems; ++j) put(&y[j], f[k + j]);
                __stcs(reinterpret_cast<uint4 *>(row + c), *reinterpret_cast<const uint4 *>(y));
            } else {
                put(&v[k], f[k]);
                row[c] = v[k];
            }
        }
    }
};

// The columns' parameters; `none` where there are none.
template <typename T, bool Vec, typename W>
__device__ __forceinline__ void load_params(float (&f)[kN], const void *p, float none, int t, int group, int cols) {
#pragma unroll
    for (int k = 0; k < kN; ++k) {
        const int c = Part<T, Vec>::column(k, t, group);
        f[k] = none;
        if (p && c < cols) f[k] = value(static_cast<const W *>(p)[c]);
    }
}

// Sums over the threads of a row, the same in all of them.  Within a warp by exchanges; a group's warps go by
// way of shared memory and a cluster's CTAs by way of each other's, two places in turn, so that one barrier
// a sum is enough (whoever writes a place again has passed the barrier of the sum between, which all reach
// after they have read it).
struct Sums {
    float2 warps[2][32], ctas[2][kMostCluster];
};
struct GroupSum {
    Sums *place;
    int group, cluster, turn;
    __device__ __forceinline__ float2 operator()(float a, float b) {
        for (int o = min(group, 32) / 2; o; o >>= 1) {
            a += __shfl_xor_sync(kFull, a, o);
            b += __shfl_xor_sync(kFull, b, o);
        }
        if (group <= 32) return make_float2(a, b);
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n = group >> 5;
        float2 *at = place->warps[turn];
        if (lane == 0) at[warp] = make_float2(a, b);
        __syncthreads();
        const float2 v = lane < n ? at[(warp & ~(n - 1)) + lane] : make_float2(0.f, 0.f);
        a = v.x, b = v.y;
        for (int o = n / 2; o; o >>= 1) {
            a += __shfl_xor_sync(kFull, a, o);
            b += __shfl_xor_sync(kFull, b, o);
        }
        a = __shfl_sync(kFull, a, 0);  // (lanes from n on hold zeros)
        b = __shfl_sync(kFull, b, 0);
        if (cluster > 1) {
            float2 *mine = place->ctas[turn];
            if (threadIdx.x < cluster)
                asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(
                                 in_cta(smem_addr(mine + blockIdx.x % cluster), threadIdx.x)),
                             "f"(a), "f"(b)
                             : "memory");
            cluster_sync();
            a = b = 0.f;
            for (int k = 0; k < cluster; ++k) {
                a += mine[k].x;
                b += mine[k].y;
            }
        }
        turn ^= 1;
        return make_float2(a, b);
    }
};

template <typename T, typename W, bool Vec>
__global__ void __launch_bounds__(kMostThreads) k_norm_forward(const NormArgs a) {
    using P = Part<T, Vec>;
    __shared__ Sums place;
    let_next_start();
    if (a.cluster > 1) cluster_sync();  // the other CTAs' shared memory may be written to from here on
    wait_for_previous();
    const int cols = a.cols, per = blockDim.x / a.group;  // rows at a time
    const int group = a.group * a.cluster, t = (threadIdx.x & (a.group - 1)) + blockIdx.x % a.cluster * a.group;
    const long long block = blockIdx.x / a.cluster, step = (long long)(gridDim.x / a.cluster) * per;
    GroupSum sum{&place, a.group, a.cluster, 0};
    float w[kN], b[kN];
    load_params<T, Vec, W>(w, a.w, 1.f, t, group, cols);
    load_params<T, Vec, W>(b, a.b, 0.f, t, group, cols);
    const float inv = 1.f / (float)cols;
    long long r = block * per + threadIdx.x / a.group;
    const T *x = static_cast<const T *>(a.x);
    P now, next;
    if (r < a.rows) now.load(x + r * a.stride, t, group, cols);
    // (all threads of a CTA go round as often: groups beyond the last row take part in the exchanges)
    for (long long r0 = block * per; r0 < a.rows; r0 += step, r += step) {
        const bool there = r < a.rows;
        if (r + step < a.rows) next.load(x + (r + step) * a.stride, t, group, cols);
        float c[kN], s = 0.f;
#pragma unroll
        for (int k = 0; k < kN; ++k) {
            c[k] = there ? value(now.v[k]) : 0.f;
            s += c[k];
        }
        const float mean = sum(s, 0.f).x * inv;
        s = 0.f;
#pragma unroll
        for (int k = 0; k < kN; ++k) {
            c[k] = P::column(k, t, group) < cols ? c[k] - mean : 0.f;
            s = fmaf(c[k], c[k], s);
        }
        const float var = sum(s, 0.f).x * inv;
        const float rstd = 1.f / sqrtf(var + a.eps);
        if (there) {
#pragma unroll
            for (int k = 0; k < kN; ++k) c[k] = fmaf(c[k] * rstd, w[k], b[k]);
            now.store(static_cast<T *>(a.y) + r * cols, t, group, cols, c);
            if (a.stats && t == 0) reinterpret_cast<float2 *>(a.stats)[r] = make_float2(mean, rstd);
        }
        now = next;
    }
}

template <typename T, typename W, bool Vec, bool Params>
__global__ void __launch_bounds__(kMostThreads) k_norm_backward(const NormArgs a) {
    using P = Part<T, Vec>;
    __shared__ Sums place;
    extern __shared__ float sums[];  // Params: [2][kN * threads], groups of less than the CTA
    let_next_start();
    if (a.cluster > 1) cluster_sync();
    wait_for_previous();
    const int cols = a.cols, per = blockDim.x / a.group;
    const int group = a.group * a.cluster, t = (threadIdx.x & (a.group - 1)) + blockIdx.x % a.cluster * a.group;
    const long long block = blockIdx.x / a.cluster, step = (long long)(gridDim.x / a.cluster) * per;
    GroupSum sum{&place, a.group, a.cluster, 0};
    float w[kN], dw[kN], db[kN];
    load_params<T, Vec, W>(w, a.w, 1.f, t, group, cols);
#pragma unroll
    for (int k = 0; k < kN; ++k) dw[k] = db[k] = 0.f;
    const float inv = 1.f / (float)cols;
    long long r = block * per + threadIdx.x / a.group;
    const T *x = static_cast<const T *>(a.x), *dy = static_cast<const T *>(a.dy);
    const float2 *stats = reinterpret_cast<const float2 *>(a.stats);
    P now_x, now_d, next_x, next_d;
    float2 now_s = make_float2(0.f, 0.f), next_s = now_s;
    if (r < a.rows) {
        now_x.load(x + r * a.stride, t, group, cols);
        now_d.load(dy + r * a.dy_stride, t, group, cols);
        now_s = __ldcs(stats + r);
    }
    for (long long r0 = block * per; r0 < a.rows; r0 += step, r += step) {
        const bool there = r < a.rows;
        if (r + step < a.rows) {
            next_x.load(x + (r + step) * a.stride, t, group, cols);
            next_d.load(dy + (r + step) * a.dy_stride, t, group, cols);
            next_s = __ldcs(stats + r + step);
        }
        float s1 = 0.f, s2 = 0.f;
        if (there) {
#pragma unroll
            for (int k = 0; k < kN; ++k) {
                const bool in = P::column(k, t, group) < cols;
                const float n = in ? (value(now_x.v[k]) - now_s.x) * now_s.y : 0.f, d = value(now_d.v[k]);
                const float g = d * w[k];
                s1 += g;
                s2 = fmaf(g, n, s2);
                if (Params) {
                    dw[k] = fmaf(d, n, dw[k]);
                    db[k] += d;
                }
            }
        }
        if (a.y) {
            const float2 s = sum(s1, s2);
            if (there) {
                float f[kN];
#pragma unroll
                for (int k = 0; k < kN; ++k) {
                    const float n = (value(now_x.v[k]) - now_s.x) * now_s.y, g = value(now_d.v[k]) * w[k];
                    f[k] = now_s.y * (g - fmaf(n, s.y, s.x) * inv);
                }
                now_x.store(static_cast<T *>(a.y) + r * cols, t, group, cols, f);
            }
        }
        now_x = next_x, now_d = next_d, now_s = next_s;
    }
    if (!Params) return;
    float *to = a.parts + (size_t)block * 2 * cols;
    if (per == 1) {
#pragma unroll
        for (int k = 0; k < kN; ++k) {
            const int c = P::column(k, t, group);
            if (c < cols) to[c] = dw[k], to[cols + c] = db[k];
        }
        return;
    }
    // the groups' sums, in their order
    const int g0 = threadIdx.x / group;
#pragma unroll
    for (int k = 0; k < kN; ++k) {
        sums[(g0 * kN + k) * group + t] = dw[k];
        sums[((per + g0) * kN + k) * group + t] = db[k];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * kN * group; i += blockDim.x) {
        const int which = i / (kN * group), j = i - which * kN * group;
        const int c = P::column(j / group, j & (group - 1), group);
        if (c >= cols) continue;
        float v = 0.f;
        for (int g = 0; g < per; ++g) v += sums[(which * per + g) * kN * group + j];
        to[which * cols + c] = v;
    }
}

// Rows that registers do not hold: a CTA to a row, which is read three times, or twice, mostly from L2.
template <typename T, typename W>
__global__ void __launch_bounds__(kMostThreads) k_norm_forward_wide(const NormArgs a) {
    __shared__ Sums place;
    let_next_start();
    wait_for_previous();
    GroupSum sum{&place, (int)blockDim.x, 1, 0};
    const int cols = a.cols;
    for (long long r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T *x = static_cast<const T *>(a.x) + r * a.stride;
        float s = 0.f;
        for (int c = threadIdx.x; c < cols; c += blockDim.x) s += value(x[c]);
        const float mean = sum(s, 0.f).x / (float)cols;
        s = 0.f;
        for (int c = threadIdx.x; c < cols; c += blockDim.x) {
            const float d = value(x[c]) - mean;
            s = fmaf(d, d, s);
        }
        const float rstd = 1.f / sqrtf(sum(s, 0.f).x / (float)cols + a.eps);
        T *y = static_cast<T *>(a.y) + r * cols;
        for (int c = threadIdx.x; c < cols; c += blockDim.x) {
            const float w = a.w ? value(static_cast<const W *>(a.w)[c]) : 1.f, b = a.b ? value(static_cast<const W *>(a.b)[c]) : 0.f;
            put(y + c, fmaf((value(x[c]) - mean) * rstd, w, b));
        }
        if (a.stats && threadIdx.x == 0) reinterpret_cast<float2 *>(a.stats)[r] = make_float2(mean, rstd);
    }
}
template <typename T, typename W>
__global__ void __launch_bounds__(kMostThreads) k_norm_backward_wide(const NormArgs a) {
    __shared__ Sums place;
    let_next_start();
    wait_for_previous();
    GroupSum sum{&place, (int)blockDim.x, 1, 0};
    const int cols = a.cols;
    for (long long r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T *x = static_cast<const T *>(a.x) + r * a.stride, *dy = static_cast<const T *>(a.dy) + r * a.dy_stride;
        const float2 st = reinterpret_cast<const float2 *>(a.stats)[r];
        float s1 = 0.f, s2 = 0.f;
        for (int c = threadIdx.x; c < cols; c += blockDim.x) {
            const float g = value(dy[c]) * (a.w ? value(static_cast<const W *>(a.w)[c]) : 1.f);
            s1 += g;
            s2 = fmaf(g, (value(x[c]) - st.x) * st.y, s2);
        }
        const float2 s = sum(s1, s2);
        T *dx = static_cast<T *>(a.y) + r * cols;
        for (int c = threadIdx.x; c < cols; c += blockDim.x) {
            const float g = value(dy[c]) * (a.w ? value(static_cast<const W *>(a.w)[c]) : 1.f);
            put(dx + c, st.y * (g - fmaf((value(x[c]) - st.x) * st.y, s.y, s.x) / (float)cols));
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

// The parts' sums in their order, eight threads to a column, in turn and then together.
template <typename W>
__global__ void __launch_bounds__(256) k_norm_params(const float *parts, int n, int cols, W *dw, W *db) {
    __shared__ float sums[8][33];
    let_next_start();
    wait_for_previous();
    const int lane = threadIdx.x & 31, turn = threadIdx.x >> 5;
    const long long c = (long long)blockIdx.x * 32 + lane;  // of both gradients
    float v = 0.f;
    if (c < 2ll * cols)
        for (int i = turn; i < n; i += 8) v += parts[(size_t)i * 2 * cols + c];
    sums[turn][lane] = v;
    __syncthreads();
    if (turn || c >= 2ll * cols) return;
    for (int k = 1; k < 8; ++k) v += sums[k][lane];
    W *to = c < cols ? dw : db;
    if (to) put(to + (c < cols ? c : c - cols), v);
}

// ----------------------------------------------------------------------------
// Host side
// ----------------------------------------------------------------------------

// How rows of so many columns are shared out: the threads of a CTA to a row, the CTAs to one.
struct Layout {
    int group, threads, cluster;  // cluster 0: rows that registers do not hold
    unsigned grid;
    unsigned blocks() const { return grid / (unsigned)std::max(1, cluster); }
};
Layout layout_of(long long rows, int cols, int sms) {
    Layout l;
    const long long parts = up(cols, kN);
    l.group = 1;
    while (l.group < kMostThreads && l.group < parts) l.group *= 2;
    l.cluster = 1;
    while (l.cluster <= kMostCluster && (long long)l.cluster * l.group < parts) l.cluster *= 2;
    l.threads = std::max(l.group, 256);
    if (l.cluster > kMostCluster) {
        l.cluster = 0;
        l.grid = (unsigned)std::min<long long>(rows, 2ll * sms);
        return l;
    }
    const long long per = l.threads / l.group, blocks = std::max(1, sms * (kMostThreads / l.threads) / l.cluster);
    l.grid = (unsigned)(l.cluster * std::min(up(rows, per), blocks));
    return l;
}
constexpr int kWideParts = 64;  // of the rows, whose sums are taken apart (wide rows)

unsigned parts_of(const Layout &l, long long rows) {
    return l.cluster ? l.blocks() : (unsigned)std::min<long long>(kWideParts, up(rows, 64));
}

inline bool lies(const void *p, long long stride, size_t size) {  // rows on 16-byte boundaries
    return (reinterpret_cast<uintptr_t>(p) | (size_t)stride * size) % 16 == 0;
}

template <typename T, typename W>
int forward_typed(NormArgs &a, cudaStream_t s) {
    const Layout l = layout_of(a.rows, a.cols, std::max(1, sm_count()));
    if (!l.cluster) return tula::launch(k_norm_forward_wide<T, W>, dim3(l.grid), l.threads, 0, s, 1, a);
    a.group = l.group;
    a.cluster = l.cluster;
    const bool vec = a.cols % (16 / (int)sizeof(T)) == 0 && lies(a.x, a.stride, sizeof(T)) && lies(a.y, a.cols, sizeof(T));
    void (*k)(const NormArgs) = vec ? k_norm_forward<T, W, true> : k_norm_forward<T, W, false>;
    return tula::launch(k, dim3(l.grid), l.threads, 0, s, l.cluster, a);
}
template <typename T, typename W>
int backward_typed(NormArgs &a, void *dw, void *db, cudaStream_t s) {
    const Layout l = layout_of(a.rows, a.cols, std::max(1, sm_count()));
    int rc = TULA_OK;
    if (l.cluster) {
        a.group = l.group;
        a.cluster = l.cluster;
        const bool vec = a.cols % (16 / (int)sizeof(T)) == 0 && lies(a.x, a.stride, sizeof(T)) && lies(a.dy, a.dy_stride, sizeof(T)) &&
                         (!a.y || lies(a.y, a.cols, sizeof(T)));
        void (*k)(const NormArgs) = a.parts ? (vec ? k_norm_backward<T, W, true, true> : k_norm_backward<T, W, false, true>)
                                            : (vec ? k_norm_backward<T, W, true, false> : k_norm_backward<T, W, false, false>);
        const int smem = a.parts && l.threads > l.group ? 2 * l.threads * kN * 4 : 0;  // 16 KB
        rc = tula::launch(k, dim3(l.grid), l.threads, smem, s, l.cluster, a);
    } else {
        if (a.y) rc = tula::launch(k_norm_backward_wide<T, W>, dim3(l.grid), l.threads, 0, s, 1, a);
        if (!rc && a.parts)
            rc = tula::launch(k_norm_sums_wide<T>, dim3((unsigned)up(a.cols, 256), parts_of(l, a.rows)), 256, 0, s, 1, a);
    }
    if (rc || !a.parts) return rc;
    return tula::launch(k_norm_params<W>, dim3((unsigned)up(2ll * a.cols, 32)), 256, 0, s, 1, (const float *)a.parts,
                        (int)parts_of(l, a.rows), a.cols, static_cast<W *>(dw), static_cast<W *>(db));
}

constexpr long long kMostCols = 1LL << 24;

template <typename F>
int by_types(int type, int param_type, F f) {
    auto second = [&](auto t) {
        if (param_type == TULA_TYPE_F32) return f(t, float());
        if (param_type == TULA_TYPE_BF16) return f(t, __nv_bfloat16());
        return f(t, __half());
    };
    if (type == TULA_TYPE_F32) return second(float());
    if (type == TULA_TYPE_BF16) return second(__nv_bfloat16());
    return second(__half());
}

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
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return by_types(type, param_type, [&](auto t, auto w) { return forward_typed<decltype(t), decltype(w)>(a, s); });
}

int tula_layer_norm_workspace_size(int64_t rows, int64_t cols, size_t *bytes) {
    if (!bytes || !good_sizes(rows, cols)) return TULA_ERR_ARG;
    // as many parts as a GPU of up to 256 SMs has CTAs (of 256 threads, four an SM)
    const long long parts = std::min<long long>(std::max<long long>(rows, 1), 4 * 256);
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
    return by_types(type, param_type, [&](auto t, auto w) { return backward_typed<decltype(t), decltype(w)>(a, dweight, dbias, s); });
}

}  // extern "C"
