// Matrices of fp32, bf16 and fp16 elements as the kernels that quantise them and read them back move them.
#pragma once

#include "tula_tc.cuh"

namespace {

// Word of two elements of a 16-bit type as two floats.
template <typename T>
__device__ __forceinline__ float2 pair_of(unsigned u) {
    if (std::is_same<T, __half>::value) {
        __half2 h;
        memcpy(&h, &u, 4);
        return __half22float2(h);
    }
    return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u));
}

// (A kernel may start while the one before it still writes x: nothing of x is read before the wait,
// which makes it visible, and nothing by the read-only path, which takes it for constant.)
//
// A part's elements as they are, zero beyond `left` of them.  Aligned: they start at a 32-byte
// boundary.  Else the 16-byte granules that hold them are loaded, an end one also by its neighbour, and
// shifted; inner: all of them lie within the matrix ([begin, end)) and the part within the row, else
// granules that reach out of it are loaded element by element.
template <typename T>
__device__ __forceinline__ uint4 load_granule(unsigned long long at, unsigned long long begin, unsigned long long end) {
    if (at >= begin && at + 16 <= end) return *reinterpret_cast<const uint4 *>(at);
    unsigned w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const unsigned long long p = at + 4 * k;
        w[k] = 0;
        if (sizeof(T) == 4) {
            if (p >= begin && p < end) w[k] = *reinterpret_cast<const unsigned *>(p);
        } else {
            if (p >= begin && p < end) w[k] = *reinterpret_cast<const unsigned short *>(p);
            if (p + 2 >= begin && p + 2 < end) w[k] |= (unsigned)*reinterpret_cast<const unsigned short *>(p + 2) << 16;
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
template <typename T, int kElems, bool Aligned>
__device__ __forceinline__ void load_part(unsigned (&w)[kElems * sizeof(T) / 4], const T *p, bool inner, long long left,
                                          unsigned long long begin, unsigned long long end) {
    constexpr int kWords = kElems * (int)sizeof(T) / 4;
    if (!inner && left <= 0) {
#pragma unroll
        for (int k = 0; k < kWords; ++k) w[k] = 0;
        return;
    }
    if (Aligned && (inner || left >= kElems)) {
#pragma unroll
        for (int k = 0; k < kWords; k += 8)
            asm volatile("ld.global.cs.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                         : "=r"(w[k]), "=r"(w[k + 1]), "=r"(w[k + 2]), "=r"(w[k + 3]), "=r"(w[k + 4]), "=r"(w[k + 5]),
                           "=r"(w[k + 6]), "=r"(w[k + 7])
                         : "l"(reinterpret_cast<const unsigned *>(p) + k));
        return;
    }
    const unsigned long long at = reinterpret_cast<unsigned long long>(p);
    const int off = (int)(at & 15);
    unsigned v[kWords + 4];
#pragma unroll
    for (int k = 0; k <= kWords / 4; ++k) {
        uint4 q = make_uint4(0, 0, 0, 0);
        if (inner)
            q = reinterpret_cast<const uint4 *>(at - off)[k];
        else if (k < kWords / 4 || off)
            q = load_granule<T>(at - off + 16 * k, begin, end);
        v[4 * k] = q.x, v[4 * k + 1] = q.y, v[4 * k + 2] = q.z, v[4 * k + 3] = q.w;
    }
#pragma unroll
    for (int k = 0; k < kWords + 2; ++k) v[k] = off & 8 ? v[k + 2] : v[k];
#pragma unroll
    for (int k = 0; k < kWords + 1; ++k) v[k] = off & 4 ? v[k + 1] : v[k];
#pragma unroll
    for (int k = 0; k < kWords; ++k) {
        w[k] = sizeof(T) == 2 && off & 2 ? __funnelshift_r(v[k], v[k + 1], 16) : v[k];
        if (inner) continue;
        if (sizeof(T) == 4)
            w[k] = k < left ? w[k] : 0u;
        else
            w[k] = 2 * k + 1 < left ? w[k] : 2 * k < left ? w[k] & 0xffffu : 0u;
    }
}

template <typename T>
__device__ __forceinline__ void floats8(float (&x)[8], const unsigned *w) {
    if (sizeof(T) == 4) {
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = __uint_as_float(w[k]);
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float2 f = pair_of<T>(w[k]);
            x[2 * k] = f.x;
            x[2 * k + 1] = f.y;
        }
    }
}

// The largest magnitude of 16-bit elements, from their own bits to fp32's.
template <typename T>
__device__ __forceinline__ unsigned top_bits(unsigned half) {
    return std::is_same<T, __half>::value ? __float_as_uint(__half2float(__ushort_as_half((unsigned short)half))) : half << 16;
}
// The larger magnitudes of a word and those so far, the signs of no meaning, a NaN kept; 16-bit
// elements by halves.  One instruction, where integer ones take a mask and a maximum.
template <typename T>
__device__ __forceinline__ unsigned larger(unsigned top, unsigned w) {
    unsigned r;
    if (sizeof(T) == 4)
        asm("max.NaN.xorsign.abs.f32 %0, %1, %2;" : "=r"(r) : "r"(top), "r"(w));
    else if (std::is_same<T, __half>::value)
        asm("max.NaN.xorsign.abs.f16x2 %0, %1, %2;" : "=r"(r) : "r"(top), "r"(w));
    else
        asm("max.NaN.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(top), "r"(w));
    return r;
}

__device__ __forceinline__ float scale_value(unsigned s) {
    return s == 255u ? __uint_as_float(0x7fffffffu) : __uint_as_float(s ? s << 23 : 0x00400000u);
}

// Eight elements to a boundary of as many bytes.
template <typename T>
__device__ __forceinline__ void store_run(T *to, const T (&y)[8]) {
    const unsigned *q = reinterpret_cast<const unsigned *>(y);
    constexpr int kHalf = sizeof(T) == 4 ? 4 : 0;  // words of four elements
    if (sizeof(T) == 2)
        __stcs(reinterpret_cast<uint4 *>(to), make_uint4(q[0], q[1], q[2], q[3]));
    else
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(q[0]), "r"(q[1]), "r"(q[2]),
                     "r"(q[3]), "r"(q[kHalf]), "r"(q[kHalf + 1]), "r"(q[kHalf + 2]), "r"(q[kHalf + 3])
                     : "memory");
}

// x / d with magic = ceil(2^64 / d): for a 32-bit x the quotient is exact; for others where
// x d < 2^64, and the host has left magic 0 where that does not hold.
__device__ __forceinline__ unsigned divide(unsigned x, unsigned long long magic, long long) {
    const unsigned long long lo = (unsigned long long)x * (unsigned)magic;
    return (unsigned)(((unsigned long long)x * (unsigned)(magic >> 32) + (lo >> 32)) >> 32);
}
__device__ __forceinline__ long long divide(long long x, unsigned long long magic, long long d) {
    return magic ? (long long)__umul64hi((unsigned long long)x, magic) : x / d;
}

// ----------------------------------------------------------------------------
// Reading back
// ----------------------------------------------------------------------------
//
// F, a format: eight codes, where they and a block's scale lie, their values.
struct DequantArgs {
    const unsigned char *codes, *scales;
    long long n, cols;  // elements, columns
    int tiles_c, lead;  // lead: elements from the boundary below out to out
    unsigned long long magic;  // ceil(2^64 / cols) (Easy: / (cols / 8)), or 0: see divide
};

// Out is one run of elements: a thread writes the eight between two boundaries of as many bytes,
// whatever rows they belong to, and takes their codes from where they lie.  Easy: rows start at
// multiples of eight.  Four such groups a thread for 16-bit types then, elsewhere one (measured
// at 8192 x 4096).  I: an unsigned where all indexes fit.
template <typename T, bool Easy>
constexpr int kGroupsOf = Easy && sizeof(T) == 2 ? 4 : 1;
template <class F, typename T, bool Easy, typename I>
__global__ void __launch_bounds__(256) k_dequantize(const DequantArgs a, T *out) {
    constexpr int kGroups = kGroupsOf<T, Easy>;
    let_next_start();
    wait_for_previous();
    I f[kGroups], r[kGroups], c[kGroups];
    typename F::Eight q[kGroups];
    unsigned s0[kGroups], s1[kGroups];
    bool whole[kGroups];  // eight elements of one row
    const I n = (I)a.n, cols = (I)a.cols;
#pragma unroll
    for (int j = 0; j < kGroups; ++j) {
        const I g = (I)blockIdx.x * (256 * kGroups) + 256 * j + threadIdx.x;
        if (Easy) {
            f[j] = 8 * g;
            r[j] = divide(g, a.magic, a.cols / 8);
            c[j] = f[j] - r[j] * cols;
            whole[j] = f[j] < n;
        } else {
            f[j] = 8 * g - (I)a.lead;  // (the first group: below 0, or beyond n for unsigned ones)
            const I at = g == 0 ? 0 : f[j];
            r[j] = divide(at, a.magic, a.cols);
            c[j] = at - r[j] * cols;
            whole[j] = (g > 0 || a.lead == 0) && f[j] < n && n - f[j] >= 8 && cols - c[j] >= 8;
        }
        if (!whole[j]) continue;
        q[j] = F::template fetch<Easy>(a.codes + (size_t)r[j] * F::pitch(a.tiles_c), c[j]);
        s1[j] = s0[j] = F::scale_at(a, r[j], c[j]);
        if (!Easy) s1[j] = F::template scale_at<I>(a, r[j], c[j] + 7);
    }
#pragma unroll
    for (int j = 0; j < kGroups; ++j) {
        if (whole[j]) {
            __align__(32) T y[8];
            F::values(y, q[j], s0[j], s1[j], Easy ? 8 : F::kBlock - (int)(c[j] & (F::kBlock - 1)));
            store_run(out + f[j], y);
        } else if (!Easy) {
            I row = r[j], col = c[j];
            const I g = (I)blockIdx.x * (256 * kGroups) + 256 * j + threadIdx.x;
            const int skip = g == 0 ? a.lead : 0;  // elements before out
            if (g > 0 && f[j] >= n) continue;
            const I left = g == 0 ? n : n - f[j];
            const int here = left < (I)(8 - skip) ? (int)left : 8 - skip;
            T *to = g == 0 ? out : out + f[j];
            for (int k = 0; k < here; ++k) {
                const float v = F::one(a.codes + (size_t)row * F::pitch(a.tiles_c), col);
                put(to + k, __fmul_rn(v, scale_value(F::scale_at(a, row, col))));
                if (++col == cols) ++row, col = 0;
            }
        }
    }
}

template <class F, typename T>
int dequantize_typed(const void *codes, const void *scales, long long rows, long long cols, void *out, cudaStream_t s) {
    DequantArgs a;
    a.codes = static_cast<const unsigned char *>(codes);
    a.scales = static_cast<const unsigned char *>(scales);
    a.n = rows * cols;
    a.cols = cols;
    a.tiles_c = (int)up(cols, kTile);
    a.lead = (int)(reinterpret_cast<uintptr_t>(out) % (8 * sizeof(T)) / sizeof(T));
    const bool easy = cols % 8 == 0 && a.lead == 0;
    const long long blocks = up(a.n + a.lead, 8 * 256 * (easy ? kGroupsOf<T, true> : kGroupsOf<T, false>));
    if (blocks >= (1LL << 31)) return TULA_ERR_ARG;
    // 32-bit indexes where the last group's, beyond n, still fits
    const bool small = (easy ? blocks * 256 * kGroupsOf<T, true> * 8 : a.n + 8 * 256 * 2) < (1LL << 32);
    const unsigned long long d = (unsigned long long)(easy ? cols / 8 : cols);
    a.magic = d > 1 && (small || (unsigned long long)a.n < ~0ull / d) ? ~0ull / d + 1 : 0;
    void (*k)(const DequantArgs, T *) = easy ? (small && d > 1 ? k_dequantize<F, T, true, unsigned> : k_dequantize<F, T, true, long long>)
                                             : (small && d > 1 ? k_dequantize<F, T, false, unsigned> : k_dequantize<F, T, false, long long>);
    return tula::launch(k, dim3((unsigned)blocks), 256, 0, s, 1, a, static_cast<T *>(out));
}
template <class F>
int dequantize(const void *codes, const void *scales, long long rows, long long cols, void *out, int type, cudaStream_t s) {
    const long long tiles = tiles_of(rows, cols);
    if (!good_type(type) || tiles < 0) return TULA_ERR_ARG;
    if (tiles == 0) return TULA_OK;
    if (!codes || !scales || !out || !aligned(codes, 16) || !aligned(scales, 16) || !aligned(out, type_size(type)))
        return TULA_ERR_ARG;
    if (type == TULA_TYPE_F32) return dequantize_typed<F, float>(codes, scales, rows, cols, out, s);
    if (type == TULA_TYPE_BF16) return dequantize_typed<F, __nv_bfloat16>(codes, scales, rows, cols, out, s);
    return dequantize_typed<F, __half>(codes, scales, rows, cols, out, s);
}

}  // namespace
