// Microscaled 4-bit matrices (MXFP4) for sm_103a: quantisation, reading back, products.
#include "tula_common.h"
#include "tula_train.h"

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <atomic>
#include <cstring>
#include <type_traits>

namespace {

constexpr unsigned kFull = 0xffffffffu;
constexpr int kTile = 128;          // rows and columns of a scale tile
constexpr int kScaleTile = 512;     // its bytes: 128 rows by 4 blocks of 32 columns
constexpr int kBlock = 32;          // elements that share a scale

__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void let_next_start() {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// ----------------------------------------------------------------------------
// Barriers and copies
// ----------------------------------------------------------------------------

constexpr uint32_t kSpinLimit = 1u << 19;  // bound on every wait (~2 s)
static __device__ unsigned g_mx_error;

__device__ __forceinline__ uint32_t smem_addr(const void *p) {
    return (uint32_t)__cvta_generic_to_shared(p);
}
__device__ __forceinline__ void mbar_init(uint32_t bar, unsigned count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_expect(uint32_t bar, unsigned bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool mbar_try(uint32_t bar, unsigned parity) {
    unsigned ok;
    asm volatile("{\n.reg .pred p;\n"
                 "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n"
                 "selp.u32 %0, 1, 0, p;\n}\n"
                 : "=r"(ok)
                 : "r"(bar), "r"(parity)
                 : "memory");
    return ok != 0;
}
// False if the wait ran out, here or before in another warp (`dead`).
__device__ __forceinline__ bool mbar_wait(uint32_t bar, unsigned parity, volatile int *dead) {
    for (uint32_t i = 0; i < kSpinLimit; ++i) {
        if (mbar_try(bar, parity)) return true;
        if (*dead) return false;
    }
    *dead = 1;
    atomicOr(&g_mx_error, 1u);
    return false;
}

__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap *map, int x, int y, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
                 "l"(map), "r"(x), "r"(y), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, unsigned bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
                 "l"(src), "r"(bytes), "r"(bar)
                 : "memory");
}

// ----------------------------------------------------------------------------
// Elements
// ----------------------------------------------------------------------------

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

// The block's scale byte from the bits of its largest magnitude (as fp32; infinities and NaN have
// larger bits than any number).
__device__ __forceinline__ unsigned scale_byte(unsigned top) {
    const unsigned e = top >> 23;
    return e == 255u ? 255u : e > 2u ? e - 2u : 0u;
}
// What its elements are multiplied by: 2^(127 - s), exact; 0 for a block that is NaN, whose codes
// are 0.
__device__ __forceinline__ float inverse_scale(unsigned s) {
    return s == 255u ? 0.f : __uint_as_float((254u - s) << 23);
}

// Eight elements' codes, the first in the lowest bits.  A magnitude of 6 or more gives 6.
__device__ __forceinline__ unsigned codes8(const float (&x)[8]) {
    unsigned r;
    asm("{\n"
        ".reg .b8 b0, b1, b2, b3;\n"
        "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n"
        "cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n"
        "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n"
        "cvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n"
        "mov.b32 %0, {b0, b1, b2, b3};\n"
        "}\n"
        : "=r"(r)
        : "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7]));
    return r;
}

// ----------------------------------------------------------------------------
// Quantisation
// ----------------------------------------------------------------------------
//
// One CTA per 128 x 128 tile of x, which is one scale tile of x and one of its transpose.  Along the
// rows a thread takes a block whole (16-bit types), so that what there is to do once a block is done
// once: with four threads to a block the kernel issued in two thirds of all cycles, and 8192 x 8192
// bf16 took 43 us in both forms instead of 39.  Four threads share a block of fp32, whose 128 bytes a
// lane would spread each load over 32 lines (39 us for 8192 x 4096, 32 so).  The transpose reads the
// tile again from shared memory, a thread per 32 rows of one column (fp32) or of two.  HBM bounds it:
// 2 or 4 bytes in and 17/32 out per element and form, against four to seven operations.
template <typename T>
struct Part {
    static constexpr int kElems = sizeof(T) == 4 ? 8 : 32;  // of a row, that a thread takes at a time
    static constexpr int kLanes = kBlock / kElems;          // to a block
    static constexpr int kWords = kElems * (int)sizeof(T) / 4;
    static constexpr int kSubs = 4 * kLanes;                // to a tile's row
};

struct QuantArgs {
    const void *x;
    long long rows, cols, stride;
    unsigned char *codes, *scales, *codes_t, *scales_t;
    int tiles_c;  // tiles along the columns
    int tiles_r;
};

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
template <typename T, bool Aligned>
__device__ __forceinline__ void load_part(unsigned (&w)[Part<T>::kWords], const T *p, bool inner, long long left,
                                          unsigned long long begin, unsigned long long end) {
    constexpr int kWords = Part<T>::kWords;
    if (!inner && left <= 0) {
#pragma unroll
        for (int k = 0; k < kWords; ++k) w[k] = 0;
        return;
    }
    if (Aligned && (inner || left >= Part<T>::kElems)) {
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
__device__ __forceinline__ unsigned mul_bf16x2(unsigned a, unsigned b) {
    unsigned r;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// inverse_scale as bf16 bits.
__device__ __forceinline__ unsigned inverse_scale_bf16(unsigned s) { return s == 255u ? 0u : (254u - s) << 7; }

// A part's codes; returns its block's scale byte.
template <typename T>
__device__ __forceinline__ unsigned quantize_part(const unsigned (&w)[Part<T>::kWords], unsigned (&q)[Part<T>::kElems / 8]) {
    constexpr int kWords = Part<T>::kWords, kEight = kWords / (Part<T>::kElems / 8);
    constexpr bool kBf16 = std::is_same<T, __nv_bfloat16>::value;
    unsigned tops[4] = {0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < kWords; ++j) tops[j & 3] = larger<T>(tops[j & 3], w[j]);
    unsigned top = larger<T>(larger<T>(tops[0], tops[1]), larger<T>(tops[2], tops[3]));
    top &= sizeof(T) == 4 ? 0x7fffffffu : 0x7fff7fffu;
    if (sizeof(T) == 2) top = top_bits<T>(max(top & 0xffffu, top >> 16));
#pragma unroll
    for (int o = 1; o < Part<T>::kLanes; o *= 2) top = max(top, __shfl_xor_sync(kFull, top, o));
    const unsigned s = scale_byte(top);
    const float f = inverse_scale(s);
    // exact in bf16 too (what falls below its range is far below the smallest code)
    const unsigned f2 = inverse_scale_bf16(s) * 0x10001u;
#pragma unroll
    for (int k = 0; k < Part<T>::kElems / 8; ++k) {
        unsigned v[kEight];
#pragma unroll
        for (int j = 0; j < kEight; ++j) v[j] = kBf16 ? mul_bf16x2(w[k * kEight + j], f2) : w[k * kEight + j];
        float x[8];
        floats8<T>(x, v);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (!kBf16) x[j] = __fmul_rn(x[j], f);
        q[k] = s == 255u ? 0u : codes8(x);
    }
    return s;
}
// Its codes and, by the block's first lane, its scale byte to where they go: part `sub` of a tile's row.
template <typename T>
__device__ __forceinline__ void put_part(const unsigned (&w)[Part<T>::kWords], int row, int sub, bool there, unsigned char *codes,
                                         unsigned char *scales) {
    unsigned q[Part<T>::kElems / 8];
    const unsigned s = quantize_part<T>(w, q);
    if (sub % Part<T>::kLanes == 0) scales[(row & 31) * 16 + (row >> 5) * 4 + sub / Part<T>::kLanes] = (unsigned char)s;
    if (!there) return;
    if constexpr (Part<T>::kElems == 32)
        *reinterpret_cast<uint4 *>(codes + 16 * sub) = make_uint4(q[0], q[1], q[2], q[3]);
    else
        *reinterpret_cast<unsigned *>(codes + 4 * sub) = q[0];
}

// The tile in shared memory: rows of 128 elements in 16-byte chunks, whose places within 128 bytes are
// exchanged so that neither the stores of parts nor the column reads (a word a lane, all of one row)
// meet in a bank.
template <typename T>
__device__ __forceinline__ int chunk_place(int row, int chunk) {
    return sizeof(T) == 4 ? chunk ^ (chunk >> 3 & 3) ^ (row & 1) << 2 : chunk ^ (chunk >> 3) ^ (row & 1) << 1;
}

// 32 rows (block rb) of word c of a tile in shared memory, that is of one column (fp32) or two:
// codes to out, `pitch` bytes a column, scale bytes to scales.
template <typename T, bool Swizzled>
__device__ __forceinline__ void quantize_cols(const unsigned *tile, int c, int rb, unsigned char *out, int pitch,
                                              unsigned char *scales) {
    unsigned w[32], top = 0;
    const int at[2] = {4 * chunk_place<T>(0, c >> 2) + (c & 3), 4 * chunk_place<T>(1, c >> 2) + (c & 3)};
#pragma unroll
    for (int k = 0; k < 32; ++k) {
        w[k] = tile[(32 * rb + k) * (kTile * (int)sizeof(T) / 4) + (Swizzled ? at[k & 1] : c)];
        top = larger<T>(top, w[k]);
    }
    constexpr bool kBf16 = std::is_same<T, __nv_bfloat16>::value;
    constexpr int kCols = 4 / (int)sizeof(T);
    top &= sizeof(T) == 4 ? 0x7fffffffu : 0x7fff7fffu;
    unsigned s[kCols];
#pragma unroll
    for (int h = 0; h < kCols; ++h)
        s[h] = scale_byte(sizeof(T) == 4 ? top : top_bits<T>(h ? top >> 16 : top & 0xffffu));
    if (kBf16) {
        const unsigned f = inverse_scale_bf16(s[0]) | inverse_scale_bf16(s[kCols - 1]) << 16;
#pragma unroll
        for (int k = 0; k < 32; ++k) w[k] = mul_bf16x2(w[k], f);
    }
#pragma unroll
    for (int h = 0; h < kCols; ++h) {
        const int col = kCols * c + h;
        const float f = inverse_scale(s[h]);
        unsigned q[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float v;
                if (sizeof(T) == 4) {
                    v = __uint_as_float(w[8 * k + j]);
                } else {
                    const float2 p = pair_of<T>(w[8 * k + j]);
                    v = h ? p.y : p.x;
                }
                x[j] = kBf16 ? v : __fmul_rn(v, f);
            }
            q[k] = s[h] == 255u ? 0u : codes8(x);
        }
        *reinterpret_cast<uint4 *>(out + col * pitch + 16 * rb) = make_uint4(q[0], q[1], q[2], q[3]);
        scales[(col & 31) * 16 + (col >> 5) * 4 + rb] = (unsigned char)s[h];
    }
}

constexpr int kOutPitch = 80;  // bytes of a column's 64 of codes, and 16 to spread the banks

// fp32: twice the threads, so that a column block is one thread's in either type's tile.
template <typename T>
struct QuantShape {
    static constexpr int kThreads = sizeof(T) == 4 ? 512 : 256;
    static constexpr int kCtas = sizeof(T) == 4 ? 2 : 4;  // an SM, that registers are left for
    static constexpr int kSmem = kTile * kTile * (int)sizeof(T) + kTile * kOutPitch;
};

template <typename T, bool Aligned, bool Rows, bool Cols>
__global__ void __launch_bounds__(QuantShape<T>::kThreads, QuantShape<T>::kCtas) k_quantize(const QuantArgs a) {
    constexpr int kThreads = QuantShape<T>::kThreads;
    constexpr int kWords = Part<T>::kWords, kSubs = Part<T>::kSubs;
    constexpr int kPitch = kTile * sizeof(T) / 4;       // words of a tile's row
    constexpr int kLoads = kTile * kSubs / kThreads;    // parts a thread
    extern __shared__ __align__(16) unsigned tile[];  // Cols
    __shared__ __align__(16) unsigned char scale_bytes[2][kScaleTile];
    let_next_start();
    wait_for_previous();
    const int tid = threadIdx.x;
    const int tr = blockIdx.x / a.tiles_c, tc = blockIdx.x % a.tiles_c;
    const long long r0 = (long long)tr * kTile, c0 = (long long)tc * kTile;
    const int sub = tid % kSubs;
    const size_t pitch = (size_t)a.tiles_c * (kTile / 2), pitch_t = (size_t)a.tiles_r * (kTile / 2);
    const unsigned long long begin = reinterpret_cast<unsigned long long>(a.x);
    const unsigned long long end = begin + ((unsigned long long)(a.rows - 1) * a.stride + a.cols) * sizeof(T);
    unsigned w[kLoads][kWords];
    const T *p0 = static_cast<const T *>(a.x) + (r0 + tid / kSubs) * a.stride + c0 + Part<T>::kElems * sub;
    const bool inner = c0 + kTile <= a.cols && (Aligned ? r0 + kTile <= a.rows : tr > 0 && r0 + kTile < a.rows);
    if (inner) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            load_part<T, Aligned>(w[i], p0 + i * (kThreads / kSubs) * a.stride, true, Part<T>::kElems, begin, end);
    } else {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const long long r = r0 + i * (kThreads / kSubs) + tid / kSubs;
            load_part<T, Aligned>(w[i], p0 + i * (kThreads / kSubs) * a.stride, false,
                                  r < a.rows ? a.cols - c0 - Part<T>::kElems * sub : 0, begin, end);
        }
    }
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const int row = i * (kThreads / kSubs) + tid / kSubs;
        if (Cols) {
#pragma unroll
            for (int k = 0; k < kWords / 4; ++k)
                *reinterpret_cast<uint4 *>(&tile[row * kPitch + 4 * chunk_place<T>(row, sub * (kWords / 4) + k)]) =
                    make_uint4(w[i][4 * k], w[i][4 * k + 1], w[i][4 * k + 2], w[i][4 * k + 3]);
        }
        if (Rows)
            put_part<T>(w[i], row, sub, inner || r0 + row < a.rows, a.codes + (size_t)(r0 + row) * pitch + c0 / 2, scale_bytes[0]);
    }
    __syncthreads();
    if (Rows && tid < 32)
        *reinterpret_cast<uint4 *>(a.scales + ((size_t)tr * a.tiles_c + tc) * kScaleTile + 16 * tid) =
            *reinterpret_cast<const uint4 *>(&scale_bytes[0][16 * tid]);
    if (!Cols) return;
    unsigned char *out = reinterpret_cast<unsigned char *>(tile + kTile * kPitch);
    constexpr int kSide = kPitch;  // words of a row
    quantize_cols<T, true>(tile, tid % kSide, tid / kSide, out, kOutPitch, scale_bytes[1]);
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 4 * kTile / kThreads; ++k) {
        const int c = (k * kThreads + tid) >> 2, part = tid & 3;
        if (c0 + c < a.cols)
            *reinterpret_cast<uint4 *>(a.codes_t + (size_t)(c0 + c) * pitch_t + r0 / 2 + 16 * part) =
                *reinterpret_cast<const uint4 *>(out + c * kOutPitch + 16 * part);
    }
    if (tid < 32)
        *reinterpret_cast<uint4 *>(a.scales_t + ((size_t)tc * a.tiles_r + tr) * kScaleTile + 16 * tid) =
            *reinterpret_cast<const uint4 *>(&scale_bytes[1][16 * tid]);
}

// The same with whole tiles brought by TMA (rows at 16-byte boundaries), persistent: while a tile
// is quantised the next ones are on their way, so that HBM does not wait for arithmetic.  For the
// transpose of any type, and for both forms of fp32 (Rows).
template <typename T>
struct QuantRing {
    static constexpr int kThreads = sizeof(T) == 4 ? 512 : 256;
    static constexpr int kCtas = sizeof(T) == 4 ? 1 : 2;  // an SM
    static constexpr int kStages = 3;
    static constexpr int kTileBytes = kTile * kTile * (int)sizeof(T);
    static constexpr int kOut = kOutPitch;
    static constexpr int kSmem = kStages * kTileBytes + kTile * kOut + 2 * kScaleTile + 128;
    static_assert(kCtas * (kSmem + 1024) <= 228 * 1024, "shared memory");
};

template <typename T, bool Rows>
__global__ void __launch_bounds__(QuantRing<T>::kThreads, QuantRing<T>::kCtas)
    k_quantize_tiles(const __grid_constant__ CUtensorMap map, const QuantArgs a) {
    using R = QuantRing<T>;
    constexpr int kPitch = kTile * sizeof(T) / 4;  // words of a tile's row
    extern __shared__ __align__(16) unsigned tile[];
    __shared__ __align__(8) unsigned long long bars[R::kStages];
    __shared__ volatile int dead;
    const int tid = threadIdx.x;
    unsigned char *base = reinterpret_cast<unsigned char *>(tile) + (-smem_addr(tile) & 127u);
    unsigned char *out = base + R::kStages * R::kTileBytes;
    unsigned char *scale_c = out + kTile * R::kOut, *scale_r = scale_c + kScaleTile;
    const uint32_t full = smem_addr(bars);
    const int n_tiles = a.tiles_r * a.tiles_c;
    if (tid == 0) {
        for (int s = 0; s < R::kStages; ++s) mbar_init(full + 8 * s, 1);
        dead = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    let_next_start();
    wait_for_previous();
    auto fetch = [&](int t, int s) {
        mbar_expect(full + 8 * s, R::kTileBytes);
        tma_load_2d(smem_addr(base) + s * R::kTileBytes, &map, t % a.tiles_c * kTile, t / a.tiles_c * kTile, full + 8 * s);
    };
    int fetched = 0;  // thread 0
    if (tid == 0)
        for (; fetched < R::kStages && blockIdx.x + fetched * gridDim.x < n_tiles; ++fetched)
            fetch(blockIdx.x + fetched * gridDim.x, fetched);
    const size_t pitch_t = (size_t)a.tiles_r * (kTile / 2);
    int i = 0;
    for (int t = blockIdx.x; t < n_tiles; t += gridDim.x, ++i) {
        const int s = i % R::kStages;
        const bool ok = mbar_wait(full + 8 * s, (i / R::kStages) & 1, &dead);
        if (!__syncthreads_and(ok)) break;  // and the last tile's codes have been read
        const unsigned *x_tile = reinterpret_cast<const unsigned *>(base + s * R::kTileBytes);
        const int tr = t / a.tiles_c, tc = t % a.tiles_c;
        const long long r0 = (long long)tr * kTile, c0 = (long long)tc * kTile;
        if (Rows) {
            constexpr int kSubs = Part<T>::kSubs, kWords = Part<T>::kWords;
            const int sub = tid % kSubs;
#pragma unroll
            for (int k = 0; k < kTile * kSubs / R::kThreads; ++k) {
                const int row = k * (R::kThreads / kSubs) + tid / kSubs;
                unsigned w[kWords];
#pragma unroll
                for (int j = 0; j < kWords / 4; ++j) {
                    const uint4 q = *reinterpret_cast<const uint4 *>(&x_tile[row * kPitch + sub * kWords + 4 * j]);
                    w[4 * j] = q.x, w[4 * j + 1] = q.y, w[4 * j + 2] = q.z, w[4 * j + 3] = q.w;
                }
                put_part<T>(w, row, sub, r0 + row < a.rows, a.codes + (size_t)(r0 + row) * a.tiles_c * (kTile / 2) + c0 / 2, scale_r);
            }
        }
        quantize_cols<T, false>(x_tile, tid % kPitch, tid / kPitch, out, R::kOut, scale_c);
        __syncthreads();  // the tile has been read, its codes and scales are there
        if (tid == 0 && blockIdx.x + fetched * gridDim.x < n_tiles) {
            fetch(blockIdx.x + fetched * gridDim.x, s);
            ++fetched;
        }
#pragma unroll
        for (int k = 0; k < 4 * kTile / R::kThreads; ++k) {
            const int c = (k * R::kThreads + tid) >> 2, part = tid & 3;
            if (c0 + c < a.cols)
                *reinterpret_cast<uint4 *>(a.codes_t + (size_t)(c0 + c) * pitch_t + r0 / 2 + 16 * part) =
                    *reinterpret_cast<const uint4 *>(out + c * R::kOut + 16 * part);
        }
        if (tid < 32)
            *reinterpret_cast<uint4 *>(a.scales_t + ((size_t)tc * a.tiles_r + tr) * kScaleTile + 16 * tid) =
                *reinterpret_cast<const uint4 *>(scale_c + 16 * tid);
        if (Rows && tid >= 32 && tid < 64)
            *reinterpret_cast<uint4 *>(a.scales + ((size_t)tr * a.tiles_c + tc) * kScaleTile + 16 * (tid - 32)) =
                *reinterpret_cast<const uint4 *>(scale_r + 16 * (tid - 32));
    }
    // no copy may be in flight when the CTA ends
    if (tid == 0)
        for (; i < fetched; ++i)
            for (uint32_t w = 0; w < kSpinLimit && !mbar_try(full + 8 * (i % R::kStages), (i / R::kStages) & 1); ++w) {}
}

// ----------------------------------------------------------------------------
// Reading back
// ----------------------------------------------------------------------------

__device__ __forceinline__ float scale_value(unsigned s) {
    return s == 255u ? __uint_as_float(0x7fffffffu) : __uint_as_float(s ? s << 23 : 0x00400000u);
}
// Two codes' values.
__device__ __forceinline__ float2 code_pair(unsigned byte) {
    unsigned h;
    asm("{\n.reg .b8 b, u1, u2, u3;\nmov.b32 {b, u1, u2, u3}, %1;\ncvt.rn.f16x2.e2m1x2 %0, b;\n}\n" : "=r"(h) : "r"(byte));
    __half2 v;
    memcpy(&v, &h, 4);
    return __half22float2(v);
}

__device__ __forceinline__ void put(float *p, float v) { *p = v; }
__device__ __forceinline__ void put(__nv_bfloat16 *p, float v) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ void put(__half *p, float v) { *p = __float2half_rn(v); }

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

struct DequantArgs {
    const unsigned char *codes, *scales;
    long long n, cols;  // elements, columns
    int tiles_c, lead;  // lead: elements from the boundary below out to out
    unsigned long long magic;  // ceil(2^64 / cols) (Easy: / (cols / 8)), or 0: see divide
};
// x / d with magic = ceil(2^64 / d): for a 32-bit x the quotient is exact; for others where
// x d < 2^64, and the host has left magic 0 where that does not hold.
__device__ __forceinline__ unsigned divide(unsigned x, unsigned long long magic, long long) {
    const unsigned long long lo = (unsigned long long)x * (unsigned)magic;
    return (unsigned)(((unsigned long long)x * (unsigned)(magic >> 32) + (lo >> 32)) >> 32);
}
__device__ __forceinline__ long long divide(long long x, unsigned long long magic, long long d) {
    return magic ? (long long)__umul64hi((unsigned long long)x, magic) : x / d;
}
template <typename I>
__device__ __forceinline__ unsigned scale_at(const DequantArgs &a, I r, I c) {
    return __ldcg(a.scales + ((size_t)(r / kTile) * a.tiles_c + c / kTile) * kScaleTile + (r & 31) * 16 + (r & 127) / 32 * 4 +
                  (c & 127) / kBlock);
}

// The values of eight codes as pairs of bf16, but for the scale.  A value's two bytes are looked up by
// byte permutations whose selectors are four codes' magnitudes at a time; then the signs are put in.
// (By conversions to fp16 and fp32 the kernel issued in 83 % of all cycles and HBM waited for it.)
__device__ __forceinline__ void code_values(unsigned (&v)[4], unsigned q) {
    const unsigned m = q & 0x77777777u, up = q << 4;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        // 0, 0.5, 1, 1.5 and 2, 3, 4, 6: high bytes 00 3f 3f 3f and 40 each, low ones 00 00 80 c0 and 00 40 80 c0
        const unsigned hi = __byte_perm(0x3f3f3f00u, 0x40404040u, m >> (16 * k));
        const unsigned lo = __byte_perm(0xc0800000u, 0xc0804000u, m >> (16 * k));
        v[2 * k] = __byte_perm(lo, hi, 0x5140);
        v[2 * k + 1] = __byte_perm(lo, hi, 0x7362);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] |= __byte_perm(up, q, (4 + k) << 12 | k << 4) & 0x80008000u;
}
// Eight elements from their codes, the first `first` with scale s0, the others with s1.
template <typename T>
__device__ __forceinline__ void scaled_values(T (&y)[8], unsigned q, unsigned s0, unsigned s1, int first) {
    unsigned v[4];
    code_values(v, q);
    if (std::is_same<T, __nv_bfloat16>::value) {
        auto bf16_scale = [](unsigned s) { return s == 255u ? 0x7fffu : s ? s << 7 : 0x0040u; };
        const unsigned b0 = bf16_scale(s0), b1 = bf16_scale(s1);
        unsigned *out = reinterpret_cast<unsigned *>(y);
#pragma unroll
        for (int k = 0; k < 4; ++k)
            out[k * (int)sizeof(T) / 2] = mul_bf16x2(v[k], (2 * k < first ? b0 : b1) | (2 * k + 1 < first ? b0 : b1) << 16);
    } else {
        const float f0 = scale_value(s0), f1 = scale_value(s1);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            put(&y[2 * k], __fmul_rn(__uint_as_float(v[k] << 16), 2 * k < first ? f0 : f1));
            put(&y[2 * k + 1], __fmul_rn(__uint_as_float(v[k] & 0xffff0000u), 2 * k + 1 < first ? f0 : f1));
        }
    }
}

// Out is one run of elements: a thread writes the eight between two boundaries of as many bytes,
// whatever rows they belong to, and takes their codes from where they lie.  Easy: rows start at
// multiples of eight.  Four such groups a thread for 16-bit types then, elsewhere one (measured
// at 8192 x 4096).  I: an unsigned where all indexes fit.
template <typename T, bool Easy>
constexpr int kGroupsOf = Easy && sizeof(T) == 2 ? 4 : 1;
template <typename T, bool Easy, typename I>
__global__ void __launch_bounds__(256) k_dequantize(const DequantArgs a, T *out) {
    constexpr int kGroups = kGroupsOf<T, Easy>;
    let_next_start();
    wait_for_previous();
    I f[kGroups], r[kGroups], c[kGroups];
    unsigned q[kGroups], s0[kGroups], s1[kGroups];
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
        const unsigned *w = reinterpret_cast<const unsigned *>(a.codes + (size_t)r[j] * a.tiles_c * (kTile / 2)) + c[j] / 8;
        q[j] = __ldcg(w);
        s1[j] = s0[j] = scale_at(a, r[j], c[j]);
        if (!Easy) {
            const int in = (int)(c[j] & 7);
            if (in) q[j] = __funnelshift_r(q[j], __ldcg(w + 1), 4 * in);
            s1[j] = scale_at<I>(a, r[j], c[j] + 7);
        }
    }
#pragma unroll
    for (int j = 0; j < kGroups; ++j) {
        if (whole[j]) {
            __align__(32) T y[8];
            scaled_values(y, q[j], s0[j], s1[j], Easy ? 8 : 32 - (int)(c[j] & 31));
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
                const unsigned byte = __ldcg(a.codes + (size_t)row * a.tiles_c * (kTile / 2) + col / 2);
                put(to + k, __fmul_rn(code_pair(col & 1 ? byte >> 4 : byte & 15u).x, scale_value(scale_at(a, row, col))));
                if (++col == cols) ++row, col = 0;
            }
        }
    }
}

// ----------------------------------------------------------------------------
// Products: tcgen05 with block scales
// ----------------------------------------------------------------------------
//
// out = A B^T by tiles of 128 rows of one operand (P, the instruction's M) by NT rows of the other
// (Q, its N).  Codes come by TMA, 256 columns (128 bytes a row) a stage, scales by bulk copies;
// one thread moves a stage's scales to tensor memory and issues its instructions (64 columns each,
// two scales a row); accumulators lie in tensor memory and four warps read them back.

constexpr int kStageK = 256;
constexpr int kMmaThreads = 192;  // a copying warp, an issuing warp, four that read back

// Shared-memory matrix descriptors: addresses in units of 16 bytes; bit 46: their version.
// Codes: rows of 128 bytes with the 128-byte swizzle, groups of eight rows 1024 bytes apart.
__device__ __forceinline__ uint64_t codes_desc(uint32_t addr) {
    return (uint64_t)((addr & 0x3ffff) >> 4) | (uint64_t)1 << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 |
           (uint64_t)2 << 61;
}
// A scale tile: 32 rows of 16 bytes, no swizzle, groups of eight rows 128 bytes apart.
__device__ __forceinline__ uint64_t scales_desc(uint32_t addr) {
    return (uint64_t)((addr & 0x3ffff) >> 4) | (uint64_t)(128 >> 4) << 32 | (uint64_t)1 << 46;
}
// The instruction's descriptor: E2M1 operands, E8M0 scales, M = 128, N.
__host__ __device__ constexpr uint32_t mma_desc(int n) {
    return 1u << 7 | 1u << 10 | (uint32_t)(n >> 3) << 17 | 1u << 23 | (128u >> 7) << 27;
}
// Which two of a word's four scales the instruction takes: id 0 or 2, of both operands.
__device__ __forceinline__ uint32_t with_scale_id(uint32_t desc, uint32_t id) {
    return desc | id << 4 | id << 29;
}

// True in one lane of a converged warp.  The tensor core's and the copies' instructions take their
// operands from uniform registers: issued from warps that run whole, with one lane elected for the
// instruction alone, they cost a few cycles each; from a branch of lane 0 a stage's ten took some
// 900 cycles, and a product of 8192^3 300 us.
__device__ __forceinline__ bool elect_one() {
    unsigned p;
    asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}\n" : "=r"(p));
    return p != 0;
}

__device__ __forceinline__ void copy_scales(uint32_t tmem, uint64_t desc) {
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, bool add) {
    asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %6, 0;\n"
                 "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n}\n" ::"r"(d),
                 "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"((unsigned)add)
                 : "memory");
}
__device__ __forceinline__ void commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tmem_alloc(uint32_t where, unsigned cols) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(where), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
__device__ __forceinline__ void tmem_free(uint32_t tmem, unsigned cols) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(cols));
}
// 16 columns of this warp's 32 lanes.
__device__ __forceinline__ void tmem_load16(float (&v)[16], uint32_t tmem) {
    unsigned r[16];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 "
                 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
                   "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(tmem));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int k = 0; k < 16; ++k) v[k] = __uint_as_float(r[k]);
}

// 32 columns, not waited for; tmem_wait makes the registers good.
__device__ __forceinline__ void tmem_load32(unsigned *r, uint32_t tmem) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 "
                 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
                   "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
                   "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
                   "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(tmem));
}
template <int N>
__device__ __forceinline__ void tmem_wait(unsigned (&r)[N]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int k = 0; k < N; ++k) asm volatile("" : "+r"(r[k]));  // no use of them moves up
}

struct MatmulArgs {
    const unsigned char *p_scales, *q_scales;
    void *out;
    long long P, Q;       // rows of each operand
    long long ld;         // elements of out from row to row
    int tiles_k;          // of 128 columns
    int grid_q;           // tiles of the product along Q
    int split;            // CTAs of a cluster that share a tile's columns
};

__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t in_cta(uint32_t addr, unsigned rank) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ float load_cluster(uint32_t addr) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr));  // (no fence for the others)
    return v;
}
__device__ __forceinline__ float4 load_cluster4(uint32_t addr) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                 : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
                 : "r"(addr)
                 : "memory");
    return v;
}

template <int NT, bool Swap>
struct MmaShape {
    static constexpr int kP = 128 * 128, kQ = NT * 128;                     // bytes of codes a stage
    static constexpr int kSP = 2 * kScaleTile, kSQ = 2 * kScaleTile;
    static constexpr int kStage = kP + kQ + kSP + kSQ;
    static constexpr int kStages = NT >= 128 ? 3 : NT >= 64 ? 4 : 5;        // two CTAs an SM
    // partial sums: lines along out's rows, four floats apart to spread the banks
    static constexpr int kLines = Swap ? NT : 128, kLine = Swap ? 128 : NT, kPitch = kLine + 4;
    static constexpr int kSmem = kStages * kStage + 1024;                   // aligned to 1024 at run time
    static constexpr int kScaleP = NT;                                      // tensor memory columns
    static constexpr int kScaleQ = kScaleP + 8;
    static constexpr int kUsed = kScaleQ + 8;
    static constexpr int kCols = kUsed <= 64 ? 64 : kUsed <= 128 ? 128 : 256;
    static_assert(kLines * kPitch * 4 <= kStages * kStage && 2 * kSmem <= 226 * 1024, "shared memory");
};

// One tile of 128 rows of P by NT of Q a cluster; its CTAs share the columns, and add up their
// partial sums through distributed shared memory in the order of their ranks.  Swap: out is
// [Q][P], its rows run along P.
template <int NT, bool Swap, typename T>
__global__ void __launch_bounds__(kMmaThreads) k_matmul(const __grid_constant__ CUtensorMap map_p,
                                                        const __grid_constant__ CUtensorMap map_q, const MatmulArgs a) {
    using S = MmaShape<NT, Swap>;
    extern __shared__ __align__(16) unsigned tile[];
    __shared__ __align__(8) unsigned long long bars[2 * S::kStages + 1];
    __shared__ uint32_t tmem_at;
    __shared__ volatile int dead;
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(kFull, tid >> 5, 0);
    const uint32_t stages = (smem_addr(tile) + 1023) & ~1023u;
    const uint32_t full = smem_addr(bars), empty = full + 8 * S::kStages, done = empty + 8 * S::kStages;
    const int rank = blockIdx.x % a.split, t = blockIdx.x / a.split;
    const int tp = t / a.grid_q, tq = t % a.grid_q;
    const int all_k = (a.tiles_k + 1) / 2, per = (all_k + a.split - 1) / a.split;
    const int k_begin = min(rank * per, all_k), n_k = min(per, all_k - k_begin);  // stages of this CTA
    // A thread of those that read back has a row of P: out's rows along Q are stored from there if
    // they lie at 16-byte boundaries, and else, as partial sums are, by way of shared memory.
    const bool shared = a.split > 1 || (!Swap && (((a.ld * sizeof(T)) | reinterpret_cast<uintptr_t>(a.out)) & 15));
    if (tid == 0) {
        for (int s = 0; s < S::kStages; ++s) {
            mbar_init(full + 8 * s, 1);
            mbar_init(empty + 8 * s, 1);
        }
        mbar_init(done, 1);
        dead = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) tmem_alloc(smem_addr(&tmem_at), S::kCols);
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = __shfl_sync(kFull, tmem_at, 0);
    let_next_start();
    wait_for_previous();

    if (warp == 0) {
        int issued = 0;
        bool ok = true;
        for (int i = 0; i < n_k; ++i) {
            const int s = i % S::kStages, k = k_begin + i;
            if (i >= S::kStages) ok = __all_sync(kFull, mbar_wait(empty + 8 * s, (i / S::kStages - 1) & 1, &dead));
            if (!ok) break;
            const uint32_t at = stages + s * S::kStage, bar = full + 8 * s;
            const int tiles = min(2, a.tiles_k - 2 * k);  // scale tiles along the columns
            if (elect_one()) {
                mbar_expect(bar, S::kP + S::kQ + 2 * tiles * kScaleTile);
                tma_load_2d(at, &map_p, k * (kStageK / 2), tp * 128, bar);
                tma_load_2d(at + S::kP, &map_q, k * (kStageK / 2), tq * NT, bar);
                bulk_load(at + S::kP + S::kQ, a.p_scales + ((size_t)tp * a.tiles_k + 2 * k) * kScaleTile, tiles * kScaleTile, bar);
                // the scale tile that these rows of Q are in
                bulk_load(at + S::kP + S::kQ + S::kSP, a.q_scales + ((size_t)tq * a.tiles_k + 2 * k) * kScaleTile,
                          tiles * kScaleTile, bar);
            }
            __syncwarp();
            issued = i + 1;
        }
        // The issuing warp's arrivals have all landed before the CTA ends, also those on stages that nothing
        // is copied to any more.
        for (int i = max(0, issued - S::kStages); ok && i < issued; ++i)
            ok = __all_sync(kFull, mbar_wait(empty + 8 * (i % S::kStages), (i / S::kStages) & 1, &dead));
        // Nor may a copy be in flight then.
        if (dead)
            for (int i = max(0, issued - S::kStages); i < issued; ++i) {
                const int s = i % S::kStages;
                for (uint32_t w = 0; w < kSpinLimit && !mbar_try(full + 8 * s, (i / S::kStages) & 1); ++w) {}
            }
        __syncwarp();
    } else if (warp == 1) {
        bool ok = true;
        for (int i = 0; i < n_k; ++i) {
            const int s = i % S::kStages;
            ok = __all_sync(kFull, mbar_wait(full + 8 * s, (i / S::kStages) & 1, &dead));
            if (!ok) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t at = stages + s * S::kStage, sc = at + S::kP + S::kQ;
            const int tiles = min(2, a.tiles_k - 2 * (k_begin + i));
            const uint64_t da = codes_desc(at), db = codes_desc(at + S::kP);
            if (elect_one()) {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    if (j == tiles) break;
                    copy_scales(tmem + S::kScaleP + 4 * j, scales_desc(sc + j * kScaleTile));
                    copy_scales(tmem + S::kScaleQ + 4 * j, scales_desc(sc + S::kSP + j * kScaleTile));
                }
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    if (j == tiles) break;
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        mma(tmem, da + 2 * (2 * j + h), db + 2 * (2 * j + h), with_scale_id(mma_desc(NT), 2 * h),
                            tmem + S::kScaleP + 4 * j, tmem + S::kScaleQ + 4 * j, i > 0 || j > 0 || h > 0);
                }
                commit(empty + 8 * s);
            }
            __syncwarp();
        }
        if (ok && n_k && elect_one()) commit(done);  // (without stages nothing waits for it)
        __syncwarp();
    } else {
        const bool ok = __all_sync(kFull, n_k == 0 || mbar_wait(done, 0, &dead));
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const int quad = warp & 3;  // the quarter of tensor memory's lanes that this warp may read
        const int row = quad * 32 + lane;
        const long long p = (long long)tp * 128 + row;
        T *out = static_cast<T *>(a.out);
        for (int c = 0; ok && c < NT; c += 16) {
            const long long q0 = (long long)tq * NT + c;
            if (q0 >= a.Q) break;
            float v[16];
            __syncwarp();
            if (n_k) {
                tmem_load16(v, tmem + ((unsigned)(quad * 32) << 16) + c);
            } else {
#pragma unroll
                for (int k = 0; k < 16; ++k) v[k] = 0.f;
            }
            if (shared) {
                // the stages' place: every copy has landed and every instruction has read it
                if (Swap) {
#pragma unroll
                    for (int k = 0; k < 16; ++k)
                        asm volatile("st.shared.f32 [%0], %1;" ::"r"(stages + 4 * ((c + k) * S::kPitch + row)), "f"(v[k]) : "memory");
                } else {
#pragma unroll
                    for (int k = 0; k < 16; k += 4)
                        asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(stages + 4 * (row * S::kPitch + c + k)),
                                     "f"(v[k]), "f"(v[k + 1]), "f"(v[k + 2]), "f"(v[k + 3])
                                     : "memory");
                }
            } else if (p < a.P) {
                if (!Swap && q0 + 16 <= a.Q) {
                    __align__(16) T y[16];
#pragma unroll
                    for (int k = 0; k < 16; ++k) put(&y[k], v[k]);
#pragma unroll
                    for (int k = 0; k < (int)sizeof(T); ++k)
                        reinterpret_cast<uint4 *>(out + p * a.ld + q0)[k] = reinterpret_cast<const uint4 *>(y)[k];
                } else {
#pragma unroll
                    for (int k = 0; k < 16; ++k)
                        if (q0 + k < a.Q) put(out + (Swap ? (q0 + k) * a.ld + p : p * a.ld + q0 + k), v[k]);
                }
            }
        }
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    }
    __syncthreads();
    if (warp == 1) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        tmem_free(tmem, S::kCols);
    }
    if (!shared) return;
    if (a.split > 1) cluster_sync();
    // This CTA's share of the tile's lines, four elements a thread where they lie at a boundary of four,
    // else a warp to a line.
    T *out = static_cast<T *>(a.out);
    const int q_here = (int)min((long long)NT, a.Q - (long long)tq * NT);
    const int p_here = (int)min(128ll, a.P - (long long)tp * 128);
    const int lines = Swap ? q_here : p_here, line = Swap ? p_here : q_here;
    const int share = (lines + a.split - 1) / a.split, first = rank * share;
    const long long line0 = Swap ? (long long)tq * NT : (long long)tp * 128, col0 = Swap ? (long long)tp * 128 : (long long)tq * NT;
    const bool vec = a.ld % 4 == 0 && (reinterpret_cast<uintptr_t>(a.out) & (4 * sizeof(T) - 1)) == 0;
    const int n_lines = min(share, lines - first);
    if (!vec) {
        constexpr int kPer = S::kLine / 32;
        for (int o = first + warp; o < first + n_lines; o += kMmaThreads / 32) {
            float sum[kPer];
#pragma unroll
            for (int k = 0; k < kPer; ++k) sum[k] = 0.f;
#pragma unroll
            for (int r = 0; r < 8; ++r) {
                if (r >= a.split) break;
                const uint32_t at = in_cta(stages + 4 * (o * S::kPitch + lane), r);
#pragma unroll
                for (int k = 0; k < kPer; ++k) {
                    const float v = load_cluster(at + 128 * k);
                    sum[k] = r ? __fadd_rn(sum[k], v) : v;
                }
            }
#pragma unroll
            for (int k = 0; k < kPer; ++k)
                if (lane + 32 * k < line) put(out + (line0 + o) * a.ld + col0 + lane + 32 * k, sum[k]);
        }
    }
    constexpr int kQuads = S::kLine / 4;
    for (int i = tid; vec && i < n_lines * kQuads; i += kMmaThreads) {
        const int o = first + i / kQuads, n = i % kQuads * 4;
        if (n >= line) continue;
        const uint32_t at = stages + 4 * (o * S::kPitch + n);
        float4 part[8];
#pragma unroll
        for (int r = 0; r < 8; ++r)
            if (r < a.split) part[r] = load_cluster4(in_cta(at, r));
        float4 sum = part[0];
#pragma unroll
        for (int r = 1; r < 8; ++r)
            if (r < a.split)
                sum = make_float4(__fadd_rn(sum.x, part[r].x), __fadd_rn(sum.y, part[r].y), __fadd_rn(sum.z, part[r].z),
                                  __fadd_rn(sum.w, part[r].w));
        T *to = out + (line0 + o) * a.ld + col0 + n;
        __align__(16) T y[4];
        put(&y[0], sum.x), put(&y[1], sum.y), put(&y[2], sum.z), put(&y[3], sum.w);
        if (vec && n + 4 <= line) {
            if (sizeof(T) == 4)
                *reinterpret_cast<uint4 *>(to) = *reinterpret_cast<const uint4 *>(y);
            else
                *reinterpret_cast<uint2 *>(to) = *reinterpret_cast<const uint2 *>(y);
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (n + k < line) to[k] = y[k];
        }
    }
    if (a.split > 1) cluster_sync();  // the others have read this CTA's sums
}

// ----------------------------------------------------------------------------
// Large products: pairs of CTAs
// ----------------------------------------------------------------------------
//
// Two CTAs of a cluster compute a tile of 256 rows of A by 256 of B with one instruction stream
// (cta_group::2): each holds its 128 rows of A, 128 of the 256 rows of B, and its 128 rows of
// accumulators.  A stage of 256 columns is 35.8 KB a CTA for 2 x 128 x 256 x 256 operations, twice
// the operations a byte of 128 x 128 tiles; an SM takes in 64 bytes a clock, which bounds 8192^3 at
// 135 us (150 measured a few at a time, 160 over seconds; the tensor pipe active 78 % of it).  Products
// with short sums are bound by writing (16384 x 16384 x 512: 143 to 147 us, fill_ of as much 136).
// Persistent: a pair takes every n-th tile.  Tensor memory has 512 columns: two accumulators of 256 that
// overlap in 32, and the scales' 24.  Four warps read an accumulator back, the columns that the other
// one needs first, while the next tile's instructions run.

constexpr int kPairThreads = 192;
struct Pair {
    static constexpr int kStages = 6;
    static constexpr int kA = 128 * 128, kB = 128 * 128;
    static constexpr int kSA = 2 * kScaleTile, kSB = 4 * kScaleTile;  // the scales of all 256 rows of B
    static constexpr int kStage = kA + kB + kSA + kSB;
    static constexpr int kOut = 4 * 4096;  // a buffer a warp, 32 rows of 128 bytes
    static constexpr int kBars = 2 * kStages + 2;
    static constexpr int kSmem = kStages * kStage + kOut + 8 * kBars + 16;
    static constexpr int kAcc1 = 224, kScaleA = 480, kScaleB = 488;  // tensor memory columns
    static_assert(kStage % 1024 == 0 && kSmem <= 227 * 1024, "shared memory");
};

struct PairArgs {
    void *out;
    long long M, N;
    int tiles_k;
    int tiles_m, tiles_n;  // of 256
    int word;              // bytes that divide out's address and rows: 16 (stored by TMA), 8, 4 or 2
};

__device__ __forceinline__ void tma_load_pair(uint32_t dst, const CUtensorMap *map, int x, int y, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], "
                 "[%4];" ::"r"(dst),
                 "l"(map), "r"(x), "r"(y), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ void copy_scales_pair(uint32_t tmem, uint64_t desc) {
    asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}
__device__ __forceinline__ void mma_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, bool add) {
    asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %6, 0;\n"
                 "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n}\n" ::"r"(d),
                 "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"((unsigned)add)
                 : "memory");
}
// Arrives on the barrier of both CTAs once every instruction before has completed.
__device__ __forceinline__ void commit_pair(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
                 "h"((unsigned short)3)
                 : "memory");
}
__device__ __forceinline__ void arrive_cluster(uint32_t bar) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__host__ __device__ constexpr uint32_t pair_desc() {
    return 1u << 7 | 1u << 10 | (uint32_t)(256 >> 3) << 17 | 1u << 23 | (256u >> 7) << 27;
}

// Tiles in the order in which the pairs take them: columns of `kBand` tiles of A, so that those in
// work at a time share rows of both operands in L2.
constexpr int kBand = 8;
__device__ __forceinline__ void tile_at(int t, const PairArgs &a, int &tm, int &tn) {
    const int band = t / (kBand * a.tiles_n), in = t - band * kBand * a.tiles_n;
    const int rows = min(kBand, a.tiles_m - band * kBand);
    tm = band * kBand + in % rows;
    tn = in / rows;
}

// 32 rows of 128 bytes from a warp's buffer to out, W bytes a lane; `here` bytes of each row, `rows` of
// them.  Eight rows are read before any is stored.  (16-bit elements in pairs from odd places took twice
// the time: lanes at the ends part ways.)
template <int W>
__device__ __forceinline__ void store_rows(const unsigned char *buffer, unsigned char *to, long long pitch, int here, int rows) {
    using Word = std::conditional_t<W == 8, uint2, std::conditional_t<W == 4, unsigned, unsigned short>>;
    constexpr int kLanes = W == 8 ? 16 : 32;           // to a row
    constexpr int kPer = 128 / (kLanes * W);           // words a lane takes of it
    constexpr int kAtOnce = 32 / kLanes, kStep = 8 / kAtOnce;
    const int lane = threadIdx.x & 31, byte = lane % kLanes * W;
    for (int r0 = 0; r0 < 32; r0 += 8) {
        Word u[kStep][kPer];
#pragma unroll
        for (int j = 0; j < kStep; ++j)
#pragma unroll
            for (int k = 0; k < kPer; ++k) {
                const int r = r0 + j * kAtOnce + (kAtOnce > 1 ? lane / kLanes : 0);
                u[j][k] = *reinterpret_cast<const Word *>(buffer + r * 128 + ((byte + 32 * W * k) ^ ((r & 7) << 4)));
            }
#pragma unroll
        for (int j = 0; j < kStep; ++j) {
            const int r = r0 + j * kAtOnce + (kAtOnce > 1 ? lane / kLanes : 0);
            unsigned char *p = to + r * pitch + byte;
#pragma unroll
            for (int k = 0; k < kPer; ++k)
                if (byte + 32 * W * k < here && r < rows) *reinterpret_cast<Word *>(p + 32 * W * k) = u[j][k];
        }
    }
}

template <typename T>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kPairThreads, 1)
    k_matmul_pair(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                  const __grid_constant__ CUtensorMap map_sa, const __grid_constant__ CUtensorMap map_sb,
                  const __grid_constant__ CUtensorMap map_out, const PairArgs a) {
    // All of the 227 KB but some: nothing in static shared memory, so that the stages start at a
    // multiple of 1024 bytes without room to move them there (checked below).
    extern __shared__ __align__(1024) unsigned char all[];
    unsigned long long *bars = reinterpret_cast<unsigned long long *>(all + Pair::kStages * Pair::kStage + Pair::kOut);
    uint32_t *tmem_at = reinterpret_cast<uint32_t *>(bars + Pair::kBars);
    volatile int &dead = *reinterpret_cast<volatile int *>(tmem_at + 1);
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(kFull, tid >> 5, 0);
    const unsigned rank = blockIdx.x & 1;
    const int pairs = gridDim.x / 2, pair = blockIdx.x / 2, n_tiles = a.tiles_m * a.tiles_n;
    const uint32_t stages = smem_addr(all);
    const uint32_t outs = stages + Pair::kStages * Pair::kStage;
    const uint32_t full = smem_addr(bars), empty = full + 8 * Pair::kStages;
    const uint32_t acc_full = empty + 8 * Pair::kStages, acc_free = acc_full + 8;
    const int n_k = (a.tiles_k + 1) / 2;
    if (stages & 1023u) {  // no kernel that this may happen to has been seen
        if (tid == 0) atomicOr(&g_mx_error, 2u);
        return;
    }
    if (tid == 0) {
        for (int s = 0; s < Pair::kStages; ++s) {
            mbar_init(full + 8 * s, 1);
            mbar_init(empty + 8 * s, 1);
        }
        mbar_init(acc_full, 1);
        mbar_init(acc_free, 8);  // four warps of each CTA
        dead = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(tmem_at)), "r"(512)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    cluster_sync();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = 0;  // all 512 columns were asked for
    let_next_start();
    wait_for_previous();

    if (warp == 0) {
        int i = 0;  // stages filled
        bool ok = true;
        for (int t = pair; ok && t < n_tiles; t += pairs) {
            int tm, tn;
            tile_at(t, a, tm, tn);
            for (int k = 0; k < n_k; ++k, ++i) {
                const int s = i % Pair::kStages;
                if (i >= Pair::kStages) ok = __all_sync(kFull, mbar_wait(empty + 8 * s, (i / Pair::kStages - 1) & 1, &dead));
                if (!ok) break;
                const uint32_t at = stages + s * Pair::kStage, bar = in_cta(full + 8 * s, 0);
                if (elect_one()) {
                    if (rank == 0) mbar_expect(full + 8 * s, 2 * Pair::kStage);  // both CTAs' copies
                    tma_load_pair(at, &map_a, k * (kStageK / 2), tm * 256 + rank * 128, bar);
                    tma_load_pair(at + Pair::kA, &map_b, k * (kStageK / 2), tn * 256 + rank * 128, bar);
                    tma_load_pair(at + Pair::kA + Pair::kB, &map_sa, k * 256, tm * 2 + rank, bar);
                    tma_load_pair(at + Pair::kA + Pair::kB + Pair::kSA, &map_sb, k * 256, tn * 2, bar);
                }
                __syncwarp();
            }
        }
        // The other CTA's arrivals on this one's barriers have all landed before it ends.
        for (int j = max(0, i - Pair::kStages); ok && j < i; ++j)
            ok = __all_sync(kFull, mbar_wait(empty + 8 * (j % Pair::kStages), (j / Pair::kStages) & 1, &dead));
        // No copy may be in flight when the CTA ends.  On the way out of a wait that ran out
        // the copies' barrier may be the other CTA's: a millisecond is far more than they take.
        if (!ok)
            for (int w = 0; w < 1000; ++w) __nanosleep(1000);
        __syncwarp();
    } else if (warp == 1) {
        if (rank == 0) {
            int i = 0, n = 0;
            bool ok = true;
            for (int t = pair; ok && t < n_tiles; t += pairs, ++n) {
                if (n > 0) ok = __all_sync(kFull, mbar_wait(acc_free, (n - 1) & 1, &dead));
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t acc = tmem + (n & 1 ? Pair::kAcc1 : 0);
                for (int k = 0; ok && k < n_k; ++k, ++i) {
                    const int s = i % Pair::kStages;
                    ok = __all_sync(kFull, mbar_wait(full + 8 * s, (i / Pair::kStages) & 1, &dead));
                    if (!ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint32_t at = stages + s * Pair::kStage, sc = at + Pair::kA + Pair::kB;
                    const int tiles = min(2, a.tiles_k - 2 * k);
                    const uint64_t da = codes_desc(at), db = codes_desc(at + Pair::kA);
                    if (elect_one()) {
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            if (j == tiles) break;
                            copy_scales_pair(tmem + Pair::kScaleA + 4 * j, scales_desc(sc + j * kScaleTile));
#pragma unroll
                            for (int h = 0; h < 2; ++h)
                                copy_scales_pair(tmem + Pair::kScaleB + 8 * j + 4 * h,
                                                 scales_desc(sc + Pair::kSA + (2 * h + j) * kScaleTile));
                        }
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            if (j == tiles) break;
#pragma unroll
                            for (int h = 0; h < 2; ++h)
                                mma_pair(acc, da + 2 * (2 * j + h), db + 2 * (2 * j + h), with_scale_id(pair_desc(), 2 * h),
                                         tmem + Pair::kScaleA + 4 * j, tmem + Pair::kScaleB + 8 * j, k > 0 || j > 0 || h > 0);
                        }
                        commit_pair(empty + 8 * s);
                        if (k == n_k - 1) commit_pair(acc_full);
                    }
                    __syncwarp();
                }
            }
        }
        __syncwarp();
    } else {
        const int quad = warp & 3;
        constexpr int kChunk = 128 / (int)sizeof(T);  // columns of 128 bytes of out
        int n = 0;
        for (int t = pair; t < n_tiles; t += pairs, ++n) {
            int tm, tn;
            tile_at(t, a, tm, tn);
            if (!__all_sync(kFull, mbar_wait(acc_full, n & 1, &dead))) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t acc = tmem + (n & 1 ? Pair::kAcc1 : 0) + ((unsigned)(quad * 32) << 16);
            const long long row0 = (long long)tm * 256 + rank * 128 + quad * 32;
#pragma unroll 1
            for (int c = 0; c < 256 / kChunk; ++c) {
                // the columns that the two accumulators share come first
                const int chunk = n & 1 ? c : 256 / kChunk - 1 - c, col = chunk * kChunk;
                const uint32_t at = outs + quad * 4096;
                __align__(16) T y[kChunk];
                unsigned v[kChunk];
#pragma unroll
                for (int k = 0; k < kChunk; k += 32) tmem_load32(v + k, acc + col + k);
                tmem_wait(v);
                if (c == 0) {
                    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) arrive_cluster(in_cta(acc_free, 0));
                }
#pragma unroll
                for (int k = 0; k < kChunk; ++k) put(&y[k], __uint_as_float(v[k]));
                if (a.word == 16) {  // the last store has read the buffer
                    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
                    __syncwarp();
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const uint4 q = reinterpret_cast<const uint4 *>(y)[j];
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + lane * 128 + ((j ^ (lane & 7)) << 4)),
                                 "r"(q.x), "r"(q.y), "r"(q.z), "r"(q.w)
                                 : "memory");
                }
                const long long c0 = (long long)tn * 256 + col;
                if (a.word == 16) {
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) {
                        if (row0 < a.M && c0 < a.N)
                            asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];" ::"l"(&map_out),
                                         "r"((int)c0), "r"((int)row0), "r"(at)
                                         : "memory");
                        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                    }
                } else {
                    __syncwarp();
                    const int here = (int)max(0ll, min((long long)kChunk, a.N - c0)) * (int)sizeof(T);
                    const int rows = (int)max(0ll, min(32ll, a.M - row0));
                    const long long pitch = a.N * (long long)sizeof(T);
                    unsigned char *to = static_cast<unsigned char *>(a.out) + row0 * pitch + c0 * (long long)sizeof(T);
                    const unsigned char *buffer = all + (at - stages);
                    if (a.word == 8)
                        store_rows<8>(buffer, to, pitch, here, rows);
                    else if (a.word == 4)
                        store_rows<4>(buffer, to, pitch, here, rows);
                    else if (sizeof(T) == 2)
                        store_rows<2>(buffer, to, pitch, here, rows);
                    __syncwarp();
                }
            }
        }
        if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
        __syncwarp();
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    }
    __syncthreads();
    cluster_sync();
    if (warp == 1) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512));
    }
}

// Failure detection: a wait on a barrier that nothing arrives on.
__global__ void k_mx_wait_check() {
    __shared__ __align__(8) unsigned long long bar;
    __shared__ volatile int dead;
    wait_for_previous();
    if (threadIdx.x == 0) {
        mbar_init(smem_addr(&bar), 1);
        dead = 0;
    }
    __syncwarp();
    mbar_wait(smem_addr(&bar), 0, &dead);
}

// ----------------------------------------------------------------------------
// Host side
// ----------------------------------------------------------------------------

int cuda_failed(cudaError_t e) {
    tula::note_cuda_error((int)e);
    return TULA_ERR_CUDA;
}

inline long long up(long long n, long long m) { return (n + m - 1) / m; }
inline int type_size(int type) { return type == TULA_TYPE_F32 ? 4 : 2; }
inline bool good_type(int type) { return type >= TULA_TYPE_F32 && type <= TULA_TYPE_F16; }
inline bool aligned(const void *p, unsigned n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

constexpr long long kMostRows = (1LL << 31) - 1024;  // coordinates of tiles that reach beyond them fit an int

// Tiles of 128 x 128; -1 beyond what one grid and 32-bit coordinates hold.
long long tiles_of(long long rows, long long cols) {
    if (rows < 0 || cols < 0 || rows > kMostRows || cols > kMostRows) return -1;
    const long long t = up(rows, kTile) * up(cols, kTile);
    return t < (1LL << 31) ? t : -1;
}

// Lets a kernel have `smem` bytes of dynamic shared memory, once per kernel and device.
int allow_smem(const void *kernel, int smem, std::atomic<uint64_t> *done) {
    if (smem <= 48 * 1024) return TULA_OK;
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    const uint64_t bit = 1ull << (dev & 63);
    if (e == cudaSuccess && (dev > 63 || !(done->load(std::memory_order_acquire) & bit))) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e == cudaSuccess) done->fetch_or(bit, std::memory_order_release);
    }
    return e == cudaSuccess ? TULA_OK : cuda_failed(e);
}

typedef CUresult (*EncodeFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                             const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                             CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeFn encode_fn() {
    static EncodeFn fn = [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult q;
        const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q);
        return e == cudaSuccess && q == cudaDriverEntryPointSuccess ? reinterpret_cast<EncodeFn>(p) : nullptr;
    }();
    return fn;
}

// A matrix of `rows` rows of `cols` elements, `pitch` bytes apart, in boxes.
bool make_map(CUtensorMap *m, CUtensorMapDataType type, const void *base, long long rows, long long cols, long long pitch,
              int box_rows, int box_cols, CUtensorMapSwizzle swizzle) {
    const EncodeFn fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)pitch};
    const cuuint32_t box[2] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows}, steps[2] = {1, 1};
    auto encode = [&] {
        return fn(m, type, 2, const_cast<void *>(base), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
    };
    if (encode()) return true;
    // The driver's call wants a current context, which a thread whose first call this is (autograd's, for
    // a backward pass) has only once the runtime is told of its device.
    int dev = 0;
    return cudaGetDevice(&dev) == cudaSuccess && cudaSetDevice(dev) == cudaSuccess && encode();
}
// Codes in boxes of 128 bytes by box_rows rows.
bool codes_map(CUtensorMap *m, const void *codes, long long rows, int tiles_k, int box_rows) {
    const long long pitch = (long long)tiles_k * (kTile / 2);
    return make_map(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, codes, rows, pitch, pitch, box_rows, 128, CU_TENSOR_MAP_SWIZZLE_128B);
}
// Scales, a row per 128 of the matrix, in boxes of two tiles (256 words) by box_rows.
bool scales_map(CUtensorMap *m, const void *scales, long long rows, int tiles_k, int box_rows) {
    return make_map(m, CU_TENSOR_MAP_DATA_TYPE_UINT32, scales, up(rows, kTile), (long long)tiles_k * (kScaleTile / 4),
                    (long long)tiles_k * kScaleTile, box_rows, 256, CU_TENSOR_MAP_SWIZZLE_NONE);
}

// (cudaDeviceGetAttribute is a table lookup, some 30 ns)
int sm_count() {
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    return n;
}

template <typename T, bool Aligned>
int launch_quantize(const QuantArgs &a, unsigned grid, cudaStream_t s) {
    static std::atomic<uint64_t> done[3];
    const int which = a.codes && a.codes_t ? 0 : a.codes ? 1 : 2;
    void (*k)(const QuantArgs) = which == 0 ? k_quantize<T, Aligned, true, true> : k_quantize<T, Aligned, true, false>;
    if constexpr (!Aligned)  // (aligned rows' transpose alone goes by TMA)
        if (which == 2) k = k_quantize<T, Aligned, false, true>;
    const int smem = a.codes_t ? QuantShape<T>::kSmem : 0;
    const int rc = allow_smem((const void *)k, smem, &done[which]);
    if (rc) return rc;
    return tula::launch(k, dim3(grid), QuantShape<T>::kThreads, smem, s, 1, a);
}
template <typename T>
int launch_quantize_tiles(const QuantArgs &a, unsigned tiles, cudaStream_t s) {
    using R = QuantRing<T>;
    static std::atomic<uint64_t> done[2];
    void (*k)(const CUtensorMap, const QuantArgs) = k_quantize_tiles<T, false>;
    if constexpr (sizeof(T) == 4)  // (16-bit types come here for the transpose alone)
        if (a.codes) k = k_quantize_tiles<T, true>;
    const int rc = allow_smem((const void *)k, R::kSmem, &done[a.codes != nullptr]);
    if (rc) return rc;
    CUtensorMap map;
    const CUtensorMapDataType type = sizeof(T) == 4 ? CU_TENSOR_MAP_DATA_TYPE_UINT32 : CU_TENSOR_MAP_DATA_TYPE_UINT16;
    // (an only row's stride is any number)
    const long long row_bytes = (a.rows > 1 ? a.stride : up(a.cols, 8) * 8) * (long long)sizeof(T);
    if (!make_map(&map, type, a.x, a.rows, a.cols, row_bytes, kTile, kTile, CU_TENSOR_MAP_SWIZZLE_NONE))
        return cuda_failed(cudaErrorInvalidValue);
    const unsigned ctas = (unsigned)std::max(1, R::kCtas * sm_count());
    return tula::launch(k, dim3(std::min(tiles, ctas)), R::kThreads, R::kSmem, s, 1, map, a);
}

template <typename T>
int quantize_typed(const QuantArgs &a, unsigned grid, cudaStream_t s) {
    const size_t both = reinterpret_cast<uintptr_t>(a.x) | (a.rows > 1 ? (size_t)a.stride * sizeof(T) : 0);
    // Tiles by TMA for the transpose alone (us: 2048 x 1024 fp32 2.5, 3.6 without; 4096 x 4096 8.1 and 10.9;
    // 8192 x 4096 bf16 10.9 and 14.9), and for both forms of fp32 up to a tile an SM (2048 x 1024 3.3
    // and 4.5) and from eight on (8192 x 4096 29 and 32); between them what comes from L2 needs no
    // ring (4096 x 2048 8.6 and 8.0).  16-bit types' rows want the warps that the rings leave no room for:
    // 8192 x 4096 takes 22 us in both forms, 28 by TMA.
    const int sms = sm_count();
    const bool by_tma = a.codes_t && (!a.codes || (sizeof(T) == 4 && ((int)grid <= sms || (long long)grid >= 8ll * sms)));
    if (both % 16 == 0 && by_tma)
        return launch_quantize_tiles<T>(a, grid, s);
    return both % 32 == 0 ? launch_quantize<T, true>(a, grid, s) : launch_quantize<T, false>(a, grid, s);
}

template <typename T>
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
    void (*k)(const DequantArgs, T *) = easy ? (small && d > 1 ? k_dequantize<T, true, unsigned> : k_dequantize<T, true, long long>)
                                             : (small && d > 1 ? k_dequantize<T, false, unsigned> : k_dequantize<T, false, long long>);
    return tula::launch(k, dim3((unsigned)blocks), 256, 0, s, 1, a, static_cast<T *>(out));
}

template <int NT, bool Swap, typename T>
int launch_matmul(const CUtensorMap &mp, const CUtensorMap &mq, const MatmulArgs &a, unsigned grid, cudaStream_t s) {
    using S = MmaShape<NT, Swap>;
    static std::atomic<uint64_t> done;
    const int rc = allow_smem((const void *)k_matmul<NT, Swap, T>, S::kSmem, &done);
    if (rc) return rc;
    return tula::launch(k_matmul<NT, Swap, T>, dim3(grid), kMmaThreads, S::kSmem, s, a.split, mp, mq, a);
}

template <typename T>
int matmul_small(const void *a_codes, const void *a_scales, const void *b_codes, const void *b_scales, long long M, long long N,
                 long long K, void *out, cudaStream_t s) {
    // The operand with few rows is the instruction's N, so that its 128 rows are not padding; N as small as
    // they are (16 x 4096 x 4096: 4.4 us with 32, 6.1 with 128; 48 x 4096 x 25088: 9.3 with 64, 10.0).
    const bool swap = M <= 128;
    MatmulArgs a;
    a.p_scales = static_cast<const unsigned char *>(swap ? b_scales : a_scales);
    a.q_scales = static_cast<const unsigned char *>(swap ? a_scales : b_scales);
    a.P = swap ? N : M;
    a.Q = swap ? M : N;
    a.ld = N;
    a.out = out;
    a.tiles_k = (int)up(K, kTile);
    const int nt = a.Q <= 32 ? 32 : a.Q <= 64 ? 64 : 128;
    a.grid_q = (int)up(a.Q, nt);
    const long long tiles = up(a.P, 128) * a.grid_q;
    // Few tiles: up to eight CTAs share one's columns while all are resident (two an SM), two stages at
    // least for each, or four where the sums that they exchange are as long (128 x 4096 x 4096: 8.3
    // us with four CTAs, 9.2 with eight; 1 x 4096 x 4096: 4.0 us with eight).
    const int least = nt >= 64 ? 8 : 4;
    a.split = 1;
    while (a.split < 8 && tiles * a.split * 2 <= 2 * 152 && up(a.tiles_k, 2) >= least * a.split) a.split *= 2;
    if (tiles * a.split >= (1LL << 31)) return TULA_ERR_ARG;
    CUtensorMap mp, mq;
    std::memset(&mp, 0, sizeof(mp));
    std::memset(&mq, 0, sizeof(mq));
    if (K && (!codes_map(&mp, swap ? b_codes : a_codes, a.P, a.tiles_k, 128) ||
              !codes_map(&mq, swap ? a_codes : b_codes, a.Q, a.tiles_k, nt)))
        return cuda_failed(cudaErrorInvalidValue);
    const unsigned grid = (unsigned)(tiles * a.split);
    if (swap)
        return nt == 32 ? launch_matmul<32, true, T>(mp, mq, a, grid, s)
               : nt == 64 ? launch_matmul<64, true, T>(mp, mq, a, grid, s)
                          : launch_matmul<128, true, T>(mp, mq, a, grid, s);
    return nt == 32 ? launch_matmul<32, false, T>(mp, mq, a, grid, s)
           : nt == 64 ? launch_matmul<64, false, T>(mp, mq, a, grid, s)
                      : launch_matmul<128, false, T>(mp, mq, a, grid, s);
}

template <typename T>
int matmul_large(const void *a_codes, const void *a_scales, const void *b_codes, const void *b_scales, long long M, long long N,
                 long long K, void *out, cudaStream_t s) {
    PairArgs a;
    a.out = out;
    a.M = M;
    a.N = N;
    a.tiles_k = (int)up(K, kTile);
    a.tiles_m = (int)up(M, 256);
    a.tiles_n = (int)up(N, 256);
    const unsigned long long both = reinterpret_cast<unsigned long long>(out) | (unsigned long long)(N * (long long)sizeof(T));
    a.word = both % 16 == 0 ? 16 : both % 8 == 0 ? 8 : both % 4 == 0 ? 4 : 2;
    CUtensorMap ma, mb, sa, sb, mo;
    std::memset(&mo, 0, sizeof(mo));
    const CUtensorMapDataType type = sizeof(T) == 4 ? CU_TENSOR_MAP_DATA_TYPE_UINT32 : CU_TENSOR_MAP_DATA_TYPE_UINT16;
    if (!codes_map(&ma, a_codes, M, a.tiles_k, 128) || !codes_map(&mb, b_codes, N, a.tiles_k, 128) ||
        !scales_map(&sa, a_scales, M, a.tiles_k, 1) || !scales_map(&sb, b_scales, N, a.tiles_k, 2) ||
        (a.word == 16 && !make_map(&mo, type, out, M, N, N * (long long)sizeof(T), 32, 128 / (int)sizeof(T), CU_TENSOR_MAP_SWIZZLE_128B)))
        return cuda_failed(cudaErrorInvalidValue);
    static std::atomic<uint64_t> done;
    const int rc = allow_smem((const void *)k_matmul_pair<T>, Pair::kSmem, &done);
    if (rc) return rc;
    const long long tiles = (long long)a.tiles_m * a.tiles_n, pairs = std::max(1, sm_count() / 2);
    return tula::launch(k_matmul_pair<T>, dim3((unsigned)(2 * std::min(tiles, pairs))), kPairThreads, Pair::kSmem, s, 1, ma, mb, sa,
                        sb, mo, a);
}

template <typename T>
int matmul_typed(const void *a_codes, const void *a_scales, const void *b_codes, const void *b_scales, long long M, long long N,
                 long long K, void *out, cudaStream_t s) {
    // Pairs of CTAs from 32 tiles of 256 x 256 on: 1024 x 2048 x 4096 takes 9.5 us (10.3 by tiles of 128),
    // 2048 x 4096 x 512 8.5 (10.6); 1024 x 1024 x 4096, 16 tiles, 9.4 (9.1).
    if (K > 0 && M > 128 && N > 128 && up(M, 256) * up(N, 256) >= 32)
        return matmul_large<T>(a_codes, a_scales, b_codes, b_scales, M, N, K, out, s);
    return matmul_small<T>(a_codes, a_scales, b_codes, b_scales, M, N, K, out, s);
}

}  // namespace

extern "C" {

int tula_mx_size(int64_t rows, int64_t cols, size_t *code_bytes, size_t *scale_bytes) {
    if (!code_bytes || !scale_bytes || tiles_of(rows, cols) < 0) return TULA_ERR_ARG;
    *code_bytes = (size_t)rows * (size_t)up(cols, kTile) * (kTile / 2);
    *scale_bytes = (size_t)tiles_of(rows, cols) * kScaleTile;
    return TULA_OK;
}

int tula_mx_quantize(const void *x, int type, int64_t rows, int64_t cols, int64_t stride, void *codes, void *scales,
                     void *codes_t, void *scales_t, void *stream) {
    const long long tiles = tiles_of(rows, cols);
    if (!good_type(type) || tiles < 0 || stride < cols) return TULA_ERR_ARG;
    if (tiles == 0) return TULA_OK;
    if (!codes != !scales || !codes_t != !scales_t || (!codes && !codes_t)) return TULA_ERR_ARG;
    if (!x || !aligned(x, type_size(type)) || !aligned(codes, 16) || !aligned(scales, 16) || !aligned(codes_t, 16) ||
        !aligned(scales_t, 16))
        return TULA_ERR_ARG;
    QuantArgs a;
    a.x = x;
    a.rows = rows;
    a.cols = cols;
    a.stride = stride;
    a.codes = static_cast<unsigned char *>(codes);
    a.scales = static_cast<unsigned char *>(scales);
    a.codes_t = static_cast<unsigned char *>(codes_t);
    a.scales_t = static_cast<unsigned char *>(scales_t);
    a.tiles_c = (int)up(cols, kTile);
    a.tiles_r = (int)up(rows, kTile);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (type == TULA_TYPE_F32) return quantize_typed<float>(a, (unsigned)tiles, s);
    if (type == TULA_TYPE_BF16) return quantize_typed<__nv_bfloat16>(a, (unsigned)tiles, s);
    return quantize_typed<__half>(a, (unsigned)tiles, s);
}

int tula_mx_dequantize(const void *codes, const void *scales, int64_t rows, int64_t cols, void *out, int type, void *stream) {
    const long long tiles = tiles_of(rows, cols);
    if (!good_type(type) || tiles < 0) return TULA_ERR_ARG;
    if (tiles == 0) return TULA_OK;
    if (!codes || !scales || !out || !aligned(codes, 16) || !aligned(scales, 16) || !aligned(out, type_size(type)))
        return TULA_ERR_ARG;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (type == TULA_TYPE_F32) return dequantize_typed<float>(codes, scales, rows, cols, out, s);
    if (type == TULA_TYPE_BF16) return dequantize_typed<__nv_bfloat16>(codes, scales, rows, cols, out, s);
    return dequantize_typed<__half>(codes, scales, rows, cols, out, s);
}

int tula_mx_matmul(const void *a_codes, const void *a_scales, const void *b_codes, const void *b_scales, int64_t M, int64_t N,
                   int64_t K, void *out, int out_type, void *stream) {
    if (!good_type(out_type) || tiles_of(M, K) < 0 || tiles_of(N, K) < 0 || tiles_of(M, N) < 0) return TULA_ERR_ARG;
    if (M == 0 || N == 0) return TULA_OK;
    if (!out || !aligned(out, type_size(out_type))) return TULA_ERR_ARG;
    if (K && (!a_codes || !a_scales || !b_codes || !b_scales || !aligned(a_codes, 16) || !aligned(a_scales, 16) ||
              !aligned(b_codes, 16) || !aligned(b_scales, 16)))
        return TULA_ERR_ARG;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (out_type == TULA_TYPE_F32) return matmul_typed<float>(a_codes, a_scales, b_codes, b_scales, M, N, K, out, s);
    if (out_type == TULA_TYPE_BF16) return matmul_typed<__nv_bfloat16>(a_codes, a_scales, b_codes, b_scales, M, N, K, out, s);
    return matmul_typed<__half>(a_codes, a_scales, b_codes, b_scales, M, N, K, out, s);
}

int tula_mx_check_wait_timeout(void *stream) {
    return tula::launch(k_mx_wait_check, dim3(1), 32, 0, static_cast<cudaStream_t>(stream), 1);
}

int tula_mx_error(void *stream, int *error_out) {
    if (!error_out) return TULA_ERR_ARG;
    void *p = nullptr;
    unsigned v = 0;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    cudaError_t e = cudaGetSymbolAddress(&p, g_mx_error);
    if (e == cudaSuccess) e = cudaMemcpyAsync(&v, p, sizeof(v), cudaMemcpyDeviceToHost, s);
    if (e == cudaSuccess) e = cudaMemsetAsync(p, 0, sizeof(v), s);
    if (e == cudaSuccess) e = cudaStreamSynchronize(s);
    if (e != cudaSuccess) return cuda_failed(e);
    *error_out = (int)v;
    return TULA_OK;
}

}  // extern "C"
