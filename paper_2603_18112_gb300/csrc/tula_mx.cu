// Microscaled 4-bit matrices (MXFP4) for sm_103a: quantisation, reading back, products.
#include "tula_elems.cuh"
#include "tula_products.cuh"

namespace {

constexpr int kBlock = 32;          // elements that share a scale

// ----------------------------------------------------------------------------
// Elements
// ----------------------------------------------------------------------------

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
            load_part<T, Part<T>::kElems, Aligned>(w[i], p0 + i * (kThreads / kSubs) * a.stride, true, Part<T>::kElems, begin, end);
    } else {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const long long r = r0 + i * (kThreads / kSubs) + tid / kSubs;
            load_part<T, Part<T>::kElems, Aligned>(w[i], p0 + i * (kThreads / kSubs) * a.stride, false,
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

// Two codes' values.
__device__ __forceinline__ float2 code_pair(unsigned byte) {
    unsigned h;
    asm("{\n.reg .b8 b, u1, u2, u3;\nmov.b32 {b, u1, u2, u3}, %1;\ncvt.rn.f16x2.e2m1x2 %0, b;\n}\n" : "=r"(h) : "r"(byte));
    __half2 v;
    memcpy(&v, &h, 4);
    return __half22float2(v);
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

struct Read4 {
    using Eight = unsigned;
    static constexpr int kBlock = ::kBlock;
    static __device__ __forceinline__ size_t pitch(int tiles_c) { return (size_t)tiles_c * (kTile / 2); }
    template <typename I>
    static __device__ __forceinline__ unsigned scale_at(const DequantArgs &a, I r, I c) {
        return __ldcg(a.scales + ((size_t)(r / kTile) * a.tiles_c + c / kTile) * kScaleTile + (r & 31) * 16 + (r & 127) / 32 * 4 +
                      (c & 127) / kBlock);
    }
    template <bool Easy, typename I>
    static __device__ __forceinline__ unsigned fetch(const unsigned char *row, I c) {
        const unsigned *w = reinterpret_cast<const unsigned *>(row) + c / 8;
        const unsigned q = __ldcg(w);
        const int in = Easy ? 0 : (int)(c & 7);
        return in ? __funnelshift_r(q, __ldcg(w + 1), 4 * in) : q;
    }
    template <typename T>
    static __device__ __forceinline__ void values(T (&y)[8], unsigned q, unsigned s0, unsigned s1, int first) {
        scaled_values(y, q, s0, s1, first);
    }
    template <typename I>
    static __device__ __forceinline__ float one(const unsigned char *row, I c) {
        const unsigned byte = __ldcg(row + c / 2);
        return code_pair(c & 1 ? byte >> 4 : byte & 15u).x;
    }
};

// ----------------------------------------------------------------------------
// Host side
// ----------------------------------------------------------------------------

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
    return dequantize<Read4>(codes, scales, rows, cols, out, type, static_cast<cudaStream_t>(stream));
}

int tula_mx_matmul(const void *a_codes, const void *a_scales, const void *b_codes, const void *b_scales, int64_t M, int64_t N,
                   int64_t K, void *out, int out_type, void *stream) {
    return matmul<Codes4>({a_codes, a_scales, 0}, {b_codes, b_scales, 0}, M, N, K, out, out_type, static_cast<cudaStream_t>(stream));
}

int tula_mx_check_wait_timeout(void *stream) { return check_wait_timeout(stream); }

int tula_mx_error(void *stream, int *error_out) { return read_error(stream, error_out); }

}  // extern "C"
