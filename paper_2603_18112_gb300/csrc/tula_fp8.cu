// 8-bit floating-point matrices (E4M3, E5M2) with a power of two for each block of 128, for sm_103a:
// quantisation, reading back, products.
#include "tula_elems.cuh"
#include "tula_products.cuh"

namespace {

// ----------------------------------------------------------------------------
// Elements
// ----------------------------------------------------------------------------

// The block's scale byte from the bits of its largest magnitude (as fp32): the least power of two that
// brings it to at most 1.75 * 2^8 (E4M3's largest, 448) or 1.75 * 2^15 (E5M2's, 57344), so that no
// element is clipped.
template <bool E5>
__device__ __forceinline__ unsigned scale_byte(unsigned top) {
    const int e = (int)(top >> 23), s = e - (E5 ? 15 : 8) + ((top & 0x7fffffu) > 0x600000u);
    return e == 255 ? 255u : (unsigned)max(s, 0);
}
// What its elements are multiplied by: 2^(127 - s), exact (s is at most 247); 0 for a block that is NaN,
// whose codes are 0.
__device__ __forceinline__ float inverse_scale(unsigned s) { return s == 255u ? 0.f : __uint_as_float((254u - s) << 23); }

// Four elements' codes, the first in the lowest byte.
template <bool E5>
__device__ __forceinline__ unsigned codes4(float a, float b, float c, float d) {
    unsigned short lo, hi;
    if (E5) {
        asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
        asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
    } else {
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
    }
    return (unsigned)lo | (unsigned)hi << 16;
}

// ----------------------------------------------------------------------------
// Quantisation
// ----------------------------------------------------------------------------
//
// One CTA per 128 x 128 tile of x, which holds 128 blocks of its rows and of its columns, or is one block
// (Square).  A thread takes 32 bytes of a row at a time; the lanes that share a row find its largest
// magnitude together.  The transpose reads the tile again from shared memory, four lanes to a word's columns
// (one column of fp32, two of others), 32 rows each: they find the columns' largest magnitudes by two
// exchanges and write 128 bytes of codes to each column, so that one barrier is enough.  (With the tops and
// codes of columns by way of shared memory and two barriers more, 8192 x 4096 bf16 took 29 us in both forms
// instead of 23.)  fp32 rows off 32-byte boundaries come word by word, a warp to a row, and through
// shared memory too.  HBM bounds it: 2 or 4 bytes in and one out per element and form.

struct QuantArgs {
    const void *x;
    long long rows, cols, stride;
    unsigned char *codes, *scales, *codes_t, *scales_t;
    int tiles_c, tiles_r;  // of 128
};

template <typename T>
struct Shape {
    static constexpr int kElems = 32 / (int)sizeof(T);     // of a row, that a thread takes at a time
    static constexpr int kLanes = kTile / kElems;          // to a row
    static constexpr int kThreads = sizeof(T) == 4 ? 512 : 256;
    static constexpr int kCtas = sizeof(T) == 4 ? 2 : 4;   // an SM, that registers are left for
    static constexpr int kRows = kThreads / kLanes;        // at a time: 32
    static constexpr int kSide = kTile * (int)sizeof(T) / 4;  // words of a tile's row
    static constexpr int kCols = 4 / (int)sizeof(T);       // columns of a word
    static constexpr int kSmem = kTile * kTile * (int)sizeof(T);
    static_assert(kThreads == kSide * 4 && kRows == 32, "a column block is one thread's");
};

// Where 16-byte chunk `chunk` of a row of the tile lies in shared memory: so that neither the stores of
// parts nor the column reads (eight words of each of four rows, 32 rows apart) meet in a bank.
__device__ __forceinline__ int chunk_place(int row, int chunk) { return chunk ^ (chunk >> 3 & 1) ^ (row >> 5) << 1; }

// The largest magnitude of a word's elements so far, as fp32 bits (16-bit types: of both halves).
template <typename T>
__device__ __forceinline__ unsigned whole_top(unsigned top) {
    top &= sizeof(T) == 4 ? 0x7fffffffu : 0x7fff7fffu;
    return sizeof(T) == 4 ? top : top_bits<T>(max(top & 0xffffu, top >> 16));
}

// A scale byte and, after a row's last block, zeros for those that its tile of four has beyond it.
__device__ __forceinline__ void put_scale(unsigned char *scales, int row, long long tile_row, int block, int blocks, unsigned s) {
    unsigned char *to = scales + ((size_t)tile_row * ((blocks + 3) >> 2) + (block >> 2)) * kScaleTile + (row & 31) * 16 + (row >> 5) * 4;
    to[block & 3] = (unsigned char)s;
    if (block == blocks - 1)
        for (int k = (block & 3) + 1; k < 4; ++k) to[k] = 0;
}

template <typename T, bool E5, bool Aligned, bool Square, bool Rows, bool Cols>
__global__ void __launch_bounds__(Shape<T>::kThreads, Shape<T>::kCtas) k_quantize8(const QuantArgs a) {
    using S = Shape<T>;
    extern __shared__ __align__(16) unsigned tile[];  // Cols, or fp32 word by word
    __shared__ unsigned tops[S::kThreads / 32];
    let_next_start();
    wait_for_previous();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int tr = blockIdx.x / a.tiles_c, tc = blockIdx.x % a.tiles_c;
    const long long r0 = (long long)tr * kTile, c0 = (long long)tc * kTile;
    const int sub = tid % S::kLanes, row0 = tid / S::kLanes;
    const unsigned long long begin = reinterpret_cast<unsigned long long>(a.x);
    const unsigned long long end = begin + ((unsigned long long)(a.rows - 1) * a.stride + a.cols) * sizeof(T);
    constexpr bool kByWord = sizeof(T) == 4 && !Aligned, kStaged = Cols || kByWord;
    unsigned w[4][8], top_all = 0;
    const bool inner = c0 + kTile <= a.cols && (Aligned ? r0 + kTile <= a.rows : tr > 0 && r0 + kTile < a.rows);
    if constexpr (kByWord) {
        // words lane + 32 k of rows warp + 16 i
        const unsigned *p = static_cast<const unsigned *>(a.x) + (r0 + warp) * a.stride + c0 + lane;
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                unsigned &v = w[i >> 1][4 * (i & 1) + k];
                v = 0;
                if (inner || (r0 + warp + 16 * i < a.rows && c0 + lane + 32 * k < a.cols)) v = __ldcs(p + 16 * i * a.stride + 32 * k);
            }
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int r = warp + 16 * i, c = lane + 32 * k;
                const unsigned v = w[i >> 1][4 * (i & 1) + k];
                if (Square) top_all = larger<T>(top_all, v);
                tile[r * S::kSide + 4 * chunk_place(r, c >> 2) + (c & 3)] = v;
            }
    } else {
        const T *p0 = static_cast<const T *>(a.x) + (r0 + row0) * a.stride + c0 + S::kElems * sub;
        if (inner) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                load_part<T, S::kElems, Aligned>(w[i], p0 + i * 32 * a.stride, true, S::kElems, begin, end);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                load_part<T, S::kElems, Aligned>(w[i], p0 + i * 32 * a.stride, false,
                                                 r0 + row0 + 32 * i < a.rows ? a.cols - c0 - S::kElems * sub : 0, begin, end);
        }
        if (Square)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int k = 0; k < 8; ++k) top_all = larger<T>(top_all, w[i][k]);
        if (Cols)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int k = 0; k < 2; ++k)
                    *reinterpret_cast<uint4 *>(&tile[(row0 + 32 * i) * S::kSide + 4 * chunk_place(row0 + 32 * i, sub * 2 + k)]) =
                        make_uint4(w[i][4 * k], w[i][4 * k + 1], w[i][4 * k + 2], w[i][4 * k + 3]);
    }
    if (Square) {
        top_all = __reduce_max_sync(kFull, whole_top<T>(top_all));
        if (lane == 0) tops[warp] = top_all;
    }
    if (Square || kStaged) __syncthreads();
    unsigned s_all = 0;
    if (Square) {
        top_all = tops[0];
#pragma unroll
        for (int k = 1; k < S::kThreads / 32; ++k) top_all = max(top_all, tops[k]);
        s_all = scale_byte<E5>(top_all);
    }
    if (Rows && kByWord) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const uint4 q = *reinterpret_cast<const uint4 *>(
                    &tile[(row0 + 32 * i) * S::kSide + 4 * chunk_place(row0 + 32 * i, sub * 2 + k)]);
                w[i][4 * k] = q.x, w[i][4 * k + 1] = q.y, w[i][4 * k + 2] = q.z, w[i][4 * k + 3] = q.w;
            }
    }
    if (Rows) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = row0 + 32 * i;
            unsigned s = s_all;
            if (!Square) {
                unsigned top = 0;
#pragma unroll
                for (int k = 0; k < 8; ++k) top = larger<T>(top, w[i][k]);
                top = whole_top<T>(top);
#pragma unroll
                for (int o = 1; o < S::kLanes; o *= 2) top = max(top, __shfl_xor_sync(kFull, top, o));
                s = scale_byte<E5>(top);
            }
            const float f = inverse_scale(s);
            const bool there = inner || r0 + row < a.rows;
            unsigned q[S::kElems / 4];
#pragma unroll
            for (int k = 0; k < S::kElems / 8; ++k) {
                float x[8];
                floats8<T>(x, w[i] + k * 2 * sizeof(T));
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = __fmul_rn(x[j], f);
                q[2 * k] = codes4<E5>(x[0], x[1], x[2], x[3]);
                q[2 * k + 1] = codes4<E5>(x[4], x[5], x[6], x[7]);
            }
            if (s == 255u)
#pragma unroll
                for (int k = 0; k < S::kElems / 4; ++k) q[k] = 0;
            if (sub == 0) put_scale(a.scales, row, tr, tc, a.tiles_c, there ? s : 0u);
            if (there) {
                unsigned char *to = a.codes + (size_t)(r0 + row) * a.tiles_c * kTile + c0 + S::kElems * sub;
                if (sizeof(T) == 2)
                    *reinterpret_cast<uint4 *>(to) = make_uint4(q[0], q[1], q[S::kElems / 4 - 2], q[S::kElems / 4 - 1]);
                else
                    *reinterpret_cast<uint2 *>(to) = make_uint2(q[0], q[1]);
            }
        }
    }
    if (!Cols) return;
    const int c = tid >> 2, rb = tid & 3;  // word c of 32 rows
    const int at = 4 * chunk_place(32 * rb, c >> 2) + (c & 3);
    unsigned v[32], top = 0;
#pragma unroll
    for (int k = 0; k < 32; ++k) {
        v[k] = tile[(32 * rb + k) * S::kSide + at];
        if (!Square) top = larger<T>(top, v[k]);
    }
    top &= sizeof(T) == 4 ? 0x7fffffffu : 0x7fff7fffu;
#pragma unroll
    for (int h = 0; h < S::kCols; ++h) {
        const int col = S::kCols * c + h;
        unsigned s = s_all;
        if (!Square) {
            unsigned t = sizeof(T) == 4 ? top : top_bits<T>(h ? top >> 16 : top & 0xffffu);
            t = max(t, __shfl_xor_sync(kFull, t, 1));
            t = max(t, __shfl_xor_sync(kFull, t, 2));
            s = scale_byte<E5>(t);
        }
        const float f = inverse_scale(s);
        unsigned q[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            float x[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (sizeof(T) == 4) {
                    x[j] = __uint_as_float(v[4 * k + j]);
                } else {
                    const float2 p = pair_of<T>(v[4 * k + j]);
                    x[j] = h ? p.y : p.x;
                }
                x[j] = __fmul_rn(x[j], f);
            }
            q[k] = s == 255u ? 0u : codes4<E5>(x[0], x[1], x[2], x[3]);
        }
        const bool there = c0 + col < a.cols;
        if (rb == 0) put_scale(a.scales_t, col, tc, tr, a.tiles_r, there ? s : 0u);
        if (there) {
            uint4 *to = reinterpret_cast<uint4 *>(a.codes_t + (size_t)(c0 + col) * a.tiles_r * kTile + r0 + 32 * rb);
            to[0] = make_uint4(q[0], q[1], q[2], q[3]);
            to[1] = make_uint4(q[4], q[5], q[6], q[7]);
        }
    }
}

// ----------------------------------------------------------------------------
// Reading back
// ----------------------------------------------------------------------------

// Two codes' values (fp16 holds all of either format).
template <bool E5>
__device__ __forceinline__ float2 code_pair(unsigned two) {
    unsigned h;
    if (E5)
        asm("cvt.rn.f16x2.e5m2x2 %0, %1;" : "=r"(h) : "h"((unsigned short)two));
    else
        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((unsigned short)two));
    __half2 v;
    memcpy(&v, &h, 4);
    return __half22float2(v);
}

template <bool E5>
struct Read8 {
    using Eight = uint2;
    static constexpr int kBlock = 128;
    static __device__ __forceinline__ size_t pitch(int tiles_c) { return (size_t)tiles_c * kTile; }
    template <typename I>
    static __device__ __forceinline__ unsigned scale_at(const DequantArgs &a, I r, I c) {
        return __ldcg(a.scales + ((size_t)(r / kTile) * ((a.tiles_c + 3) >> 2) + c / 512) * kScaleTile + (r & 31) * 16 +
                      (r & 127) / 32 * 4 + (c & 511) / 128);
    }
    template <bool Easy, typename I>
    static __device__ __forceinline__ uint2 fetch(const unsigned char *row, I c) {
        if (Easy) return __ldcg(reinterpret_cast<const uint2 *>(row + c));
        const unsigned *w = reinterpret_cast<const unsigned *>(row) + c / 4;
        const int in = (int)(c & 3);
        const uint2 q = make_uint2(__ldcg(w), __ldcg(w + 1));
        if (!in) return q;
        return make_uint2(__funnelshift_r(q.x, q.y, 8 * in), __funnelshift_r(q.y, __ldcg(w + 2), 8 * in));
    }
    template <typename T>
    static __device__ __forceinline__ void values(T (&y)[8], uint2 q, unsigned s0, unsigned s1, int first) {
        const float f0 = scale_value(s0), f1 = scale_value(s1);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float2 v = code_pair<E5>((k < 2 ? q.x : q.y) >> 16 * (k & 1));
            put(&y[2 * k], __fmul_rn(v.x, 2 * k < first ? f0 : f1));
            put(&y[2 * k + 1], __fmul_rn(v.y, 2 * k + 1 < first ? f0 : f1));
        }
    }
    template <typename I>
    static __device__ __forceinline__ float one(const unsigned char *row, I c) {
        return code_pair<E5>(__ldcg(row + c)).x;
    }
};

// ----------------------------------------------------------------------------
// Host side
// ----------------------------------------------------------------------------

template <typename T, bool E5, bool Aligned, bool Square>
int launch_quantize(const QuantArgs &a, unsigned grid, cudaStream_t s) {
    static std::atomic<uint64_t> done[3];
    const int which = a.codes && a.codes_t ? 0 : a.codes ? 1 : 2;
    void (*k)(const QuantArgs) = which == 0   ? k_quantize8<T, E5, Aligned, Square, true, true>
                                 : which == 1 ? k_quantize8<T, E5, Aligned, Square, true, false>
                                              : k_quantize8<T, E5, Aligned, Square, false, true>;
    const int smem = a.codes_t || (sizeof(T) == 4 && !Aligned) ? Shape<T>::kSmem : 0;
    const int rc = allow_smem((const void *)k, smem, &done[which]);
    if (rc) return rc;
    return tula::launch(k, dim3(grid), Shape<T>::kThreads, smem, s, 1, a);
}
template <typename T, bool E5>
int quantize_typed(const QuantArgs &a, unsigned grid, bool square, cudaStream_t s) {
    const size_t both = reinterpret_cast<uintptr_t>(a.x) | (a.rows > 1 ? (size_t)a.stride * sizeof(T) : 0);
    if (both % 32 == 0) return square ? launch_quantize<T, E5, true, true>(a, grid, s) : launch_quantize<T, E5, true, false>(a, grid, s);
    return square ? launch_quantize<T, E5, false, true>(a, grid, s) : launch_quantize<T, E5, false, false>(a, grid, s);
}

inline bool good_code(int code) { return code == TULA_FP8_E4M3 || code == TULA_FP8_E5M2; }

// A matrix in memory of the caller's: scales, then codes.
struct Held {
    unsigned char *scales = nullptr, *codes = nullptr;
};
// The next one of a run of them; false beyond what one may have.
bool take(unsigned char *&at, long long rows, long long cols, bool wanted, Held &h) {
    size_t codes = 0, scales = 0;
    if (!wanted) return true;
    if (tula_fp8_size(rows, cols, &codes, &scales) != TULA_OK) return false;
    if (rows && cols) h.scales = at, h.codes = at + scales;
    at += scales + codes;
    return true;
}
int quantize(const tula_fp8_operand &x, long long rows, long long cols, int code, int square, const Held &h, const Held &t, void *stream) {
    if (!h.codes && !t.codes) return TULA_OK;  // not wanted, or empty
    if (x.transposed)
        return tula_fp8_quantize(x.data, x.type, cols, rows, x.stride, code, square, t.codes, t.scales, h.codes, h.scales, stream);
    return tula_fp8_quantize(x.data, x.type, rows, cols, x.stride, code, square, h.codes, h.scales, t.codes, t.scales, stream);
}
bool good_operand(const tula_fp8_operand *x, long long rows, long long cols) {
    return x && good_type(x->type) && x->stride >= (x->transposed ? rows : cols) &&
           (!rows || !cols || (x->data && aligned(x->data, type_size(x->type))));
}

}  // namespace

extern "C" {

int tula_fp8_size(int64_t rows, int64_t cols, size_t *code_bytes, size_t *scale_bytes) {
    if (!code_bytes || !scale_bytes || tiles_of(rows, cols) < 0) return TULA_ERR_ARG;
    *code_bytes = (size_t)rows * (size_t)up(cols, kTile) * kTile;
    *scale_bytes = (size_t)up(rows, kTile) * (size_t)up(cols, 4 * kTile) * kScaleTile;
    return TULA_OK;
}

int tula_fp8_quantize(const void *x, int type, int64_t rows, int64_t cols, int64_t stride, int code, int square, void *codes,
                      void *scales, void *codes_t, void *scales_t, void *stream) {
    const long long tiles = tiles_of(rows, cols);
    if (!good_type(type) || !good_code(code) || tiles < 0 || stride < cols) return TULA_ERR_ARG;
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
    const unsigned grid = (unsigned)tiles;
    const bool e5 = code == TULA_FP8_E5M2, sq = square != 0;
    if (type == TULA_TYPE_F32) return e5 ? quantize_typed<float, true>(a, grid, sq, s) : quantize_typed<float, false>(a, grid, sq, s);
    if (type == TULA_TYPE_BF16)
        return e5 ? quantize_typed<__nv_bfloat16, true>(a, grid, sq, s) : quantize_typed<__nv_bfloat16, false>(a, grid, sq, s);
    return e5 ? quantize_typed<__half, true>(a, grid, sq, s) : quantize_typed<__half, false>(a, grid, sq, s);
}

int tula_fp8_dequantize(const void *codes, const void *scales, int64_t rows, int64_t cols, int code, void *out, int type, void *stream) {
    if (!good_code(code)) return TULA_ERR_ARG;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return code == TULA_FP8_E5M2 ? dequantize<Read8<true>>(codes, scales, rows, cols, out, type, s)
                                 : dequantize<Read8<false>>(codes, scales, rows, cols, out, type, s);
}

int tula_fp8_matmul(const void *a_codes, const void *a_scales, int a_code, const void *b_codes, const void *b_scales, int b_code,
                    int64_t M, int64_t N, int64_t K, void *out, int out_type, void *stream) {
    if (!good_code(a_code) || !good_code(b_code)) return TULA_ERR_ARG;
    return matmul<Codes8>({a_codes, a_scales, a_code}, {b_codes, b_scales, b_code}, M, N, K, out, out_type,
                          static_cast<cudaStream_t>(stream));
}

int tula_fp8_linear(const tula_fp8_operand *x, const tula_fp8_operand *w, int64_t M, int64_t N, int64_t K, int code, int need_dx,
                    int need_dw, void *kept, void *temp, void *y, void *stream) {
    if (!good_operand(x, M, K) || !good_operand(w, N, K) || !good_code(code) || tiles_of(M, K) < 0 || tiles_of(N, K) < 0 ||
        tiles_of(M, N) < 0 || !aligned(kept, 16) || !aligned(temp, 16) || (M && N && (!y || !aligned(y, type_size(x->type)))))
        return TULA_ERR_ARG;
    unsigned char *k = static_cast<unsigned char *>(kept), *t = static_cast<unsigned char *>(temp);
    Held xt, wt, qx, qw;
    if (!take(k, K, M, need_dw, xt) || !take(k, K, N, need_dx, wt) || !take(t, M, K, true, qx) || !take(t, N, K, true, qw)) return TULA_ERR_ARG;
    if ((k > static_cast<unsigned char *>(kept) && !kept) || (t > static_cast<unsigned char *>(temp) && !temp)) return TULA_ERR_WORKSPACE;
    int rc = quantize(*x, M, K, code, 0, qx, xt, stream);
    if (!rc) rc = quantize(*w, N, K, code, 1, qw, wt, stream);
    if (!rc) rc = tula_fp8_matmul(qx.codes, qx.scales, code, qw.codes, qw.scales, code, M, N, K, y, x->type, stream);
    return rc;
}

int tula_fp8_linear_backward(const tula_fp8_operand *dy, int64_t M, int64_t N, int64_t K, int code, int grad_code, const void *kept,
                             void *temp, void *dx, int dx_type, void *dw, int dw_type, int need_dx, int need_dw, void *stream) {
    if (!good_operand(dy, M, N) || !good_code(code) || !good_code(grad_code) || !good_type(dx_type) || !good_type(dw_type) ||
        tiles_of(M, K) < 0 || tiles_of(N, K) < 0 || tiles_of(M, N) < 0 || !aligned(kept, 16) || !aligned(temp, 16) ||
        (need_dx && M && K && (!dx || !aligned(dx, type_size(dx_type)))) || (need_dw && N && K && (!dw || !aligned(dw, type_size(dw_type)))))
        return TULA_ERR_ARG;
    unsigned char *k = static_cast<unsigned char *>(const_cast<void *>(kept)), *t = static_cast<unsigned char *>(temp);
    Held xt, wt, rows, cols;
    if (!take(k, K, M, need_dw, xt) || !take(k, K, N, need_dx, wt) || !take(t, M, N, need_dx, rows) || !take(t, N, M, need_dw, cols))
        return TULA_ERR_ARG;
    if ((k > static_cast<unsigned char *>(const_cast<void *>(kept)) && !kept) || (t > static_cast<unsigned char *>(temp) && !temp))
        return TULA_ERR_WORKSPACE;
    int rc = quantize(*dy, M, N, grad_code, 0, rows, cols, stream);
    if (!rc && need_dx)  // dy [M, N] (w^T [K, N])^T
        rc = tula_fp8_matmul(rows.codes, rows.scales, grad_code, wt.codes, wt.scales, code, M, K, N, dx, dx_type, stream);
    if (!rc && need_dw)  // dy^T [N, M] (x^T [K, M])^T
        rc = tula_fp8_matmul(cols.codes, cols.scales, grad_code, xt.codes, xt.scales, code, N, K, M, dw, dw_type, stream);
    return rc;
}

int tula_fp8_check_wait_timeout(void *stream) { return check_wait_timeout(stream); }

int tula_fp8_error(void *stream, int *error_out) { return read_error(stream, error_out); }

}  // extern "C"
