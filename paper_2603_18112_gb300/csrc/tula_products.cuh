// Products of matrices in narrow floating point whose blocks share scales: out = A B^T on the tensor
// cores, which apply the scales.  Included by the translation units of the formats.
#pragma once

#include "tula_tc.cuh"

namespace {

constexpr int kScaleTile = 512;     // its bytes: 128 rows by 4 blocks

// ----------------------------------------------------------------------------
// Products: tcgen05 with block scales
// ----------------------------------------------------------------------------
//
// out = A B^T by tiles of 128 rows of one operand (P, the instruction's M) by NT rows of the other
// (Q, its N).  Codes come by TMA, 128 bytes of a row a stage, scales by bulk copies; one thread moves a
// stage's scales to tensor memory and issues its instructions, 32 bytes of a row each; accumulators
// lie in tensor memory and four warps read them back.

// 4-bit codes with a scale for each block of 32: a stage has 256 columns and two tiles of scales, an
// instruction 64 columns and two scales a row.
struct Codes4 {
    static constexpr int kScaleTiles = 2;  // of a stage, at most
    static __device__ __forceinline__ int stages(int tiles_k) { return (tiles_k + 1) / 2; }
    static __device__ __forceinline__ int scale_tile(int k) { return 2 * k; }  // a stage's first
    static __device__ __forceinline__ int tiles(int k, int tiles_k) { return min(2, tiles_k - 2 * k); }  // that it has
    static __device__ __forceinline__ int scale_pitch(int tiles_k) { return tiles_k; }
    static __device__ __forceinline__ int tile_of(int j) { return j >> 1; }  // instruction j's scales
    static __device__ __forceinline__ int scale_id(int j, int) { return 2 * (j & 1); }
};
// 8-bit codes with a scale for each block of 128: a stage is one block and an instruction a quarter of it;
// a tile of scales serves four stages.
struct Codes8 {
    static constexpr int kScaleTiles = 1;
    static __device__ __forceinline__ int stages(int tiles_k) { return tiles_k; }
    static __device__ __forceinline__ int scale_tile(int k) { return k >> 2; }
    static __device__ __forceinline__ int tiles(int, int) { return 1; }
    static __device__ __forceinline__ int scale_pitch(int tiles_k) { return (tiles_k + 3) >> 2; }
    static __device__ __forceinline__ int tile_of(int) { return 0; }
    static __device__ __forceinline__ int scale_id(int, int k) { return k & 3; }
};

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
// The instruction's descriptor but for the operands' formats: E8M0 scales, M, N.
__host__ __device__ constexpr uint32_t mma_desc(int m, int n) {
    return (uint32_t)(n >> 3) << 17 | 1u << 23 | (uint32_t)(m >> 7) << 27;
}
// Which of a word's four scales the instruction takes, of both operands (of two the first).
__device__ __forceinline__ uint32_t with_scale_id(uint32_t desc, uint32_t id) {
    return desc | id << 4 | id << 29;
}

__device__ __forceinline__ void copy_scales(uint32_t tmem, uint64_t desc) {
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}
template <class C>
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, bool add) {
    if (std::is_same<C, Codes4>::value)
        asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %6, 0;\n"
                     "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n}\n" ::"r"(d),
                     "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"((unsigned)add)
                     : "memory");
    else
        asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %6, 0;\n"
                     "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n}\n" ::"r"(d),
                     "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"((unsigned)add)
                     : "memory");
}
struct MatmulArgs {
    const unsigned char *p_scales, *q_scales;
    void *out;
    long long P, Q;       // rows of each operand
    long long ld;         // elements of out from row to row
    int tiles_k;          // of 128 columns
    uint32_t formats;     // of the instruction's descriptor: P's, Q's
    int grid_q;           // tiles of the product along Q
    int split;            // CTAs of a cluster that share a tile's columns
};

template <class C, int NT, bool Swap>
struct MmaShape {
    static constexpr int kP = 128 * 128, kQ = NT * 128;                     // bytes of codes a stage
    static constexpr int kSP = C::kScaleTiles * kScaleTile, kSQ = kSP;
    static constexpr int kStage = (kP + kQ + kSP + kSQ + 1023) / 1024 * 1024;
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
template <class C, int NT, bool Swap, typename T>
__global__ void __launch_bounds__(kMmaThreads) k_matmul(const __grid_constant__ CUtensorMap map_p,
                                                        const __grid_constant__ CUtensorMap map_q, const MatmulArgs a) {
    using S = MmaShape<C, NT, Swap>;
    extern __shared__ __align__(16) unsigned tile[];
    __shared__ __align__(8) unsigned long long bars[2 * S::kStages + 1];
    __shared__ uint32_t tmem_at;
    __shared__ volatile int dead;
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(kFull, tid >> 5, 0);
    const uint32_t stages = (smem_addr(tile) + 1023) & ~1023u;
    const uint32_t full = smem_addr(bars), empty = full + 8 * S::kStages, done = empty + 8 * S::kStages;
    const int rank = blockIdx.x % a.split, t = blockIdx.x / a.split;
    const int tp = t / a.grid_q, tq = t % a.grid_q;
    const int all_k = C::stages(a.tiles_k), per = (all_k + a.split - 1) / a.split;
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
            const int tiles = C::tiles(k, a.tiles_k);  // scale tiles along the columns
            const size_t pitch = C::scale_pitch(a.tiles_k), first = C::scale_tile(k);
            if (elect_one()) {
                mbar_expect(bar, S::kP + S::kQ + 2 * tiles * kScaleTile);
                tma_load_2d(at, &map_p, k * 128, tp * 128, bar);
                tma_load_2d(at + S::kP, &map_q, k * 128, tq * NT, bar);
                bulk_load(at + S::kP + S::kQ, a.p_scales + (tp * pitch + first) * kScaleTile, tiles * kScaleTile, bar);
                // the scale tile that these rows of Q are in
                bulk_load(at + S::kP + S::kQ + S::kSP, a.q_scales + (tq * pitch + first) * kScaleTile, tiles * kScaleTile,
                          bar);
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
            const int tiles = C::tiles(k_begin + i, a.tiles_k);
            const uint64_t da = codes_desc(at), db = codes_desc(at + S::kP);
            if (elect_one()) {
#pragma unroll
                for (int j = 0; j < C::kScaleTiles; ++j) {
                    if (j == tiles) break;
                    copy_scales(tmem + S::kScaleP + 4 * j, scales_desc(sc + j * kScaleTile));
                    copy_scales(tmem + S::kScaleQ + 4 * j, scales_desc(sc + S::kSP + j * kScaleTile));
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (C::tile_of(j) == tiles) break;
                    mma<C>(tmem, da + 2 * j, db + 2 * j, with_scale_id(mma_desc(128, NT) | a.formats, C::scale_id(j, k_begin + i)),
                           tmem + S::kScaleP + 4 * C::tile_of(j), tmem + S::kScaleQ + 4 * C::tile_of(j), i > 0 || j > 0);
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
    static constexpr int kSA = 2 * kScaleTile, kSB = 4 * kScaleTile;  // (8 bits: half) the scales of all 256 rows of B
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
    uint32_t formats;
    int tiles_m, tiles_n;  // of 256
    int word;              // bytes that divide out's address and rows: 16 (stored by TMA), 8, 4 or 2
};

__device__ __forceinline__ void copy_scales_pair(uint32_t tmem, uint64_t desc) {
    asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}
template <class C>
__device__ __forceinline__ void mma_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, bool add) {
    if (std::is_same<C, Codes4>::value)
        asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %6, 0;\n"
                     "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n}\n" ::"r"(d),
                     "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"((unsigned)add)
                     : "memory");
    else
        asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %6, 0;\n"
                     "tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n}\n" ::"r"(d),
                     "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"((unsigned)add)
                     : "memory");
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

template <class C, typename T>
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
    const int n_k = C::stages(a.tiles_k);
    constexpr int kLoaded = Pair::kA + Pair::kB + 3 * C::kScaleTiles * kScaleTile;  // bytes of a stage, a CTA
    if (stages & 1023u) {  // no kernel that this may happen to has been seen
        if (tid == 0) atomicOr(&g_wait_error, 2u);
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
                    if (rank == 0) mbar_expect(full + 8 * s, 2 * kLoaded);  // both CTAs' copies
                    tma_load_pair(at, &map_a, k * 128, tm * 256 + rank * 128, bar);
                    tma_load_pair(at + Pair::kA, &map_b, k * 128, tn * 256 + rank * 128, bar);
                    tma_load_pair(at + Pair::kA + Pair::kB, &map_sa, C::scale_tile(k) * 128, tm * 2 + rank, bar);
                    tma_load_pair(at + Pair::kA + Pair::kB + Pair::kSA, &map_sb, C::scale_tile(k) * 128, tn * 2, bar);
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
                    const int tiles = C::tiles(k, a.tiles_k);
                    const uint64_t da = codes_desc(at), db = codes_desc(at + Pair::kA);
                    if (elect_one()) {
#pragma unroll
                        for (int j = 0; j < C::kScaleTiles; ++j) {
                            if (j == tiles) break;
                            copy_scales_pair(tmem + Pair::kScaleA + 4 * j, scales_desc(sc + j * kScaleTile));
#pragma unroll
                            for (int h = 0; h < 2; ++h)
                                copy_scales_pair(tmem + Pair::kScaleB + 8 * j + 4 * h,
                                                 scales_desc(sc + Pair::kSA + (C::kScaleTiles * h + j) * kScaleTile));
                        }
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            if (C::tile_of(j) == tiles) break;
                            mma_pair<C>(acc, da + 2 * j, db + 2 * j, with_scale_id(mma_desc(256, 256) | a.formats, C::scale_id(j, k)),
                                        tmem + Pair::kScaleA + 4 * C::tile_of(j), tmem + Pair::kScaleB + 8 * C::tile_of(j),
                                        k > 0 || j > 0);
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

// An operand: its codes, scales and their place in the instruction's descriptor (8 bits: 0 E4M3, 1 E5M2).
struct Operand {
    const void *codes, *scales;
    int format;
};
template <class C>
long long code_pitch(long long tiles_k) { return tiles_k * (C::kScaleTiles == 2 ? kTile / 2 : kTile); }
template <class C>
uint32_t formats_of(const Operand &first, const Operand &second) {
    return std::is_same<C, Codes4>::value ? 1u << 7 | 1u << 10 : (uint32_t)first.format << 7 | (uint32_t)second.format << 10;
}
// Codes in boxes of 128 bytes by box_rows rows.
template <class C>
bool codes_map(CUtensorMap *m, const void *codes, long long rows, int tiles_k, int box_rows) {
    const long long pitch = code_pitch<C>(tiles_k);
    return make_map(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, codes, rows, pitch, pitch, box_rows, 128, CU_TENSOR_MAP_SWIZZLE_128B);
}
// Scales, a row per 128 of the matrix, in boxes of a stage's tiles by box_rows.
template <class C>
bool scales_map(CUtensorMap *m, const void *scales, long long rows, int tiles_k, int box_rows) {
    const long long tiles = C::kScaleTiles == 2 ? tiles_k : up(tiles_k, 4);
    return make_map(m, CU_TENSOR_MAP_DATA_TYPE_UINT32, scales, up(rows, kTile), tiles * (kScaleTile / 4), tiles * kScaleTile, box_rows,
                    C::kScaleTiles * (kScaleTile / 4), CU_TENSOR_MAP_SWIZZLE_NONE);
}

template <class C, int NT, bool Swap, typename T>
int launch_matmul(const CUtensorMap &mp, const CUtensorMap &mq, const MatmulArgs &a, unsigned grid, cudaStream_t s) {
    using S = MmaShape<C, NT, Swap>;
    static std::atomic<uint64_t> done;
    const int rc = allow_smem((const void *)k_matmul<C, NT, Swap, T>, S::kSmem, &done);
    if (rc) return rc;
    return tula::launch(k_matmul<C, NT, Swap, T>, dim3(grid), kMmaThreads, S::kSmem, s, a.split, mp, mq, a);
}

template <class C, typename T>
int matmul_small(const Operand &p, const Operand &q, long long M, long long N, long long K, void *out, cudaStream_t s) {
    // The operand with few rows is the instruction's N, so that its 128 rows are not padding; N as small as
    // they are (16 x 4096 x 4096: 4.4 us with 32, 6.1 with 128; 48 x 4096 x 25088: 9.3 with 64, 10.0).
    const bool swap = M <= 128;
    MatmulArgs a;
    a.p_scales = static_cast<const unsigned char *>((swap ? q : p).scales);
    a.q_scales = static_cast<const unsigned char *>((swap ? p : q).scales);
    a.P = swap ? N : M;
    a.Q = swap ? M : N;
    a.ld = N;
    a.out = out;
    a.tiles_k = (int)up(K, kTile);
    a.formats = swap ? formats_of<C>(q, p) : formats_of<C>(p, q);
    const int nt = a.Q <= 32 ? 32 : a.Q <= 64 ? 64 : 128;
    a.grid_q = (int)up(a.Q, nt);
    const long long tiles = up(a.P, 128) * a.grid_q;
    // Few tiles: up to eight CTAs share one's columns while all are resident (two an SM), two stages at
    // least for each, or four where the sums that they exchange are as long (128 x 4096 x 4096: 8.3
    // us with four CTAs, 9.2 with eight; 1 x 4096 x 4096: 4.0 us with eight).
    const int least = nt >= 64 ? 8 : 4;
    a.split = 1;
    while (a.split < 8 && tiles * a.split * 2 <= 2 * 152 && (C::kScaleTiles == 2 ? up(a.tiles_k, 2) : a.tiles_k) >= least * a.split) a.split *= 2;
    if (tiles * a.split >= (1LL << 31)) return TULA_ERR_ARG;
    CUtensorMap mp, mq;
    std::memset(&mp, 0, sizeof(mp));
    std::memset(&mq, 0, sizeof(mq));
    if (K && (!codes_map<C>(&mp, (swap ? q : p).codes, a.P, a.tiles_k, 128) ||
              !codes_map<C>(&mq, (swap ? p : q).codes, a.Q, a.tiles_k, nt)))
        return cuda_failed(cudaErrorInvalidValue);
    const unsigned grid = (unsigned)(tiles * a.split);
    if (swap)
        return nt == 32 ? launch_matmul<C, 32, true, T>(mp, mq, a, grid, s)
               : nt == 64 ? launch_matmul<C, 64, true, T>(mp, mq, a, grid, s)
                          : launch_matmul<C, 128, true, T>(mp, mq, a, grid, s);
    return nt == 32 ? launch_matmul<C, 32, false, T>(mp, mq, a, grid, s)
           : nt == 64 ? launch_matmul<C, 64, false, T>(mp, mq, a, grid, s)
                      : launch_matmul<C, 128, false, T>(mp, mq, a, grid, s);
}

template <class C, typename T>
int matmul_large(const Operand &p, const Operand &q, long long M, long long N, long long K, void *out, cudaStream_t s) {
    PairArgs a;
    a.out = out;
    a.M = M;
    a.N = N;
    a.tiles_k = (int)up(K, kTile);
    a.formats = formats_of<C>(p, q);
    a.tiles_m = (int)up(M, 256);
    a.tiles_n = (int)up(N, 256);
    const unsigned long long both = reinterpret_cast<unsigned long long>(out) | (unsigned long long)(N * (long long)sizeof(T));
    a.word = both % 16 == 0 ? 16 : both % 8 == 0 ? 8 : both % 4 == 0 ? 4 : 2;
    CUtensorMap ma, mb, sa, sb, mo;
    std::memset(&mo, 0, sizeof(mo));
    const CUtensorMapDataType type = sizeof(T) == 4 ? CU_TENSOR_MAP_DATA_TYPE_UINT32 : CU_TENSOR_MAP_DATA_TYPE_UINT16;
    if (!codes_map<C>(&ma, p.codes, M, a.tiles_k, 128) || !codes_map<C>(&mb, q.codes, N, a.tiles_k, 128) ||
        !scales_map<C>(&sa, p.scales, M, a.tiles_k, 1) || !scales_map<C>(&sb, q.scales, N, a.tiles_k, 2) ||
        (a.word == 16 && !make_map(&mo, type, out, M, N, N * (long long)sizeof(T), 32, 128 / (int)sizeof(T), CU_TENSOR_MAP_SWIZZLE_128B)))
        return cuda_failed(cudaErrorInvalidValue);
    static std::atomic<uint64_t> done;
    const int rc = allow_smem((const void *)k_matmul_pair<C, T>, Pair::kSmem, &done);
    if (rc) return rc;
    const long long tiles = (long long)a.tiles_m * a.tiles_n, pairs = std::max(1, sm_count() / 2);
    return tula::launch(k_matmul_pair<C, T>, dim3((unsigned)(2 * std::min(tiles, pairs))), kPairThreads, Pair::kSmem, s, 1, ma, mb, sa,
                        sb, mo, a);
}

template <class C, typename T>
int matmul_typed(const Operand &p, const Operand &q, long long M, long long N, long long K, void *out, cudaStream_t s) {
    // Pairs of CTAs from 32 tiles of 256 x 256 on: 1024 x 2048 x 4096 takes 9.5 us (10.3 by tiles of 128),
    // 2048 x 4096 x 512 8.5 (10.6); 1024 x 1024 x 4096, 16 tiles, 9.4 (9.1).
    if (K > 0 && M > 128 && N > 128 && up(M, 256) * up(N, 256) >= 32)
        return matmul_large<C, T>(p, q, M, N, K, out, s);
    return matmul_small<C, T>(p, q, M, N, K, out, s);
}

template <class C>
int matmul(const Operand &p, const Operand &q, long long M, long long N, long long K, void *out, int out_type, cudaStream_t s) {
    if (!good_type(out_type) || tiles_of(M, K) < 0 || tiles_of(N, K) < 0 || tiles_of(M, N) < 0) return TULA_ERR_ARG;
    if (M == 0 || N == 0) return TULA_OK;
    if (!out || !aligned(out, type_size(out_type))) return TULA_ERR_ARG;
    if (K && (!p.codes || !p.scales || !q.codes || !q.scales || !aligned(p.codes, 16) || !aligned(p.scales, 16) ||
              !aligned(q.codes, 16) || !aligned(q.scales, 16)))
        return TULA_ERR_ARG;
    if (out_type == TULA_TYPE_F32) return matmul_typed<C, float>(p, q, M, N, K, out, s);
    if (out_type == TULA_TYPE_BF16) return matmul_typed<C, __nv_bfloat16>(p, q, M, N, K, out, s);
    return matmul_typed<C, __half>(p, q, M, N, K, out, s);
}

}  // namespace
